"""Acceptance on trees where p or q holds what no distribution has: a row with a NaN or +inf gives no token, however its drafts fared."""
import numpy as np
import pytest
import torch

from test_gpu_tree_accept import Round, kb  # noqa: F401

pytestmark = pytest.mark.gpu


def _rejecting(seed, V, drawn, requests):
    """Requests whose row 0 has three children, none of which can be kept: p has nothing at their tokens."""
    r = Round(seed, [[-1, 0, 0, 0, 1]] * requests, V, drawn)
    for b in range(requests):
        s = int(r.start[b])
        r.token[s + 1:s + 4] = np.array([5, 7, 11]) % V + b % 3     # three tokens, apart from one another
        r.p[s, r.token[s + 1:s + 4]] = 0.0
        if drawn:
            r.q[s, r.token[s + 1:s + 4]] = 0.1
    return r


@pytest.mark.parametrize("drawn", [True, False])
@pytest.mark.parametrize("value", [np.nan, -np.nan, np.inf])
@pytest.mark.parametrize("V", [40, 700, 33000])
def test_one_value_of_p_that_is_not_finite(kb, drawn, value, V):  # noqa: F811
    """At a token of the first, the second or the last child, at another one, at the ends: rejections or not, no token."""
    at = [lambda r, s: r.token[s + 1], lambda r, s: r.token[s + 2], lambda r, s: r.token[s + 3], lambda r, s: 20, lambda r, s: 0, lambda r, s: V - 1]
    r = _rejecting(V, V, drawn, 2 * len(at) + 1)
    for b in range(len(at)):
        s = int(r.start[b])
        x = at[b](r, s)
        r.p[s, x] = value
        if np.isposinf(value) and b < 3 and (drawn or b == 0):       # a child whose weight is infinite is kept if it is tested before any sum is
            r.u[s + 1:s + 4] = np.nan
        s = int(r.start[len(at) + b])                                # no child is tested
        r.token[s + 1:s + 4] = -1
        r.p[s, min(x, V - 1)] = value
    path, kept, nxt = r.run(kb)
    assert nxt[:-1] == [-1] * (2 * len(at)) and kept[:-1] == [0] * (2 * len(at))
    assert (path, kept, nxt) == r.want() and 0 <= nxt[-1] < V        # the last request has nothing of the kind


@pytest.mark.parametrize("V", [40, 700, 33000])
def test_one_nan_of_q(kb, V):  # noqa: F811
    """It counts from the first rejection on; a row of which no draft was rejected does not look at q."""
    r = _rejecting(V + 1, V, True, 9)
    for b in range(4):
        s = int(r.start[b])
        r.q[s, (int(r.token[s + 1]), int(r.token[s + 3]), 20, V - 1)[b]] = np.nan
        s = int(r.start[4 + b])
        r.token[s + 1:s + 4] = -1
        r.q[s, (0, 20, 30, V - 1)[b]] = np.nan
    path, kept, nxt = r.run(kb)
    assert nxt[:4] == [-1] * 4 and all(0 <= t < V for t in nxt[4:]) and kept == [0] * 9
    assert (path, kept, nxt) == r.want()


@pytest.mark.parametrize("drawn", [True, False])
def test_a_row_that_is_left_by_its_first_draft_is_not_looked_at(kb, drawn):  # noqa: F811
    r = Round(5, [[-1, 0, 0, 1, 1]] * 3, 900, drawn)
    for b in range(3):
        s = int(r.start[b])
        r.u[s:s + 5] = 0.0
        r.token[s + 1:s + 5] = [3, 4, 5, 6]
        r.p[s, 3], r.p[s + 1, 5:7] = 0.5, 0.0                        # row 1 is kept, rows 3 and 4 are not
        r.p[s, 800] = np.nan
        if drawn:
            r.q[s, 3], r.q[s, 900 - 1] = 0.5, np.nan
    r.p[int(r.start[1]) + 1, 17] = np.nan                            # the row that the token comes from
    if drawn:
        r.q[int(r.start[2]) + 1, 17] = np.nan
    path, kept, nxt = r.run(kb)
    assert kept == [1, 1, 1] and nxt[1] == -1 and 0 <= nxt[0] < 900 and (nxt[2] == -1) == drawn
    assert (path, kept, nxt) == r.want()


def test_no_draft_is_kept_behind_a_sum_that_is_nan(kb):  # noqa: F811
    """Chosen drafts: the NaN at the second child's token is no part of the sum that the third one would be held against."""
    r = Round(6, [[-1, 0, 0, 0]] * 2, 300, False)
    for b in range(2):
        s = int(r.start[b])
        r.token[s + 1:s + 4] = [3, 4, 5]
        r.p[s, 3:6] = [0.0, np.nan if b == 0 else 0.0, 0.5]
        r.u[s:s + 4] = 0.1
    path, kept, nxt = r.run(kb)
    assert kept == [0, 1] and nxt[0] == -1 and path[4:6] == [0, 3]
    assert (path, kept, nxt) == r.want()


@pytest.mark.parametrize("V", [2, 33, 5000])
@pytest.mark.parametrize("children", [12, 40, 400, 1000])
def test_many_rejections_at_one_row(kb, V, children):  # noqa: F811
    """All children are the token of which p has less than q.  After the first rejection only ids behind it have weight, in shares that every further one leaves as they are
    up to q: Z is small each time, and what is left of a row stays exact to some 2^-50 however often."""
    r = Round(8, [[-1] + [0] * children] * 4, V, True)
    for b, (top, more) in enumerate([(0.9, 0.05), (0.99, 0.005), (0.5, 0.25), (0.999, 1e-6)]):
        s = int(r.start[b])
        r.q[s], r.p[s] = 0.0, 0.0
        r.q[s, 0], r.q[s, 1] = top, 1 - top
        r.p[s, 0], r.p[s, 1] = top + more, 1 - top - more
        if V > 2:
            r.q[s, 0], r.q[s, 20] = top / 2, top / 2
            r.p[s, 0], r.p[s, 20] = top / 2 + more, top / 2
        r.token[s + 1:s + 1 + children], r.u[s:s + 1 + children] = 1, np.float32(1 - 2 ** -24)
        r.last[b] = np.float32(1 - 2 ** -24)
    path, kept, nxt = r.run(kb)
    assert kept == [0] * 4 and nxt == [0] * 4                        # token 0 is all that is ever left
    assert (path, kept, nxt) == r.want()


def test_siblings_of_drafts_that_are_next_to_p(kb):  # noqa: F811
    """q so near p that the first rejections leave next to nothing; many drafts, not only drawn ones.  The oracle's decisions throughout."""
    rng = np.random.default_rng(3)
    for seed in range(12):
        V = int(rng.choice([3, 8, 60, 1000]))
        r = Round(40 + seed, [[-1] + [0] * 30 + [5] * 10] * 20, V, True, sharp=2, zeros=0.1, mix=1.0)
        r.p = (r.q * (1 + 10.0 ** -rng.integers(1, 6) * rng.standard_normal(r.q.shape))).astype(np.float32)
        r.p /= r.p.sum(1, keepdims=True)
        r.token = np.where(rng.random(len(r.token)) < 0.7, rng.integers(0, V, len(r.token)), r.token)
        r.u = np.where(rng.random(len(r.u)) < 0.8, np.float32(1 - 2 ** -20), r.u).astype(np.float32)
        assert r.run(kb) == r.want()


@pytest.mark.parametrize("at", [1, 20, 31, 32, 40, 70])
def test_a_nan_among_many_chosen_drafts(kb, at):  # noqa: F811
    """Children in several groups of 32 rows; the one at `at` has the NaN, the last one all the weight there is."""
    n = 72
    r = Round(9, [[-1] + [0] * (n - 1)] * 2, 500, False)
    for b in range(2):
        s = int(r.start[b])
        r.token[s + 1:s + n] = np.arange(1, n)
        r.p[s, 1:n - 1], r.p[s, n - 1] = 0.0, 0.5
        r.u[s:s + n] = 0.9
        r.u[s + n - 1] = 0.25
    r.p[int(r.start[0]), at] = np.nan
    path, kept, nxt = r.run(kb)
    assert kept == [0, 1] and nxt[0] == -1 and path[n + 1] == n - 1
    assert (path, kept, nxt) == r.want()


@pytest.mark.parametrize("at", [[2, 3], [4, 37], [33, 1000], [1, 2, 3, 4, 1023]])
def test_tokens_that_come_again_among_many_rows(kb, at):  # noqa: F811
    """Chosen drafts: of siblings with one token the first one counts, the others have nothing left.  All rows are row 0's children, or of two parents in turn."""
    n = 1024
    for parents in ([-1] + [0] * (n - 1), [-1, 0] + [i % 2 for i in range(n - 2)]):
        r = Round(10, [parents], 3000, False)
        r.token[1:] = np.arange(1, n)
        r.token[at] = 2000
        r.p[:] = 1.0 / 3000
        r.u[:] = np.float32(1 - 2 ** -24)
        r.u[at[1:]] = 0.0                                            # kept whatever is left
        got = r.run(kb)
        assert got == r.want()


def test_rows_without_siblings_cost_little(kb):  # noqa: F811
    """Chosen drafts: a chain of 1024 rows has no siblings to compare, 16 times as many rows as one of 64 must not take 256 times as long."""
    took = []
    for n in (64, 1024):
        r = Round(12, [list(range(-1, n - 1))], 1000, False, mix=0.0)
        args, out = r.on_device(), [torch.zeros(k, dtype=torch.int32, device="cuda") for k in (n, 1, 1)]
        args[5].fill_(1.0)                                           # nothing is kept: what the rows cost, not the path
        kb.knnssd_tree_accept(*args, *out)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            for _ in range(20):
                kb.knnssd_tree_accept(*args, *out)
        e = [torch.cuda.Event(enable_timing=True) for _ in range(2)]
        times = []
        for _ in range(7):
            e[0].record()
            graph.replay()
            e[1].record()
            torch.cuda.synchronize()
            times.append(e[0].elapsed_time(e[1]))
        took.append(np.median(times))
        assert out[1].tolist() == [0]
    assert took[1] < 12 * took[0]
