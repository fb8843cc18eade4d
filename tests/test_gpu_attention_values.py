"""Attention of new rows where scores or values are not finite, or large, against the definition: a row's result follows from what it sees.

A score that is NaN or +inf makes its row NaN; one of -inf has the weight 0; what a row does not see has no part in it, whatever it holds.
Tolerances of finite results are those of test_gpu_paged_attention.py.
"""
import numpy as np
import pytest
import torch

from test_gpu_paged_attention import Paged, _attend64, _check, _packed

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def kb():
    if not torch.cuda.is_available():
        pytest.fail("the gpu tests need a CUDA device")
    from paper_2505_16162_b200 import build
    build.build()
    from paper_2505_16162_b200 import binding
    return binding


def _by_scores(q, k, v, seen, scale):
    """_attend64 where scores may be anything: (result, tolerance)."""
    n, H, hd = q.shape
    outs = []
    for h in range(H):
        kh, vh = (x[:, h * k.shape[1] // H][:, None] for x in (k, v))
        s = torch.where(seen, torch.stack([(q[i, h].double()[None] * kh[:, 0].double()).sum(1) for i in range(n)]) * scale, -torch.inf)
        o, t = _attend64(q[:, h:h + 1], kh, vh, seen & s.isfinite(), scale)
        o[(s.isnan() | (s == torch.inf)).any(1)] = torch.nan
        outs.append((o, t))
    return torch.cat([o for o, _ in outs], 1), torch.cat([t for _, t in outs], 1)


@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("lens,first,page", [(20, 0, 16), (20, 8, 64), (300, 128, 64), (300, 256, 16)])
def test_keys_that_are_not_finite_bf16(kb, value, lens, first, page):
    p = Paged(41, [lens] * 16, [6] * 16, 2, 64, page, "bf16")
    for b in range(16):                                              # one position of each request, all places modulo 16
        at = first + b
        p.k[int(p.table[b, at // page]), 1, at % page, 7] = value
        p.dense[b][0][at, 1, 7] = value
    q = p.q(4, 64, "bf16")
    got = p.run(kb, q)
    for b in range(16):
        r = slice(6 * b, 6 * b + 6)
        want, tol = _by_scores(q[r], *p.dense[b], p.seen(b), 64 ** -0.5)
        assert want.isnan().any() and not want.isnan().all()
        _check(got[r], want, tol, f"position {first + b}")


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_queries_that_are_nan_in_first_rows(kb, dtype):
    lens = [1, 2, 2, 3, 40, 9]
    q, k, v, start = _packed(43, lens, 4, 2, 64, dtype)
    for b, i in ((0, 0), (1, 0), (2, 1), (3, 1), (4, 0), (5, 8)):
        q[int(start[b]) + i, 1 + b % 3, 11] = torch.nan
    got = kb.knnssd_packed_attention(q, k, v, start)
    for b, n in enumerate(lens):
        r = slice(int(start[b]), int(start[b]) + n)
        _check(got[r], *_by_scores(q[r], k[r], v[r], torch.ones(n, n, dtype=torch.bool, device="cuda").tril(), 64 ** -0.5), f"prompt {b}")


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_rows_of_nan_alone_in_parts(kb, dtype):
    """A context that several workers share: the joined row is NaN whichever part has the score."""
    p = Paged(47, [40000], [2], 1, 128, 64, dtype)
    for at in (0, 1, 17, 20000, 39999):
        page, off = int(p.table[0, at // 64]), at % 64
        old = p.k[page, 0, off, 0].clone()
        p.k[page, 0, off, 0] = torch.nan
        q = p.q(2, 128, dtype)
        assert p.run(kb, q).isnan().all(), f"position {at}"
        p.k[page, 0, off, 0] = old
    q[0, 1, 5] = torch.nan
    got = p.run(kb, q)
    assert got[0, 1].isnan().all() and got[0, 0].isfinite().all() and got[1].isfinite().all()


@pytest.mark.parametrize("dtype,cache", [("fp32", "fp32"), ("fp32", "bf16"), ("bf16", "bf16")])
@pytest.mark.parametrize("page", [16, 64])
def test_large_values_that_are_not_seen(kb, dtype, cache, page):
    """The last new row's V is near the type's largest, all places modulo 16: the rows before it are as if it were not there."""
    p = Paged(53, [60 + b for b in range(16)], [4] * 16, 2, 64, page, cache)
    for b in range(16):
        at = p.lens[b] + 3
        p.v[int(p.table[b, at // page]), :, at % page] = 3e38
        p.dense[b][1][at] = 3e38
    q = p.q(4, 64, dtype)
    got = p.run(kb, q)
    for b in range(16):
        r = slice(4 * b, 4 * b + 3)
        seen = p.seen(b)[:3, :-1]
        _check(got[r], *_attend64(q[r], p.dense[b][0][:-1], p.dense[b][1][:-1], seen, 64 ** -0.5), f"request {b}")


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_scores_far_below_the_largest_weigh_nothing(kb, dtype):
    """Scores 400 powers of two below the row's largest, at all places modulo 8 but one: their large V have no part in the result."""
    lens = [9] * 8
    q, k, v, start = _packed(59, lens, 2, 2, 64, dtype)
    q[:], k[:] = 0.0, 0.0
    q[:, :, 0], k[:, :, 0] = 8.0, -277.0                             # scale 1/8: scores -277, or 0 at one position: 2^-399.6
    v[:] = 3e38
    for b in range(8):
        k[9 * b + b, :, 0] = 0.0
        v[9 * b + b] = 1.5
    got = kb.knnssd_packed_attention(q, k, v, start)
    for b in range(8):
        assert (got[9 * b + b:9 * b + 9] == 1.5).all(), f"position {b}"


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_values_that_are_not_finite_in_long_prompts(kb, dtype):
    """A NaN in one dimension of V every 64 rows: rows before it, in its block too, are finite in that dimension, over all that they see."""
    lens = [6000, 70, 2500]
    q, k, v, start = _packed(61, lens, 4, 2, 128, dtype)
    for b, n in enumerate(lens):
        for at in range(63, n, 64):
            v[int(start[b]) + at, 1, at // 64] = (torch.nan, torch.inf, -torch.inf)[at // 64 % 3]
    got = kb.knnssd_packed_attention(q, k, v, start)
    for b, n in enumerate(lens):
        r = slice(int(start[b]), int(start[b]) + n)
        _check(got[r], *_attend64(q[r], k[r], v[r], torch.ones(n, n, dtype=torch.bool, device="cuda").tril(), 128 ** -0.5), f"prompt {b}")


@pytest.mark.parametrize("page", [16, 128])
def test_values_that_are_not_finite_behind_long_contexts(kb, page):
    p = Paged(67, [30000, 900, 5000], [40, 3, 130], 2, 128, page, "bf16")
    for b in (0, 2):
        at = p.lens[b] + p.fresh[b] - 1
        p.v[int(p.table[b, at // page]), 0, at % page] = torch.nan
        p.dense[b][1][at, 0] = torch.nan
    q = p.q(6, 128, "bf16")
    _check(p.run(kb, q), *p.want(q))


# ---- waits that give up ---------------------------------------------------------------------------------------------
def _stopped(kb, call, tiles):
    kb.knnssd_debug_attention_timeout(200, tiles)
    try:
        got = call()
        with pytest.raises(kb.KnnssdError) as e:
            kb.knnssd_attention_status()
        assert e.value.status == 7
        kb.knnssd_attention_status()                                 # told once
    finally:
        kb.knnssd_debug_attention_timeout(0)
    return got.double()


@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("lens,fresh,KV", [([700], [3], 1), ([30000, 40], [2, 140], 2), ([200] * 90, [1] * 45 + [90] * 45, 4)])
def test_a_wait_that_gives_up_over_pages(kb, page, lens, fresh, KV):
    p = Paged(71, lens, fresh, KV, 64, page, "bf16")
    q = p.q(2 * KV, 64, "bf16")
    want, tol = p.want(q)
    kb.knnssd_attention_status()
    for tiles in (0, 1, 4):
        got = _stopped(kb, lambda: p.run(kb, q), tiles)
        lost = got.isnan().any(2)
        assert got[lost].isnan().all() and (tiles > 0 or lost.all()) and lost.any()
        _check(got[~lost], want[~lost], tol[~lost], f"rows that were not lost, {tiles} tiles")
        _check(p.run(kb, q), want, tol, "the call behind it")
        kb.knnssd_attention_status()


def test_a_wait_that_gives_up_in_packed_prompts(kb):
    lens = [700, 1, 33, 0, 260]
    q, k, v, start = _packed(73, lens, 4, 2, 128, "bf16")
    q2, k2, v2 = (torch.cat([x, x[:9]]) for x in (q, k, v))          # rows that no prompt has
    want = kb.knnssd_packed_attention(q, k, v, start).double()
    for tiles in (0, 2, 5):
        got = _stopped(kb, lambda: kb.knnssd_packed_attention(q2, k2, v2, start), tiles)
        assert got[-9:].abs().max() == 0
        lost = got[:-9].isnan().any(2)
        assert lost.any() and got[:-9][lost].isnan().all() and torch.equal(got[:-9][~lost], want[~lost])
    assert torch.equal(kb.knnssd_packed_attention(q, k, v, start).double(), want)


def test_refusals_of_the_hook_and_under_a_capture(kb):
    with pytest.raises(kb.KnnssdError) as e:
        kb.knnssd_debug_attention_timeout(1000001)
    assert e.value.status == 1
    x = torch.zeros(4, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        x += 1
        with pytest.raises(kb.KnnssdError) as e:
            kb.knnssd_attention_status()
        assert e.value.status == 6
        x += 1
    graph.replay()
    assert x.tolist() == [2.0] * 4                                   # the capture has not noticed


# ---- fp32 rows: infinities, and values near the type's largest ----------------------------------------------------------
@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("cache", ["fp32", "bf16"])
@pytest.mark.parametrize("lens,first", [(20, 0), (300, 128)])
def test_keys_that_are_not_finite_fp32(kb, value, cache, lens, first):
    p = Paged(79, [lens] * 16, [6] * 16, 2, 64, 16, cache)
    for b in range(16):
        at = first + b
        p.k[int(p.table[b, at // 16]), 1, at % 16, 7] = value
        p.dense[b][0][at, 1, 7] = value
    q = p.q(4, 64, "fp32")
    got = p.run(kb, q)
    for b in range(16):
        r = slice(6 * b, 6 * b + 6)
        want, tol = _by_scores(q[r], *p.dense[b], p.seen(b), 64 ** -0.5)
        assert want.isnan().any() and not want.isnan().all()
        _check(got[r], want, tol, f"position {first + b}")


@pytest.mark.parametrize("dtype,cache", [("fp32", "fp32"), ("fp32", "bf16"), ("bf16", "bf16")])
@pytest.mark.parametrize("lens,fresh", [([50, 40], [4, 1]), ([30000, 10], [2, 20])])
def test_an_infinite_value_that_is_seen_is_the_result(kb, dtype, cache, lens, fresh):
    p = Paged(83, lens, fresh, 1, 128, 16, cache)
    for b, at, d, val in ((0, 17, 3, torch.inf), (0, 18, 9, -torch.inf), (1, lens[1] + fresh[1] - 1, 100, torch.inf)):
        p.v[int(p.table[b, at // 16]), 0, at % 16, d] = val
        p.dense[b][1][at, 0, d] = val
    q = p.q(4, 128, dtype)
    want, tol = p.want(q)
    for b, at, d, val in ((0, 17, 3, torch.inf), (0, 18, 9, -torch.inf), (1, lens[1] + fresh[1] - 1, 100, torch.inf)):
        r = torch.arange(p.rows, device="cuda")
        sees = (r >= p.start[b]) & (r < p.start[b + 1]) & (lens[b] + r - p.start[b] >= at)
        want[sees, :, d] = val
    got = p.run(kb, q).double()
    inf = want.isinf()
    assert torch.equal(got[inf], want[inf])
    _check(got[~inf], want[~inf], tol[~inf])


@pytest.mark.parametrize("what", ["fp32 over pages", "packed"])
def test_the_largest_values_that_are_not_seen_fp32(kb, what):
    """V of the type's largest: rounded to bf16, as the first of three terms, it is infinite."""
    most = torch.finfo(torch.float32).max
    lens = [37] * 16
    if what == "packed":
        q, k, v, start = _packed(89, lens, 4, 2, 64, "fp32")
        for b in range(16):
            v[37 * b + 20 + b] = most
        got = kb.knnssd_packed_attention(q, k, v, start)
        for b in range(16):
            r = slice(37 * b, 37 * b + 20 + b)
            n = 20 + b
            _check(got[r], *_attend64(q[r], k[r], v[r], torch.ones(n, n, dtype=torch.bool, device="cuda").tril(), 64 ** -0.5), f"prompt {b}")
        return
    p = Paged(97, [60 + b for b in range(16)], [4] * 16, 2, 64, 16, "fp32")
    for b in range(16):
        at = p.lens[b] + 3
        p.v[int(p.table[b, at // 16]), :, at % 16] = -most
    q = p.q(4, 64, "fp32")
    got = p.run(kb, q)
    for b in range(16):
        r = slice(4 * b, 4 * b + 3)
        _check(got[r], *_attend64(q[r], p.dense[b][0][:-1], p.dense[b][1][:-1], p.seen(b)[:3, :-1], 64 ** -0.5), f"request {b}")


# ---- rows that no request has -----------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("start", [[5, 70, 100], [130, 130, 130], [0, 0, 0], [7, 7, 40]])
def test_rows_before_the_first_request(kb, dtype, start):
    q, k, v, _ = _packed(101, [130], 4, 2, 64, dtype)
    out = torch.full((130, 4, 64), torch.nan, device="cuda", dtype=q.dtype)
    kb.knnssd_packed_attention(q, k, v, torch.tensor(start, dtype=torch.int32, device="cuda"), out=out)
    for a, b in zip(start, start[1:]):
        if b > a:
            _check(out[a:b], *_attend64(q[a:b], k[a:b], v[a:b], torch.ones(b - a, b - a, dtype=torch.bool, device="cuda").tril(), 64 ** -0.5))
    assert not out[:start[0]].any() and not out[start[-1]:].any()
