"""Which drafts of a tree are kept, and their K and V moved together: equal to the oracle's, whole numbers.

A test or a draw lies so near a border that 64-bit sums in another order decide otherwise with a probability of some 2^-50 times the vocabulary: never here.
"""
import numpy as np
import pytest
import torch

from oracle import trees as ot

pytestmark = pytest.mark.gpu
I32 = dict(dtype=torch.int32, device="cuda")


@pytest.fixture(scope="module")
def kb():
    if not torch.cuda.is_available():
        pytest.fail("the gpu tests need a CUDA device")
    from paper_2505_16162_b200 import build
    build.build()
    from paper_2505_16162_b200 import binding
    return binding


def _parents(rng, n, back):
    return [max(0, i - int(rng.integers(1, back + 1))) if i else -1 for i in range(n)]


def _rows(rng, n, V, sharp, zeros):
    """n distributions in fp32, a share `zeros` of their values 0."""
    w = rng.random((n, V)) ** sharp
    w[rng.random((n, V)) < zeros] = 0.0
    w[np.arange(n), rng.integers(0, V, n)] += 0.3
    return (w / w.sum(1, keepdims=True)).astype(np.float32)


class Round:
    """Trees of several requests with the distributions behind their rows; `before` and `behind` rows of nobody."""

    def __init__(self, seed, parents, V, drawn, sharp=6, zeros=0.3, mix=0.5, before=0, behind=0):
        rng = np.random.default_rng(seed)
        self.rng, self.parents, self.V, self.before, self.behind = rng, parents, V, before, behind
        self.start = np.cumsum([before] + [len(p) for p in parents])
        R = int(self.start[-1]) + behind
        self.q = _rows(rng, R, V, sharp, zeros)
        self.p = mix * self.q + (1 - mix) * _rows(rng, R, V, sharp, zeros)      # fp32
        self.p /= self.p.sum(1, keepdims=True)
        if not drawn:
            rank = np.argsort(-self.q, axis=1)[:, :64]
        self.token = rng.integers(0, V, R)
        for s, par in zip(self.start, parents):
            for i in range(1, len(par)):
                up = s + par[i]
                if par[i] < 0:
                    continue
                if drawn:
                    self.token[s + i] = min(V - 1, int(np.searchsorted(np.cumsum(self.q[up].astype(np.float64)), rng.random() * self.q[up].astype(np.float64).sum(), side="right")))
                else:
                    self.token[s + i] = rank[up, par[:i].count(par[i]) % rank.shape[1]]
        self.u, self.last = rng.random(R).astype(np.float32), np.minimum(rng.random(len(parents)).astype(np.float32), np.float32(1 - 2 ** -24))
        if not drawn:
            self.q = None

    def want(self):
        path, kept, nxt = np.full(len(self.token), -1), [], []
        for b, par in enumerate(self.parents):
            rows = slice(self.start[b], self.start[b] + len(par))
            if not par:
                kept.append(0)
                nxt.append(-1)
                continue
            k, t = ot.accept(self.p[rows], None if self.q is None else self.q[rows], self.token[rows].tolist(), par, self.u[rows], self.last[b])
            path[self.start[b]:self.start[b] + len(k)] = k
            kept.append(len(k) - 1)
            nxt.append(t)
        return path.tolist(), kept, nxt

    def on_device(self):
        parent = np.full(len(self.token), 2)
        parent[self.before:len(parent) - self.behind] = [x for p in self.parents for x in p]
        f = lambda x: None if x is None else torch.as_tensor(np.ascontiguousarray(x), dtype=torch.float32, device="cuda")  # noqa: E731
        i = lambda x: torch.as_tensor(np.ascontiguousarray(x), **I32)  # noqa: E731
        return [f(self.p), f(self.q), i(self.token), i(parent), i(self.start), f(self.u), f(self.last)]

    def run(self, kb):
        out = [torch.full((n,), 77, **I32) for n in (len(self.token), len(self.parents), len(self.parents))]
        kb.knnssd_tree_accept(*self.on_device(), *out)
        return tuple(t.tolist() for t in out)


@pytest.mark.parametrize("drawn", [True, False])
@pytest.mark.parametrize("V", [1, 2, 31, 32, 33, 257, 1000, 4099])
def test_small_vocabularies(kb, drawn, V):
    for seed in range(6):
        rng = np.random.default_rng(seed)
        parents = [_parents(rng, int(n), int(back)) for n, back in zip(rng.integers(0, 20, 40), rng.integers(1, 8, 40))]
        r = Round(100 * V + seed, parents, V, drawn, before=seed % 3, behind=seed % 2)
        assert r.run(kb) == r.want()


@pytest.mark.parametrize("drawn", [True, False])
@pytest.mark.parametrize("V,requests,rows,back", [(32000, 1, 6, 1), (32000, 7, 25, 5), (152064, 3, 12, 6), (65537, 2, 64, 64), (3001, 70, 9, 3), (500003, 1, 4, 2)])
def test_vocabularies_of_models(kb, drawn, V, requests, rows, back):
    for seed in range(3):
        rng = np.random.default_rng(seed)
        r = Round(7 * V + seed, [_parents(rng, max(1, rows - (b % 3)), back) for b in range(requests)], V, drawn, sharp=40, zeros=0.8 if seed else 0.0)
        assert r.run(kb) == r.want()


@pytest.mark.parametrize("drawn", [True, False])
def test_many_children_and_many_rows(kb, drawn):
    rng = np.random.default_rng(1)
    parents = [[-1] + [0] * 200, [-1] + [0] * 63, _parents(rng, 300, 90), [-1, 0] + [1] * 100 + [101] * 30, list(range(-1, 400))]
    for mix in (0.02, 0.9):
        r = Round(5 + int(10 * mix), parents, 5000, drawn, sharp=3, zeros=0.0, mix=mix)
        assert r.run(kb) == r.want()


def test_only_the_first_1024_rows_are_looked_at(kb):
    r = Round(2, [[-1] + [0] * 1040, [-1, 0]], 64, False, mix=0.0)
    r.p[0] = 0.0
    r.p[0, :40] = 1 / 40
    r.token[1:1024] = 50                                             # no weight there
    r.token[1024:1041] = 7                                           # these would be kept
    r.u[:] = 0.0
    path, kept, nxt = r.run(kb)
    assert kept[0] == 0 and path[:1041] == [0] + [-1] * 1040 and nxt[0] == int(r.last[0] * 40)


@pytest.mark.parametrize("drawn", [True, False])
def test_borders(kb, drawn):
    """Uniforms of 0 and next to 1, distributions that are equal, that are one point, that leave nothing; drafts that no sibling differs from."""
    V = 300
    parents = [[-1, 0, 0, 1, 1, 2, 2]] * 12
    r = Round(11, parents, V, drawn)
    top = np.float32(1 - 2 ** -24)
    for b in range(12):
        s = int(r.start[b])
        rows = slice(s, s + 7)
        if b in (0, 1):
            r.u[rows], r.last[b] = (0.0, 0.0) if b else (top, top)
        if b in (2, 3) and drawn:                                    # p is q: every draft is kept, the uniforms being below 1
            r.p[rows] = r.q[rows]
            r.u[rows] = top
        if b in (4, 5):                                              # all of p on one token, that the first child is or is not
            r.p[rows] = 0.0
            r.p[s, r.token[s + 1] if b == 4 else (r.token[s + 1] + 1) % V] = 1.0
            r.p[s + 1:s + 7, 17] = 1.0
        if b == 6:                                                   # children that are the same token
            r.token[rows] = r.token[s + 1]
            r.u[rows] = top
        if b == 7 and drawn:                                         # p below q everywhere: a rejection leaves nothing
            r.p[rows] = r.q[rows] * np.float32(0.5)
            r.u[rows] = top
        if b == 8:
            r.last[b] = top
            r.p[rows, V - 3:] = 0.0                                  # the crossing lies before ids without weight
        if b == 9:
            r.last[b], r.u[rows] = 0.0, top
            r.p[rows, :5] = 0.0
        if b == 10:
            r.p[rows] = 0.0                                          # no weight at all
        if b == 11 and not drawn:                                    # the children hold all of p
            r.p[s] = 0.0
            r.p[s, r.token[s + 1]] = r.p[s, r.token[s + 2]] = 0.5
            r.u[rows] = top
    got, want = r.run(kb), r.want()
    assert got == want
    assert got[2][10] == -1


def test_rows_that_are_passed_over(kb):
    for drawn in (True, False):
        r = Round(3, [[-1, 0, 0, 1, 2, 0], [-1, 5, 0, 3, 0], [-1, 0, -1, 2, -7], [3, 0, 0], []], 50, drawn, mix=0.9, before=1, behind=2)
        r.u[:] = 0.0
        r.token[1 + 1] = -1                                          # row 1 of the first request, and what follows it
        r.token[1 + 6 + 2] = 50
        assert r.run(kb) == r.want()


def test_values_that_are_no_distribution_end_all_the_same(kb):
    """NaN and infinities in p or q, uniforms outside [0, 1): whatever comes, within the rows and ids, -1 for the token."""
    for drawn in (True, False):
        r = Round(9, [[-1, 0, 0, 1, 1]] * 6, 700, drawn)
        s = r.start
        r.p[s[0]:s[1]] = np.nan
        r.p[s[1]:s[2], 5] = np.inf
        if drawn:
            r.q[s[2]:s[3]] = np.nan
        r.u[s[3]:s[4]], r.last[3] = np.nan, np.nan
        r.last[4] = 1.0
        r.p[s[5], 3] = -np.inf
        path, kept, nxt = r.run(kb)
        assert nxt[0] == -1 and nxt[3] == -1 and nxt[4] == -1
        assert all(-1 <= t < 700 for t in nxt) and all(0 <= k < 5 for k in kept) and all(-1 <= x < 5 for x in path)


def test_a_chain_is_a_round_of_speculative_sampling(kb):
    rng = np.random.default_rng(8)
    for seed in range(20):
        k, V = int(rng.integers(0, 9)), int(rng.choice([50, 1000, 32000]))
        r = Round(seed, [list(range(-1, k))], V, True, mix=0.8)
        p, q, token, _, _, u, last = r.on_device()
        path, kept, nxt = r.run(kb)
        assert kb.knnssd_spec_accept(p, q[:k].contiguous(), token[1:].tolist(), u[1:].tolist(), float(last[0])) == (kept[0], nxt[0])
        assert path == list(range(kept[0] + 1)) + [-1] * (k - kept[0])


def test_greedy_paths(kb):
    rng = np.random.default_rng(4)
    parents = [_parents(rng, int(n), int(back)) for n, back in zip(rng.integers(0, 130, 300), rng.integers(1, 9, 300))] + [list(range(-1, 500)), [-1] + [0] * 90, [-1, 7, -1, 2]]
    before, behind = 3, 5
    start = np.cumsum([before] + [len(p) for p in parents])
    R = int(start[-1]) + behind
    best, token, parent = rng.integers(0, 4, R), rng.integers(0, 4, R), np.full(R, 1)
    parent[before:R - behind] = [x for p in parents for x in p]
    token[start[300] + 1:start[301]] = best[start[300]:start[301] - 1]           # the long chain agrees to its end
    path, kept, nxt = np.full(R, -1), [], []
    for s, p in zip(start, parents):
        k, t = ot.agree(best[s:].tolist(), token[s:s + len(p)].tolist(), p) if p else ([], -1)
        path[s:s + len(k)] = k
        kept.append(max(0, len(k) - 1))
        nxt.append(int(t))
    out = [torch.full((n,), 77, **I32) for n in (R, len(parents), len(parents))]
    kb.knnssd_tree_agree(*(torch.as_tensor(x, **I32) for x in (best, token, parent, start)), *out)
    assert [t.tolist() for t in out] == [path.tolist(), kept, nxt]
    assert max(kept) == 500


# ---- the kept rows' K and V ----------------------------------------------------------------------------------------------
def _pools(seed, n, lens, fresh, KV, hd, page, dtype, spare=3):
    g = torch.Generator(device="cuda").manual_seed(seed)
    held = [-(-(a + r) // page) for a, r in zip(lens, fresh)]
    n_pages = sum(held) + spare
    ids = np.random.default_rng(seed).permutation(n_pages)
    table, at = np.full((len(lens), max(held) + 1), -1, np.int32), 0
    for b, h in enumerate(held):
        table[b, :h] = ids[at:at + h]
        at += h
    pools = [torch.randn(n_pages, KV, page, hd, generator=g, device="cuda").to(dtype) for _ in range(n)]
    return pools, torch.as_tensor(table, device="cuda")


def _moved(pools, table, lens, start, path, page):
    """On copies, row by row in order; a position without a page is left out."""
    pools, table = [p.clone() for p in pools], table.tolist()
    n_pages = pools[0].shape[0]
    for b, m in enumerate(lens):
        before = -1
        for j, r in enumerate(path[start[b]:start[b + 1]]):
            if r <= before or r >= start[b + 1] - start[b]:
                break
            before = r
            places = [(table[b][x // page], x % page) if x // page < len(table[b]) else (-1, 0) for x in (m + r, m + j)]
            if any(not 0 <= i < n_pages for i, _ in places):
                continue
            (sp, so), (dp, do) = places
            for p in pools:
                p[dp, :, do] = p[sp, :, so]
    return pools


def _keep(kb, pools, table, lens, start, path):
    k, v = pools[:len(pools) // 2], pools[len(pools) // 2:]
    kb.knnssd_keep_rows(kb.PagePools(k, v), table, torch.tensor(lens, **I32), torch.tensor(start, **I32), torch.tensor(path, **I32))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("KV,hd,page,layers", [(2, 64, 16, 3), (5, 128, 32, 1), (8, 128, 128, 2), (1, 64, 64, 4), (3, 128, 16, 150)])
def test_kept_rows_move_together(kb, dtype, KV, hd, page, layers):
    rng = np.random.default_rng(KV + page)
    lens, fresh = [0, 15, 100, 3, 31, 64], [9, 40, 64, 0, 1, 150]
    start = np.cumsum([2] + fresh).tolist()
    path = [0, 1] + [-1] * (sum(fresh) + 3)
    for b, n in enumerate(fresh):
        if n:
            kept = [0] + sorted(rng.choice(np.arange(1, n), int(rng.integers(0, n)), replace=False).tolist()) if n > 1 else [0]
            path[start[b]:start[b] + len(kept)] = kept
    pools, table = _pools(KV, 2 * layers, lens, fresh, KV, hd, page, dtype)
    want = _moved(pools, table, lens, start, path, page)
    _keep(kb, pools, table, lens, start, path)
    assert all(torch.equal(a, b) for a, b in zip(pools, want))


def test_long_paths_that_overlap(kb):
    """Every row but one moves one place down: what a row leaves, the next one takes."""
    lens, fresh = [5, 50], [300, 129]
    start = [0, 300, 429]
    path = [0] + list(range(2, 300)) + [-1] + list(range(1, 129)) + [-1]
    pools, table = _pools(1, 4, lens, fresh, 2, 64, 16, torch.bfloat16)
    want = _moved(pools, table, lens, start, path, 16)
    _keep(kb, pools, table, lens, start, path)
    assert all(torch.equal(a, b) for a, b in zip(pools, want))


def test_paths_that_end_and_pages_that_are_gone(kb):
    lens, fresh = [40, 10, 7, 20, 0], [10, 10, 10, 70, 12]
    start = np.cumsum([0] + fresh).tolist()
    path = [0, 3, 3, 5] + [-1] * 6 + [0, 4, 2, 9] + [-1] * 6 + [0, 10, 11] + [-1] * 7 + [0] + list(range(2, 50)) + [49, 60] + [-1] * 19 + [-1, 4, 5] + [-1] * 9
    pools, table = _pools(2, 2, lens, fresh, 2, 64, 16, torch.float32)
    table[3, 2], table[3, 4] = -1, pools[0].shape[0] + 5
    want = _moved(pools, table, lens, start, path, 16)
    _keep(kb, pools, table, lens, start, path)
    assert all(torch.equal(a, b) for a, b in zip(pools, want))
    before = [p.clone() for p in pools]
    _keep(kb, pools, table, [-3, 2 ** 31 - 40, 2 ** 30, -2 ** 31, 1000], start, path)            # lengths out of range: nothing there to move
    assert all(torch.equal(a, b) for a, b in zip(pools, before))


def test_pools_beyond_32_bits(kb):
    n_pages = 2 ** 31 // (8 * 64 * 128) + 9
    pools = [torch.zeros(n_pages, 8, 64, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    for p in pools:
        p[-1] = torch.randn(8, 64, 128, device="cuda").bfloat16()
    table = torch.tensor([[n_pages - 1]], **I32)
    want = _moved([p[-1:] for p in pools], torch.tensor([[0]]), [4], [0, 6], [0, 2, 5, -1, -1, -1], 64)
    _keep(kb, pools, table, [4], [0, 6], [0, 2, 5, -1, -1, -1])
    assert all(torch.equal(a[-1:], b) for a, b in zip(pools, want)) and not any(p[:-1].any() for p in pools)


def test_refusals_of_the_binding(kb):
    pools, table = _pools(3, 2, [10], [4], 2, 64, 16, torch.bfloat16)
    for k, v in (([], []), ([pools[0]], []), ([pools[0]], [pools[1].float()]), ([pools[0]], [pools[1][:1]]), ([pools[0].cpu()], [pools[1].cpu()]), ([pools[0].half()], [pools[1].half()]), ([pools[0]], [pools[0]])):
        with pytest.raises(ValueError):
            kb.PagePools(k, v)
    ok = kb.PagePools([pools[0]], [pools[1]])
    lens, start, path = torch.tensor([10], **I32), torch.tensor([0, 4], **I32), torch.tensor([0, 2, -1, -1], **I32)
    for bad in ((table.long(), lens, start, path), (table[0], lens, start, path), (table, lens.cpu(), start, path), (table, lens, start[:1], path), (table, lens, start, path.long())):
        with pytest.raises(ValueError):
            kb.knnssd_keep_rows(ok, *bad)
    r = Round(1, [[-1, 0]], 40, True)
    args = r.on_device()
    out = [torch.zeros(n, **I32) for n in (2, 1, 1)]
    for i, bad in ((0, args[0].double()), (0, args[0][:1]), (1, args[1][:, :20]), (2, args[2].long()), (4, args[4][:1]), (5, args[5].double()), (6, args[6].cpu())):
        with pytest.raises(ValueError):
            kb.knnssd_tree_accept(*[bad if i == j else a for j, a in enumerate(args)], *out)
    with pytest.raises(ValueError):
        kb.knnssd_tree_accept(*args, out[0][:1], *out[1:])
    with pytest.raises(ValueError):
        kb.knnssd_tree_agree(args[2], args[2][:1], args[3], args[4], *out)
    with pytest.raises(kb.KnnssdError) as e:
        thin = [p[..., :32].contiguous() for p in pools]
        kb.knnssd_keep_rows(kb.PagePools(thin[:1], thin[1:]), table, lens, start, path)
    assert e.value.status == 2


@pytest.mark.parametrize("drawn", [True, False])
@pytest.mark.parametrize("V", [999, 1002, 8193])
def test_rows_that_begin_anywhere(kb, drawn, V):
    """p and q whose rows, and whose own beginnings, are not on 16-byte boundaries."""
    rng = np.random.default_rng(V)
    for shift in (0, 1, 3):
        r = Round(V + shift, [_parents(rng, 9, 3) for _ in range(5)], V, drawn)
        p, q, *rest = r.on_device()
        moved = []
        for x in (p, q):
            if x is not None:
                wide = torch.full((x.numel() + 8,), torch.nan, device="cuda")
                wide[shift:shift + x.numel()] = x.flatten()
                x = wide[shift:shift + x.numel()].view(x.shape)
            moved.append(x)
        out = [torch.full((n,), 77, **I32) for n in (len(r.token), 5, 5)]
        kb.knnssd_tree_accept(*moved, *rest, *out)
        assert tuple(t.tolist() for t in out) == r.want()
