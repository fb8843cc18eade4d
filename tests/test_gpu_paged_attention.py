"""Attention of new rows over pages and over packed prompts, against a plain evaluation in 64 bits.

Tolerances, per element, from the arithmetic.  With A = sum_j p_j |v_j| (p: the exact softmax weights) and a score error e (relative error of
a weight: 2 e, numerator and sum), the result is off by at most A (2 e + r): r the roundings behind the weights.
  e      a product of 24-bit operands is exact to 2^-22 relative, hd of them are added in fp32: (hd + 16) 2^-24 sum_i |q_i k_i| scale at most, and
         the exponent is formed from it by one more product (2^-23 |s|); exp2 itself 2^-22
  fp32   r = 2^-20: fp32 sums of the weights and of p v in pieces of 16
  bf16   r = 2^-7 (1 + 2^-8): the weights are rounded to bf16 (eight bits: 2^-8), and so is the result (2^-8 of |o| <= A)
"""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def kb():
    if not torch.cuda.is_available():
        pytest.fail("the gpu tests need a CUDA device")
    from paper_2505_16162_b200 import build
    build.build()
    from paper_2505_16162_b200 import binding
    return binding


def _attend64(q, k, v, seen, scale):
    """q [n][H][hd], k, v [m][KV][hd] -> (result, tolerance); seen [n][m]: what a row looks at.  Values that a row does not see play no part."""
    n, H, hd = q.shape
    KV = k.shape[1]
    out, tol = (torch.zeros(n, H, hd, dtype=torch.float64, device=q.device) for _ in range(2))
    r = 2.0 ** -7 * (1 + 2.0 ** -8) if q.dtype == torch.bfloat16 else 2.0 ** -20
    for h in range(H):
        qh, kh, vh = q[:, h].double(), k[:, h * KV // H].double(), v[:, h * KV // H].double()
        s = torch.where(seen, qh @ torch.nan_to_num(kh).T * scale, -torch.inf)
        size = torch.where(seen, qh.abs() @ torch.nan_to_num(kh).abs().T * scale, 0.0)
        e = ((hd + 16) * 2.0 ** -24 * size.amax(1) + 2.0 ** -23 * torch.where(seen, s.abs(), 0.0).amax(1) + 2.0 ** -22)[:, None] if seen.shape[1] else 0.0
        some = seen.any(1, keepdim=True)
        p = torch.where(some, torch.softmax(torch.where(some, s, 0.0), 1), 0.0)
        odd = ~torch.isfinite(vh)
        out[:, h] = p @ torch.where(odd, 0.0, vh)
        tol[:, h] = (p @ torch.where(odd, 0.0, vh).abs()) * (2 * e + r) + 1e-30
        if odd.any():                                                # a row that sees one: whatever IEEE makes of it
            hit = (seen[:, :, None] & odd[None]).any(1)
            out[:, h] = torch.where(hit, torch.nan, out[:, h])
    return out, tol


def _check(got, want, tol, what=""):
    got = got.double()
    nan = want.isnan()
    assert not got[nan].isfinite().any(), f"{what}: a value that is not finite was lost"
    assert got[~nan].isfinite().all(), f"{what}: values that are not finite where none are seen"
    off = ((got - want).abs() / tol)[~nan]
    assert off.numel() == 0 or off.max() <= 1.0, f"{what}: {float(off.max()):.2f} times the tolerance"


class Paged:
    """Requests' pages scattered over a pool whose unused places are NaN."""

    def __init__(self, seed, lens, fresh, KV, hd, page, cache, spare=3, wide=2, spread=1.0):
        self.g = torch.Generator(device="cuda").manual_seed(seed)
        self.lens, self.fresh, self.page = list(lens), list(fresh), page
        held = [-(-(a + n) // page) for a, n in zip(lens, fresh)]
        n_pages = sum(held) + spare
        ids = np.random.default_rng(seed).permutation(n_pages)
        table = np.full((len(lens), max(held) + wide), -1, np.int32)
        self.k = torch.full((n_pages, KV, page, hd), torch.nan, dtype=TYPES[cache], device="cuda")
        self.v = self.k.clone()
        self.dense, at = [], 0
        for b, n in enumerate(held):
            table[b, :n] = ids[at:at + n]
            at += n
            m = lens[b] + fresh[b]
            kv = [(spread * torch.randn(m, KV, hd, generator=self.g, device="cuda")).to(TYPES[cache]) for _ in range(2)]
            self.dense.append(kv)
            for pool, x in zip((self.k, self.v), kv):
                pos = torch.arange(m, device="cuda")
                pool[torch.as_tensor(table[b], device="cuda").long()[pos // page], :, pos % page] = x
        self.table = torch.as_tensor(table, device="cuda")
        self.dlens = torch.tensor(self.lens, dtype=torch.int32, device="cuda")
        self.start = torch.tensor(np.concatenate([[0], np.cumsum(fresh)]), dtype=torch.int32, device="cuda")
        self.rows = int(sum(fresh))

    def seen(self, b):
        m, n = self.lens[b] + self.fresh[b], self.fresh[b]
        return torch.arange(m, device="cuda")[None] <= self.lens[b] + torch.arange(n, device="cuda")[:, None]

    def want(self, q, scale=None, hide=None):
        outs = []
        for b in range(len(self.lens)):
            s = self.seen(b)
            if hide is not None:
                s = s & ~hide(b)[None]
            r0 = int(self.start[b])
            outs.append(_attend64(q[r0:r0 + self.fresh[b]], *self.dense[b], s, q.shape[2] ** -0.5 if scale is None else scale))
        return torch.cat([o for o, _ in outs]), torch.cat([t for _, t in outs])

    def q(self, H, hd, dtype, spread=1.5):
        return (spread * torch.randn(self.rows, H, hd, generator=self.g, device="cuda")).to(TYPES[dtype])

    def run(self, kb, q, **kw):
        return kb.knnssd_paged_attention(q, self.k, self.v, self.table, self.dlens, self.start, **kw)


HEADS = [(4, 4, 64), (8, 2, 64), (5, 5, 128), (10, 2, 128), (6, 1, 128), (40, 8, 128), (24, 1, 64), (70, 2, 64)]
KINDS = [("fp32", "fp32"), ("fp32", "bf16"), ("bf16", "bf16")]
LENGTHS = [
    ([0], [1]), ([95], [1]), ([0], [17]), ([15], [1]), ([16], [16]), ([1280], [5]),
    ([0, 31, 700, 3, 64, 127], [1, 5, 1, 0, 16, 2]),
    ([5, 0, 0, 2000, 1], [0, 0, 130, 9, 33]),
]


@pytest.mark.parametrize("dtype,cache", KINDS)
@pytest.mark.parametrize("H,KV,hd", HEADS)
@pytest.mark.parametrize("at", range(len(LENGTHS)))
def test_new_rows_over_pages(kb, dtype, cache, H, KV, hd, at):
    lens, fresh = LENGTHS[at]
    page = (16, 32, 64, 128)[(at + H) % 4]
    p = Paged(7 * at + H, lens, fresh, KV, hd, page, cache)
    q = p.q(H, hd, dtype)
    want, tol = p.want(q)
    for hint in (0, max(fresh)):
        _check(p.run(kb, q, max_fresh=hint), want, tol, f"max_fresh {hint}")


@pytest.mark.parametrize("dtype,cache", KINDS)
@pytest.mark.parametrize("H,KV,hd,lens,fresh", [(8, 2, 128, [20011], [1]), (4, 4, 64, [9000, 40, 33000], [3, 1, 2]), (10, 2, 128, [5000, 0], [260, 300])])
def test_long_contexts_in_many_parts(kb, dtype, cache, H, KV, hd, lens, fresh):
    p = Paged(3, lens, fresh, KV, hd, 64, cache)
    q = p.q(H, hd, dtype)
    _check(p.run(kb, q), *p.want(q))


@pytest.mark.parametrize("dtype,cache", KINDS)
def test_many_requests_of_all_lengths(kb, dtype, cache):
    rng = np.random.default_rng(5)
    lens, fresh = rng.integers(0, 90, 700).tolist(), rng.integers(0, 4, 700).tolist()
    p = Paged(5, lens, fresh, 2, 64, 16, cache)
    q = p.q(6, 64, dtype)
    _check(p.run(kb, q, max_fresh=3), *p.want(q))


@pytest.mark.parametrize("dtype,cache", KINDS)
@pytest.mark.parametrize("scale", [0.0, 0.31, 5.0])
def test_scale_and_flat_and_steep_weights(kb, dtype, cache, scale):
    p = Paged(9, [300, 77], [5, 40], 2, 128, 16, cache)
    q = p.q(4, 128, dtype)
    _check(p.run(kb, q, scale=scale), *p.want(q, scale=scale))


@pytest.mark.parametrize("dtype,cache", KINDS)
@pytest.mark.parametrize("fresh", [[1, 5, 2], [150, 5, 200]])
def test_pages_that_are_gone_leave_rows_that_see_nothing(kb, dtype, cache, fresh):
    p = Paged(11, [40, 100, 0], fresh, 2, 64, 16, cache)
    gone = {0: range(0, 99), 1: (0, 3), 2: (0,)}                     # all of the first request's, two in the middle, the first of the last's
    for b, cols in gone.items():
        for c in cols:
            if c < p.table.shape[1]:
                p.table[b, c] = -1 if (b + c) % 2 else p.k.shape[0] + 7
    hide = lambda b: torch.isin(torch.arange(p.lens[b] + p.fresh[b], device="cuda") // 16, torch.tensor(list(gone[b]), device="cuda"))  # noqa: E731
    q = p.q(4, 64, dtype)
    want, tol = p.want(q, hide=hide)
    got = p.run(kb, q)
    assert got[:fresh[0]].abs().max() == 0 and not want[:fresh[0]].any()
    _check(got, want, tol)


@pytest.mark.parametrize("dtype,cache", KINDS)
@pytest.mark.parametrize("lens,fresh", [([33], [7]), ([130], [300]), ([4, 250], [16, 129])])
def test_what_is_not_finite_reaches_only_rows_that_see_it(kb, dtype, cache, lens, fresh):
    p = Paged(13, lens, fresh, 2, 128, 16, cache)
    for b, (a, n) in enumerate(zip(lens, fresh)):
        for i, val in ((n // 2, torch.inf), (n - 2, torch.nan)):     # V of one position among the new ones, of another in two dimensions
            page, off = int(p.table[b, (a + i) // 16]), (a + i) % 16
            p.v[page, 1, off, 5:7] = val
            p.dense[b][1][a + i, 1, 5:7] = val
    q = p.q(6, 128, dtype)
    want, tol = p.want(q)
    assert want.isnan().any() and not want.isnan().all()
    _check(p.run(kb, q), want, tol)


def test_scores_that_are_not_finite_stay_in_their_rows(kb):
    p = Paged(17, [50], [4], 2, 64, 16, "bf16")
    q = p.q(2, 64, "bf16")
    q[2, 1, 3] = torch.nan
    got = p.run(kb, q)
    want, tol = p.want(torch.nan_to_num(q))
    want[2, 1] = torch.nan
    _check(got, want, tol)
    low = Paged(18, [50], [4], 2, 64, 16, "bf16")                    # scores at the lowest end: all far below zero, weights still sum to one
    low.k.fill_(-300.0)
    low.dense[0][0].fill_(-300.0)
    q = torch.full((4, 2, 64), 300.0, dtype=torch.bfloat16, device="cuda")
    _check(low.run(kb, q), *low.want(q))


def test_rows_behind_the_last_request_and_strides(kb):
    p = Paged(19, [64, 5], [3, 2], 2, 64, 32, "bf16")
    wide = torch.randn(9, 6 * 64 + 72, device="cuda").bfloat16()
    q = wide[:, 8:8 + 6 * 64].unflatten(1, (6, 64))                  # rows some distance apart
    got = p.run(kb, q)
    assert got[5:].abs().max() == 0
    _check(got[:5], *p.want(q[:5]))
    out = torch.empty_like(got)
    assert p.run(kb, q, out=out) is out and torch.equal(out, got)


def test_lengths_out_of_range_stay_inside_the_pool(kb):
    p = Paged(23, [40, 10, 30], [2, 2, 2], 2, 64, 16, "bf16")
    q = p.q(4, 64, "bf16")
    want, tol = p.want(q)
    p.k.nan_to_num_()                                                # the places behind a request's length in its own pages are seen then
    p.v.nan_to_num_()
    p.dlens[0] = 2 ** 30                                             # positions that the table has no pages for are not seen
    p.dlens[1] = -5
    got = p.run(kb, q)
    _check(got[4:], want[4:], tol[4:])
    assert got.isfinite().all()
    p.start[3] = 1000                                                # more rows than there are
    assert p.run(kb, q).isfinite().all()


def test_pool_beyond_32_bits(kb):
    KV, hd, page = 8, 128, 64
    n_pages = 2 ** 31 // (KV * hd * page) + 40                       # elements, not bytes, pass 2^31
    k = torch.empty((n_pages, KV, page, hd), dtype=torch.bfloat16, device="cuda")
    v = torch.empty_like(k)
    small = Paged(29, [1000], [3], KV, hd, page, "bf16", spare=0)
    n = small.k.shape[0]
    k[-n:], v[-n:] = small.k, small.v
    small.k, small.v = k, v
    small.table = torch.where(small.table >= 0, small.table + (n_pages - n), small.table)
    q = small.q(16, hd, "bf16")
    _check(small.run(kb, q), *small.want(q))


def test_another_stream_and_a_graph(kb):
    p = Paged(31, [500, 3], [5, 140], 2, 128, 16, "bf16")
    q = p.q(4, 128, "bf16")
    want, tol = p.want(q)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = p.run(kb, q)
        again = p.run(kb, q)
    s.synchronize()
    _check(got, want, tol)
    assert torch.equal(got, again)                                   # the same call gives the same bits
    out = torch.zeros_like(got)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        p.run(kb, q, out=out)
    p.dlens[0] = 300                                                 # other lengths, same shapes
    p.lens[0] = 300
    p.dense[0] = [x[:305] for x in p.dense[0]]
    graph.replay()
    graph.replay()
    torch.cuda.synchronize()
    _check(out, *p.want(q))


# ---- packed prompts -------------------------------------------------------------------------------------------------
def _packed(seed, lens, H, KV, hd, dtype, spread=1.2):
    g = torch.Generator(device="cuda").manual_seed(seed)
    R = sum(lens)
    qkv = (spread * torch.randn(R, (H + 2 * KV) * hd, generator=g, device="cuda")).to(TYPES[dtype])
    q, k, v = qkv[:, :H * hd].unflatten(1, (H, hd)), qkv[:, H * hd:(H + KV) * hd].unflatten(1, (KV, hd)), qkv[:, (H + KV) * hd:].unflatten(1, (KV, hd))
    return q, k, v, torch.tensor(np.concatenate([[0], np.cumsum(lens)]), dtype=torch.int32, device="cuda")


def _packed_want(q, k, v, lens, scale=None):
    outs, at = [], 0
    for n in lens:
        seen = torch.ones(n, n, dtype=torch.bool, device="cuda").tril()
        outs.append(_attend64(q[at:at + n], k[at:at + n], v[at:at + n], seen, q.shape[2] ** -0.5 if scale is None else scale))
        at += n
    return torch.cat([o for o, _ in outs]), torch.cat([t for _, t in outs])


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("H,KV,hd", HEADS)
@pytest.mark.parametrize("lens", [[1], [2, 1, 1], [16], [17, 0, 3], [127], [128, 129, 0], [255, 256, 257, 1], [600, 5, 64]])
def test_packed_prompts(kb, dtype, H, KV, hd, lens):
    q, k, v, start = _packed(sum(lens) + H, lens, H, KV, hd, dtype)
    _check(kb.knnssd_packed_attention(q, k, v, start), *_packed_want(q, k, v, lens))


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("H,KV,hd,lens", [(4, 2, 128, [3001]), (2, 2, 64, [1, 2500, 777]), (10, 2, 128, [1500, 1, 1023])])
def test_long_packed_prompts(kb, dtype, H, KV, hd, lens):
    q, k, v, start = _packed(1, lens, H, KV, hd, dtype)
    _check(kb.knnssd_packed_attention(q, k, v, start), *_packed_want(q, k, v, lens))


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_many_short_prompts(kb, dtype):
    lens = np.random.default_rng(2).integers(0, 40, 300).tolist()
    q, k, v, start = _packed(2, lens, 4, 2, 64, dtype)
    _check(kb.knnssd_packed_attention(q, k, v, start), *_packed_want(q, k, v, lens))


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("lens", [[40, 30], [300, 290, 17]])
def test_prompts_do_not_see_one_another_nor_what_comes(kb, dtype, lens):
    q, k, v, start = _packed(3, lens, 4, 2, 128, dtype)
    at = lens[0]
    v[at // 2, 1, 3] = torch.nan                                     # in the middle of the first prompt
    v[at, 0, 100] = torch.inf                                        # the first row of the second: all of it sees that
    v[at - 1, 0, 64:] = torch.nan                                    # the last row of the first
    want, tol = _packed_want(q, k, v, lens)
    _check(kb.knnssd_packed_attention(q, k, v, start), want, tol)
    k[at + 5:at + 7, 0] = torch.nan                                  # keys of the second prompt
    got = kb.knnssd_packed_attention(q, k, v, start)
    _check(got[:at + 5], want[:at + 5], tol[:at + 5])
    assert got[at + 5:at + lens[1], :2].isnan().all()


def test_packed_rows_that_no_prompt_has(kb):
    q, k, v, start = _packed(4, [70, 60], 4, 2, 64, "bf16")
    start = torch.tensor([0, 70, 100], dtype=torch.int32, device="cuda")
    got = kb.knnssd_packed_attention(q, k, v, start)
    assert got[100:].abs().max() == 0
    _check(got[:100], *_packed_want(q[:100], k[:100], v[:100], [70, 30]))


def test_packed_twice_the_same_bits_and_other_layouts(kb):
    lens = [400, 33, 900]
    q, k, v, start = _packed(6, lens, 8, 2, 128, "bf16")
    got = kb.knnssd_packed_attention(q, k, v, start)
    assert torch.equal(got, kb.knnssd_packed_attention(q, k, v, start))
    assert torch.equal(got, kb.knnssd_packed_attention(q.contiguous(), k.contiguous(), v.contiguous(), start))


# ---- refusals -------------------------------------------------------------------------------------------------------
def test_refusals(kb):
    p = Paged(37, [10], [2], 2, 64, 16, "bf16")
    q = p.q(4, 64, "bf16")
    with pytest.raises(ValueError):
        kb.knnssd_paged_attention(q, p.k, p.v[:1], p.table, p.dlens, p.start)
    with pytest.raises(ValueError):
        kb.knnssd_paged_attention(q.half(), p.k, p.v, p.table, p.dlens, p.start)
    with pytest.raises(ValueError):
        kb.knnssd_paged_attention(q, p.k, p.v, p.table.long(), p.dlens, p.start)
    with pytest.raises(ValueError):
        kb.knnssd_paged_attention(q, p.k, p.v, p.table, p.dlens, p.start[:1])
    with pytest.raises(ValueError):
        kb.knnssd_paged_attention(q.transpose(0, 1), p.k, p.v, p.table, p.dlens, p.start)
    with pytest.raises(ValueError):
        p.run(kb, q, out=torch.empty(2, 4, 64, device="cuda"))

    def status(fn, *args, **kw):
        with pytest.raises(kb.KnnssdError) as e:
            fn(*args, **kw)
        return e.value.status
    assert status(p.run, kb, q[:, :3].contiguous()) == 2             # 3 query heads on 2 K/V heads
    assert status(p.run, kb, q, max_fresh=-1) == 1
    assert status(p.run, kb, q, scale=float("nan")) == 1
    f32 = [x.float() for x in (p.k, p.v)]
    assert status(kb.knnssd_paged_attention, q, *f32, p.table, p.dlens, p.start) == 2       # bf16 rows, fp32 cache
    odd = [x[:, :, :12].contiguous() for x in (p.k, p.v)]
    assert status(kb.knnssd_paged_attention, q, *odd, p.table, p.dlens, p.start) == 2       # pages of 12 positions
    thin = [x[..., :32].contiguous() for x in (p.k, p.v)]
    assert status(kb.knnssd_paged_attention, q[..., :32].contiguous(), *thin, p.table, p.dlens, p.start) == 2
    shifted = torch.zeros(2 * 4 * 64 + 4, dtype=torch.bfloat16, device="cuda")[4:].view(2, 4, 64)
    assert status(p.run, kb, shifted) == 2                           # 8 bytes past a 16-byte boundary
    q, k, v, start = _packed(5, [20], 4, 2, 64, "bf16")
    with pytest.raises(ValueError):
        kb.knnssd_packed_attention(q, k.float(), v, start)
    with pytest.raises(ValueError):
        kb.knnssd_packed_attention(q, k[:10], v[:10], start)
    assert status(kb.knnssd_packed_attention, q[:, :3], k, v, start) == 2
    ragged = torch.zeros(20, 4 * 64 + 2, dtype=torch.bfloat16, device="cuda")[:, :256].unflatten(1, (4, 64))
    assert status(kb.knnssd_packed_attention, ragged, k, v, start) == 2       # rows that are no multiple of 16 bytes apart
    none = kb.knnssd_packed_attention(q[:0], k[:0], v[:0], start)
    assert none.shape == (0, 4, 64)                                  # no rows: nothing to do


@pytest.mark.parametrize("dtype,cache", KINDS)
@pytest.mark.parametrize("KV,lens,fresh", [(2, [30011, 5000], [60, 3]), (8, [700] * 39 + [9000], [2] * 38 + [200, 1])])
def test_a_hint_that_is_too_low_changes_nothing(kb, dtype, cache, KV, lens, fresh):
    p = Paged(23, lens, fresh, KV, 128, 64, cache)
    q = p.q(4 * KV, 128, dtype)
    got = p.run(kb, q, max_fresh=1)
    _check(got, *p.want(q))
    assert torch.equal(got, p.run(kb, q)) and torch.equal(got, p.run(kb, q, max_fresh=300))
