"""Tables of a tree's rows and their attention over pages, against the oracle's words and a plain evaluation in 64 bits.

Tolerances are those of attention over pages (``test_gpu_paged_attention``): the arithmetic is the same, a row sees fewer positions.
"""
import numpy as np
import pytest
import torch

from oracle import trees as ot
from test_gpu_paged_attention import HEADS, KINDS, Paged, _check

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
    """A tree whose rows follow one of the `back` rows before them; with back 0, several of them nothing at all."""
    if back == 0:
        return [-1 if i == 0 or rng.random() < 0.2 else int(rng.integers(0, i)) for i in range(n)]
    return [max(0, i - int(rng.integers(1, back + 1))) if i else -1 for i in range(n)]


def _tables(kb, lens, parents, before=0, behind=0):
    """What the library makes of the requests' parents, with rows of nobody around them."""
    start = torch.tensor(np.cumsum([before] + [len(p) for p in parents]), **I32)
    R = int(start[-1]) + behind
    parent = torch.full((R,), 5, **I32)
    parent[before:R - behind] = torch.tensor([x for p in parents for x in p], **I32)
    pos, seen, state = torch.full((R,), 77, **I32), torch.full((R,), 77, dtype=torch.int64, device="cuda"), torch.full((len(parents),), 77, **I32)
    kb.knnssd_tree_tables(torch.tensor(lens, **I32), start, parent, pos, seen, state)
    return start, pos, seen, state


def _signed(word):
    return word - (1 << 64) if word >> 63 else word


TREES = [
    [[-1]], [[-1, 0, 0, 1, 1, 2]], [list(range(-1, 63))], [list(range(-1, 64))], [list(range(-1, 699))],
    [[-1] + [0] * 63], [[-1] + [0] * 64], [[-1] + [0] * 65],                     # the last: row 65 does not follow row 1
    [list(range(-1, 300)) + [300] * 63], [list(range(-1, 300)) + [299] * 63], [list(range(-1, 300)) + [300] * 64, [-1, 0]],
    [[-1, -1, 0, 1]], [[-1] * 64], [[-1] * 65], [[-1, 0, 3], [-1, 0]], [[-1, -2]], [[0]], [[-1, 1]], [[], [-1, 0], []],
    [list(range(-1, 70)) + [3]], [list(range(-1, 63)) + [0]], [list(range(-1, 64)) + [0]], [list(range(-1, 64)) + [1]], [[-1, 0, 0] + list(range(2, 63)) + [63]],
]


@pytest.mark.parametrize("at", range(len(TREES)))
def test_tables_of_small_trees(kb, at):
    parents, lens = TREES[at], [9 + 100 * b for b in range(len(TREES[at]))]
    start, pos, seen, state = _tables(kb, lens, parents, before=2, behind=3)
    assert pos[:2].tolist() == [-1] * 2 and pos[-3:].tolist() == [-1] * 3 and seen[:2].tolist() == [0] * 2 and seen[-3:].tolist() == [0] * 3
    for b, p in enumerate(parents):
        rows = slice(int(start[b]), int(start[b + 1]))
        want = ot.words(p)
        assert int(state[b]) == (want is None)
        assert pos[rows].tolist() == ([-1] * len(p) if want is None else [lens[b] + int(d) for d in want[0]])
        assert seen[rows].tolist() == ([0] * len(p) if want is None else [_signed(w) for w in want[1]])


def test_tables_of_many_requests(kb):
    rng = np.random.default_rng(3)
    parents = [_parents(rng, int(n), int(back)) for n, back in zip(rng.integers(0, 65, 900), rng.integers(0, 12, 900))]
    for b in range(5, 900, 50):
        parents[b] = list(range(-1, int(rng.integers(1, 800)))) + [0] * (b % 3 == 0)
    lens = rng.integers(0, 5000, 900).tolist()
    lens[17], lens[18] = -1, 2 ** 31 - 1
    start, pos, seen, state = _tables(kb, lens, parents)
    want = [None if not 0 <= m < 2 ** 31 - 1000 and p else ot.words(p) for m, p in zip(lens, parents)]
    want[17] = None
    assert state.tolist() == [int(w is None) for w in want]
    assert pos.tolist() == [x for m, p, w in zip(lens, parents, want) for x in ([-1] * len(p) if w is None else (m + w[0]).tolist())]
    assert seen.tolist() == [x for p, w in zip(parents, want) for x in ([0] * len(p) if w is None else map(_signed, w[1]))]


class Trees(Paged):
    """Requests whose new rows are trees, or see what the words in `words` say."""

    def __init__(self, kb, seed, lens, parents, *args, words=None, **kw):
        super().__init__(seed, lens, [len(p) for p in parents], *args, **kw)
        if words is None:
            _, self.pos, self.words, state = _tables(kb, lens, parents)
            assert not state.any()
            made = [ot.words(p)[1] for p in parents]
            assert self.words.tolist() == [_signed(w) for m in made for w in m]
        else:
            made = words
            self.words = torch.tensor([_signed(w) for m in words for w in m], dtype=torch.int64, device="cuda")
        self.made = made

    def seen(self, b):
        m, n = self.lens[b], self.fresh[b]
        return torch.as_tensor(np.stack([ot.seen(m + n, m + i, self.made[b][i]) for i in range(n)]) if n else np.zeros((0, m), bool), device="cuda")

    def run(self, kb, q, **kw):
        return kb.knnssd_tree_attention(q, self.k, self.v, self.table, self.dlens, self.start, self.words, **kw)


def _wider(table, by):
    return torch.cat([table, torch.full((table.shape[0], by), -1, **I32)], dim=1).contiguous()


# (lengths held, rows and how far back their parents lie, of each request)
LENGTHS = [
    ([0], [(1, 1)]), ([95], [(13, 4)]), ([0], [(64, 20)]), ([15], [(30, 0)]), ([1280], [(25, 5)]), ([63], [(64, 63)]),
    ([0, 31, 700, 3, 64, 127], [(1, 1), (40, 7), (64, 64), (0, 1), (16, 3), (2, 1)]),
    ([5, 0, 0, 500, 1], [(0, 1), (64, 0), (150, 1), (64, 9), (33, 2)]),
]


@pytest.mark.parametrize("dtype,cache", KINDS)
@pytest.mark.parametrize("H,KV,hd", HEADS)
@pytest.mark.parametrize("at", range(len(LENGTHS)))
def test_trees_over_pages(kb, dtype, cache, H, KV, hd, at):
    lens, rows = LENGTHS[at]
    rng = np.random.default_rng(50 + at)
    page = (16, 32, 64, 128)[(at + H) % 4]
    p = Trees(kb, 7 * at + H, lens, [_parents(rng, *r) for r in rows], KV, hd, page, cache)
    q = p.q(H, hd, dtype)
    want, tol = p.want(q)
    for wide in (p.table, _wider(p.table, 5000 // page)):            # tables with room for short contexts, and for long ones
        p.table = wide
        for hint in (0, max(p.fresh)):
            _check(p.run(kb, q, max_fresh=hint), want, tol, f"{wide.shape[1]} pages, max_fresh {hint}")


@pytest.mark.parametrize("dtype,cache", KINDS)
@pytest.mark.parametrize("H,KV,hd,page", [(4, 2, 64, 16), (10, 2, 128, 64), (3, 3, 128, 16)])
@pytest.mark.parametrize("more", [0, 5000])
def test_words_of_all_kinds(kb, dtype, cache, H, KV, hd, page, more):
    """Words that come of no tree: none of 64, one, all but its own, random ones; rows of a short request that see nothing."""
    rng = np.random.default_rng(H)
    lens, fresh = [0, 20, 200, 1000, 0], [7, 40, 150, 3, 64]
    kinds = [lambda i: 0, lambda i: 1, lambda i: (1 << 64) - 2, lambda i: int(rng.integers(0, 1 << 63)) * 2 + int(rng.integers(0, 2)), lambda i: 1 << 63, lambda i: 1 << (i % 64)]
    words = [[kinds[(i + b) % len(kinds)](i) for i in range(n)] for b, n in enumerate(fresh)]
    p = Trees(kb, 3, lens, [[-1] * n for n in fresh], KV, hd, page, cache, words=words, wide=2 + more // page)
    q = p.q(H, hd, dtype)
    want, tol = p.want(q)
    got = p.run(kb, q)
    assert got[0].abs().max() == 0 and not want[0].any()             # word 0, nothing held
    _check(got, want, tol)


@pytest.mark.parametrize("dtype,cache", KINDS)
@pytest.mark.parametrize("lens,fresh", [([300, 0, 77], [5, 64, 200]), ([20011], [1]), ([40] * 300, [3] * 300)])
def test_chains_are_the_rows_of_paged_attention(kb, dtype, cache, lens, fresh):
    """To the bit for bf16 rows where the table has room for long contexts, which is the same kernel."""
    for wide in (300, 2):
        p = Trees(kb, 9, lens, [list(range(-1, n - 1)) for n in fresh], 2, 128, 16, cache, wide=wide)
        q = p.q(6, 128, dtype)
        got = p.run(kb, q)
        assert wide == 2 or dtype == "fp32" or torch.equal(got, Paged.run(p, kb, q))
        _check(got, *p.want(q))


@pytest.mark.parametrize("dtype,cache", KINDS)
@pytest.mark.parametrize("H,KV,hd,lens,rows", [(8, 2, 128, [20011], [(48, 12)]), (4, 4, 64, [9000, 40, 13000], [(3, 2), (64, 8), (25, 5)]), (10, 2, 128, [5000, 0], [(64, 20), (64, 3)])])
def test_long_contexts_in_many_parts(kb, dtype, cache, H, KV, hd, lens, rows):
    rng = np.random.default_rng(2)
    p = Trees(kb, 3, lens, [_parents(rng, *r) for r in rows], KV, hd, 64, cache)
    q = p.q(H, hd, dtype)
    _check(p.run(kb, q), *p.want(q))


@pytest.mark.parametrize("dtype,cache", KINDS)
@pytest.mark.parametrize("H,KV,n,most", [(2, 1, 300, 40), (8, 1, 700, 90), (3, 1, 1000, 20)])
def test_more_requests_than_a_block_has_threads(kb, dtype, cache, H, KV, n, most):
    rng = np.random.default_rng(n)
    p = Trees(kb, n, rng.integers(0, most, n).tolist(), [_parents(rng, int(r), 2) for r in rng.integers(0, 3, n)], KV, 64, 16, cache)
    q = p.q(H, 64, dtype)
    want, tol = p.want(q)
    for table in (p.table, _wider(p.table, 300)):
        p.table = table
        _check(p.run(kb, q), want, tol)


@pytest.mark.parametrize("dtype,cache", KINDS)
def test_many_requests_of_all_lengths(kb, dtype, cache):
    rng = np.random.default_rng(5)
    n = 400
    p = Trees(kb, 5, rng.integers(0, 90, n).tolist(), [_parents(rng, int(r), 4) for r in rng.integers(0, 9, n)], 2, 64, 16, cache)
    q = p.q(6, 64, dtype)
    _check(p.run(kb, q, max_fresh=8), *p.want(q))


@pytest.mark.parametrize("dtype,cache", KINDS)
@pytest.mark.parametrize("lens,rows", [([33], [(20, 4)]), ([130, 2], [(64, 9), (64, 0)]), ([700], [(64, 30)])])
@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("more", [0, 5000])
def test_what_is_not_finite_reaches_only_rows_that_see_it(kb, dtype, cache, lens, rows, page, more):
    """Siblings' K and V, and the rows' that a row has behind it, play no part whatever they are."""
    rng = np.random.default_rng(8)
    p = Trees(kb, 13, lens, [_parents(rng, *r) for r in rows], 2, 128, page, cache, wide=2 + more // page)
    for b, (a, n) in enumerate(zip(lens, p.fresh)):
        for i, val in ((n // 2, torch.inf), (n - 2, torch.nan), (3, -torch.inf)):
            at, off = int(p.table[b, (a + i) // page]), (a + i) % page
            p.v[at, 1, off, 5:7] = val
            p.dense[b][1][a + i, 1, 5:7] = val
    q = p.q(6, 128, dtype)
    want, tol = p.want(q)
    assert want.isnan().any() and not want.isnan().all()
    _check(p.run(kb, q), want, tol)
    # a key that is not finite makes the rows NaN that see it, and no other
    b, i = 0, p.fresh[0] // 3
    p.k[int(p.table[b, (lens[b] + i) // page]), 0, (lens[b] + i) % page] = torch.nan
    hit = torch.tensor([bool(p.seen(b)[r, lens[b] + i]) for r in range(p.fresh[0])], device="cuda")
    got = p.run(kb, q)
    assert got[:p.fresh[0]][hit][:, :3].isnan().all()
    want[:p.fresh[0]][hit.nonzero()[:, 0], :3] = torch.nan
    rest = torch.ones_like(want, dtype=torch.bool)
    rest[:p.fresh[0]][hit.nonzero()[:, 0], :3] = False
    _check(got[rest], want[rest], tol[rest])


@pytest.mark.parametrize("dtype,cache", KINDS)
@pytest.mark.parametrize("wide", [2, 300])
def test_pages_that_are_gone(kb, dtype, cache, wide):
    rng = np.random.default_rng(4)
    p = Trees(kb, 11, [40, 100, 0], [_parents(rng, 30, 5), _parents(rng, 64, 9), _parents(rng, 20, 2)], 2, 64, 16, cache, wide=wide)
    gone = {0: range(0, 99), 1: (0, 6, 7), 2: (0,)}
    for b, cols in gone.items():
        for c in cols:
            if c < p.table.shape[1]:
                p.table[b, c] = -1 if (b + c) % 2 else p.k.shape[0] + 7
    hide = lambda b: torch.isin(torch.arange(p.lens[b] + p.fresh[b], device="cuda") // 16, torch.tensor(list(gone[b]), device="cuda"))  # noqa: E731
    q = p.q(4, 64, dtype)
    want, tol = p.want(q, hide=hide)
    got = p.run(kb, q)
    assert got[:30].abs().max() == 0 and not want[:30].any()
    _check(got, want, tol)


@pytest.mark.parametrize("dtype,cache", KINDS)
def test_a_tree_level_by_level(kb, dtype, cache):
    """The words of a tree's rows hold for calls of some of its rows, the rows before counted as held."""
    parents = [[-1, 0, 0, 0, 1, 1, 2, 3, 4, 5, 5, 7], [-1, 0, 0, 1, 2, 2, 2, 3, 4, 6, 6, 6]]
    levels = [(0, 1), (1, 4), (4, 8), (8, 12)]
    p = Trees(kb, 21, [100, 7], parents, 2, 128, 16, cache)
    q = p.q(6, 128, dtype)
    want, tol = p.want(q)
    for a, z in levels:
        rows = torch.tensor([12 * b + i for b in range(2) for i in range(a, z)], device="cuda")
        got = kb.knnssd_tree_attention(q[rows], p.k, p.v, p.table, p.dlens + a, torch.tensor([0, z - a, 2 * (z - a)], **I32), p.words[rows])
        _check(got, want[rows], tol[rows], f"rows {a} .. {z - 1}")


@pytest.mark.parametrize("wide", [2, 300])
def test_rows_of_nobody_and_strides(kb, wide):
    rng = np.random.default_rng(6)
    p = Trees(kb, 19, [64, 5], [_parents(rng, 9, 3), _parents(rng, 4, 2)], 2, 64, 32, "bf16", wide=wide)
    wide = torch.randn(20, 6 * 64 + 72, device="cuda").bfloat16()
    q = wide[:, 8:8 + 6 * 64].unflatten(1, (6, 64))
    p.words = torch.cat([torch.full((3,), -1, dtype=torch.int64, device="cuda"), p.words, torch.full((4,), -1, dtype=torch.int64, device="cuda")])
    p.start += 3
    got = p.run(kb, q)
    assert got[:3].abs().max() == 0 and got[16:].abs().max() == 0
    p.start -= 3
    _check(got[3:16], *p.want(q[3:16]))
    out = torch.empty_like(got)
    p.start += 3
    assert p.run(kb, q, out=out) is out and torch.equal(out, got)


@pytest.mark.parametrize("dtype,cache", KINDS)
@pytest.mark.parametrize("wide", [2, 300])
def test_lengths_out_of_range_stay_inside_the_pool(kb, dtype, cache, wide):
    rng = np.random.default_rng(1)
    p = Trees(kb, 23, [40, 10, 30], [_parents(rng, 8, 3) for _ in range(3)], 2, 64, 16, cache, wide=wide)
    q = p.q(4, 64, dtype)
    want, tol = p.want(q)
    p.k.nan_to_num_()
    p.v.nan_to_num_()
    p.dlens[0], p.dlens[1] = 2 ** 30, -5
    got = p.run(kb, q)
    _check(got[16:], want[16:], tol[16:])
    assert got.isfinite().all()
    p.start[3] = 1000
    assert p.run(kb, q).isfinite().all()


def test_pool_beyond_32_bits(kb):
    KV, hd, page = 8, 128, 64
    n_pages = 2 ** 31 // (KV * hd * page) + 40
    k = torch.empty((n_pages, KV, page, hd), dtype=torch.bfloat16, device="cuda")
    v = torch.empty_like(k)
    rng = np.random.default_rng(1)
    small = Trees(kb, 29, [1000], [_parents(rng, 20, 4)], KV, hd, page, "bf16", spare=0)
    n = small.k.shape[0]
    k[-n:], v[-n:] = small.k, small.v
    small.k, small.v = k, v
    small.table = torch.where(small.table >= 0, small.table + (n_pages - n), small.table)
    for dtype in ("bf16", "fp32"):
        q = small.q(16, hd, dtype)
        _check(small.run(kb, q), *small.want(q))


def test_refusals_of_the_binding(kb):
    rng = np.random.default_rng(1)
    p = Trees(kb, 37, [10], [_parents(rng, 6, 2)], 2, 64, 16, "bf16")
    q = p.q(4, 64, "bf16")
    good = p.words
    for words in (good.int(), good[:5], good.cpu(), torch.stack([good, good], 1)[:, 0]):
        p.words = words
        with pytest.raises(ValueError):
            p.run(kb, q)
    p.words = good
    with pytest.raises(ValueError):
        kb.knnssd_tree_attention(q.half(), p.k, p.v, p.table, p.dlens, p.start, p.words)
    with pytest.raises(ValueError):
        kb.knnssd_tree_tables(p.dlens, p.start, p.start, torch.zeros(2, **I32), good[:2], torch.zeros(2, **I32))
    state = torch.full((1,), 5, **I32)
    none, words = torch.empty(0, **I32), torch.empty(0, dtype=torch.int64, device="cuda")
    kb.knnssd_tree_tables(p.dlens, torch.zeros(2, **I32), none, none, words, state)
    assert state.tolist() == [0]
