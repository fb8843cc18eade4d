"""The operators over pages in the forms that a launch's sizes choose: large pages and holes of every size, K/V heads in pairs and alone, many query
heads a K/V head, many rows of the store, several threads."""
import threading

import numpy as np
import pytest
import torch

from test_gpu_paged_attention import TYPES, Paged, _attend64, _check, _packed, _packed_want

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def kb():
    if not torch.cuda.is_available():
        pytest.fail("the gpu tests need a CUDA device")
    from paper_2505_16162_b200 import build
    build.build()
    from paper_2505_16162_b200 import binding
    return binding


# ---- pages ------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("page", [16, 64, 128, 256, 2048])
@pytest.mark.parametrize("dtype,cache", [("fp32", "bf16"), ("bf16", "bf16")])
def test_pages_of_any_size(kb, page, dtype, cache):
    p = Paged(103 + page, [700, 0, 2047, 130, 5000], [5, 300, 2, 1, 0], 2, 128, page, cache)
    q = p.q(10, 128, dtype)
    _check(p.run(kb, q), *p.want(q))


@pytest.mark.parametrize("page", [16, 64, 128, 256])
@pytest.mark.parametrize("fresh", [[1, 5, 2, 3], [150, 5, 200, 130]])
def test_holes_of_pages(kb, page, fresh):
    """Whole tiles of 128 positions, halves of them and single pages missing, at the start, in the middle, at the end."""
    lens = [256 - 64, 900, 515, 1000]
    p = Paged(107, lens, fresh, 2, 64, page, "bf16")
    gone = [range(0, 10 ** 6), range(128, 384), range(448, 512), list(range(0, 64)) + list(range(640, 768)) + list(range(960, 1000))]
    cols = [sorted({x // page for x in g if x < p.table.shape[1] * page}) for g in gone]
    for b, c in enumerate(cols):
        for i in c:
            p.table[b, i] = -1 if (b + i) % 2 else p.k.shape[0] + 7
    hide = lambda b: torch.isin(torch.arange(lens[b] + fresh[b], device="cuda") // page, torch.tensor(cols[b], device="cuda"))  # noqa: E731
    q = p.q(6, 64, "bf16")
    want, tol = p.want(q, hide=hide)
    got = p.run(kb, q)
    assert not got[:fresh[0]].any()
    _check(got, want, tol)


@pytest.mark.parametrize("page", [64, 128, 256])
@pytest.mark.parametrize("lens,fresh", [([33], [7]), ([130], [300]), ([4, 250], [16, 129])])
def test_values_that_are_not_finite_in_large_pages(kb, page, lens, fresh):
    p = Paged(109, lens, fresh, 2, 128, page, "bf16")
    for b, (a, n) in enumerate(zip(lens, fresh)):
        for i, val in ((n // 2, torch.inf), (n - 2, torch.nan)):
            p.v[int(p.table[b, (a + i) // page]), 1, (a + i) % page, 5:7] = val
            p.dense[b][1][a + i, 1, 5:7] = val
    q = p.q(6, 128, "bf16")
    want, tol = p.want(q)
    assert want.isnan().any() and not want.isnan().all()
    _check(p.run(kb, q), want, tol)


@pytest.mark.parametrize("page", [64, 256])
def test_lengths_out_of_range_in_large_pages(kb, page):
    p = Paged(113, [40, 10, 300], [2, 2, 2], 2, 64, page, "bf16")
    q = p.q(4, 64, "bf16")
    want, tol = p.want(q)
    p.k.nan_to_num_()
    p.v.nan_to_num_()
    p.dlens[0] = 2 ** 30
    p.dlens[1] = -5
    got = p.run(kb, q)
    _check(got[4:], want[4:], tol[4:])
    assert got.isfinite().all()


# ---- heads ------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("H,KV", [(3, 1), (10, 5), (7, 7)])
@pytest.mark.parametrize("page", [16, 64])
def test_heads_in_pairs_with_one_left(kb, H, KV, page):
    """Items enough that halves of a block take two K/V heads each; an odd number of them leaves one alone."""
    rng = np.random.default_rng(H)
    n = -(-2 * 160 // KV) + 5
    lens, fresh = rng.integers(0, 300, n).tolist(), rng.choice([0, 1, 2, 5, 43, 90], n).tolist()
    p = Paged(127, lens, fresh, KV, 64, page, "bf16")
    q = p.q(H, 64, "bf16")
    _check(p.run(kb, q), *p.want(q))
    n = [int(x) for x in rng.integers(0, 60, n)]
    q, k, v, start = _packed(131, n, H, KV, 64, "bf16")
    _check(kb.knnssd_packed_attention(q, k, v, start), *_packed_want(q, k, v, n))


@pytest.mark.parametrize("H,KV", [(130, 1), (260, 2), (300, 1)])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_more_query_heads_than_a_block_has_rows(kb, H, KV, dtype):
    p = Paged(137, [200, 3, 600], [3, 1, 2], KV, 64, 64, dtype)
    q = p.q(H, 64, dtype)
    _check(p.run(kb, q), *p.want(q))
    q, k, v, start = _packed(139, [5, 140], H, KV, 64, dtype)
    _check(kb.knnssd_packed_attention(q, k, v, start), *_packed_want(q, k, v, [5, 140]))


# ---- the store --------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("rows,H,KV,hd,dtype,cache", [(1025, 40, 8, 128, "bf16", "bf16"), (1500, 3, 1, 128, "fp32", "fp32"), (7, 40, 40, 128, "fp32", "bf16"),
                                                      (1030, 40, 40, 128, "fp32", "bf16"), (9, 70, 70, 64, "bf16", "bf16"), (1024, 5, 5, 64, "fp32", "bf16")])
def test_rotary_store_of_many_rows_and_heads(kb, rows, H, KV, hd, dtype, cache):
    """More than a block's threads take at once: several turns of the heads, the last one ragged.  Against 64 bits: three roundings of the larger term, then the type's."""
    g = torch.Generator(device="cuda").manual_seed(rows)
    page = 16
    n_pages = -(-rows // page) + 2
    qkv = torch.randn(rows, (H + 2 * KV) * hd, generator=g, device="cuda").to(TYPES[dtype])
    rng = np.random.default_rng(rows)
    pos = torch.tensor(rng.integers(0, 5000, rows), dtype=torch.int32, device="cuda")
    slot = torch.tensor(rng.permutation(n_pages * page)[:rows], dtype=torch.int32, device="cuda")
    pos[3], pos[4], slot[5], slot[6] = -1, 5000, -1, n_pages * page
    cs = kb.rotary_table(5000, hd, 10000.0)
    k, v = (torch.randn(n_pages, KV, page, hd, generator=g, device="cuda").to(TYPES[cache]) for _ in range(2))
    k_rows = torch.full((rows, KV, hd), torch.nan, device="cuda", dtype=TYPES[dtype])
    known = (pos >= 0) & (pos < 5000)
    kept = known & (slot >= 0) & (slot < n_pages * page)
    x = qkv.double().view(rows, -1, hd)
    c, s = (cs[pos.clamp(0, 4999).long()][:, None, :, i].double() for i in (0, 1))
    a, b = x[:, :H + KV, :hd // 2], x[:, :H + KV, hd // 2:]
    turned = torch.cat([a * c - b * s, b * c + a * s], -1) * known[:, None, None]
    size = torch.cat([(a * c).abs() + (b * s).abs(), (b * c).abs() + (a * s).abs()], -1) * known[:, None, None]
    by_slot = lambda t: t.transpose(1, 2).reshape(-1, KV, hd)  # noqa: E731
    want_k, want_v = by_slot(k).double().clone(), by_slot(v).clone()
    want_k[slot[kept].long()], want_v[slot[kept].long()] = turned[kept, H:], x[kept, H + KV:].to(v.dtype)
    tol_k = torch.zeros_like(want_k)
    tol_k[slot[kept].long()] = size[kept, H:]
    q = kb.knnssd_rotary_store(qkv, cs, pos, slot, k, v, k_rows=k_rows)
    eps = lambda t: (3 * 2.0 ** -24 + (2.0 ** -8 if t == "bf16" else 0.0)) * (1 + 2.0 ** -8)  # noqa: E731
    assert ((q.double() - turned[:, :H]).abs() <= eps(dtype) * size[:, :H]).all()
    assert ((k_rows.double() - turned[:, H:]).abs() <= eps(dtype) * size[:, H:]).all()
    assert ((by_slot(k).double() - want_k).abs() <= eps(cache) * tol_k).all()
    assert torch.equal(by_slot(v), want_v)


# ---- threads ----------------------------------------------------------------------------------------------------------
def test_several_threads_at_once(kb):
    sets = []
    for i, dtype in enumerate(["bf16", "fp32", "bf16", "fp32"]):
        p = Paged(149 + i, [300 + 70 * i, 20, 9000], [3, 150, 1], 2, 64, (16, 64)[i // 2], "bf16")
        q = p.q(4, 64, dtype)
        sets.append((p, q, p.run(kb, q)))
    torch.cuda.synchronize()
    failed = []

    def work(p, q, want):
        try:
            s = torch.cuda.Stream()
            with torch.cuda.stream(s):
                outs = [p.run(kb, q) for _ in range(60)]
            s.synchronize()
            if not all(torch.equal(o, want) for o in outs):
                failed.append("another result")
        except Exception as e:                                       # noqa: BLE001
            failed.append(repr(e))

    threads = [threading.Thread(target=work, args=a) for a in sets]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not failed, failed
