"""Block tables, slot maps and the rows' way into the pages: integers exactly, rotated values within the roundings of fp32."""
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


class Pool:
    """The state on the GPU, and the same state stepped one page at a time on the host."""

    def __init__(self, n_requests, page, max_pages, n_pages, max_rows, seed=0):
        self.page, self.n_pages, self.max_pages, self.max_rows = page, n_pages, max_pages, max_rows
        ids = np.random.default_rng(seed).permutation(n_pages).astype(np.int32)
        self.host = {"owned": np.zeros(n_requests, np.int32), "table": np.full((n_requests, max_pages), -1, np.int32), "free": ids, "count": n_pages}
        self.owned, self.table, self.free, self.count = (torch.as_tensor(np.array(x, dtype=np.int32), device="cuda") for x in
                                                         (self.host["owned"], self.host["table"], ids, [n_pages]))
        zeros = lambda n: torch.full((n,), 77, dtype=torch.int32, device="cuda")  # noqa: E731
        self.start, self.request, self.pos, self.slot, self.info = zeros(n_requests + 1), zeros(max_rows), zeros(max_rows), zeros(max_rows), zeros(4)

    def step(self, kb, lens, fresh):
        kb.knnssd_page_tables(torch.tensor(lens, dtype=torch.int32, device="cuda"), torch.tensor(fresh, dtype=torch.int32, device="cuda"), self.owned, self.table,
                              self.free, self.count, self.page, self.start, self.request, self.pos, self.slot, self.info)

    def step_host(self, lens, fresh):
        h = self.host
        bad = 0
        need = []
        for a, n, have in zip(lens, fresh, h["owned"]):
            if a < 0 or n < -1 or have < 0 or have > self.max_pages:
                bad |= 8
                need.append(int(have))
                continue
            need.append(0 if n < 0 else -(-(a + n) // self.page))
            if need[-1] > self.max_pages:
                bad |= 2
        rows = sum(max(n, 0) for a, n in zip(lens, fresh) if a >= 0)
        given = sum(max(int(o) - n, 0) for o, n in zip(h["owned"], need))
        taken = sum(max(n - int(o), 0) for o, n in zip(h["owned"], need))
        if rows > self.max_rows:
            bad |= 4
        if taken > h["count"] + given:
            bad |= 1
        if bad:
            return {"info": [0, 0, 0, bad], "start": [0] * (len(lens) + 1), "rows": []}
        for b, n in enumerate(need):
            for p in range(n, int(h["owned"][b])):
                h["free"][h["count"]] = h["table"][b, p]
                h["count"] += 1
                h["table"][b, p] = -1
        for b, n in enumerate(need):
            for p in range(int(h["owned"][b]), n):
                h["count"] -= 1
                h["table"][b, p] = h["free"][h["count"]]
        out, start = [], [0]
        for b, (a, n) in enumerate(zip(lens, fresh)):
            for i in range(max(n, 0)):
                out.append((b, a + i, int(h["table"][b, (a + i) // self.page]) * self.page + (a + i) % self.page))
            start.append(len(out))
        h["owned"][:] = need
        return {"info": [rows, taken, given, 0], "start": start, "rows": out}

    def compare(self, want):
        h = self.host
        assert self.info.tolist() == want["info"]
        assert self.start.tolist() == want["start"]
        assert np.array_equal(self.owned.cpu().numpy(), h["owned"]) and np.array_equal(self.table.cpu().numpy(), h["table"])
        assert int(self.count) == h["count"] and np.array_equal(self.free.cpu().numpy(), h["free"])
        rows = want["rows"] + [(-1, -1, -1)] * (self.max_rows - len(want["rows"]))
        assert list(zip(self.request.tolist(), self.pos.tolist(), self.slot.tolist())) == rows


@pytest.mark.parametrize("n,page,max_rows", [(1, 16, 64), (3, 16, 700), (40, 32, 1500), (300, 16, 5000), (1025, 128, 9000), (2500, 16, 12000)])
def test_steps_of_a_server(kb, n, page, max_rows):
    rng = np.random.default_rng(n)
    pool = Pool(n, page, 40, 9 * n + 60, max_rows)
    lens = np.zeros(n, np.int64)
    for step in range(7):
        fresh = rng.integers(0, 6, n)
        fresh[rng.random(n) < 0.1] = -1
        starts = rng.integers(0, n, max(1, n // 40))
        fresh[starts] = rng.integers(0, min(90, max_rows // 4), len(starts))
        want = pool.step_host(lens.tolist(), fresh.tolist())
        pool.step(kb, lens.tolist(), fresh.tolist())
        pool.compare(want)
        assert want["info"][3] in (0, 1, 4)
        if want["info"][3] == 0:                                     # some of the new rows are kept
            lens = np.where(fresh < 0, 0, lens + rng.integers(0, np.maximum(fresh, 0) + 1))


def test_a_request_grows_to_its_last_page_and_back(kb):
    pool = Pool(2, 16, 5, 9, 150)
    for lens, fresh in (([0, 0], [80, 64]), ([80, 64], [0, 0]), ([79, 1], [1, 0]), ([17, 16], [0, 0]), ([16, 0], [0, -1]), ([0, 0], [0, 0]), ([0, 5], [-1, 11])):
        want = pool.step_host(lens, fresh)
        pool.step(kb, lens, fresh)
        pool.compare(want)
        assert want["info"][3] == 0


@pytest.mark.parametrize("lens,fresh,code", [([0, 0], [200, 0], 2), ([0, 0], [80, 80], 1), ([0, 0], [60, 60], 4), ([-1, 0], [1, 1], 8), ([0, 0], [-2, 1], 8), ([0, 2 ** 31 - 1], [1, 2 ** 31 - 1], 6)])
def test_a_step_that_does_not_fit_changes_nothing(kb, lens, fresh, code):
    pool = Pool(2, 16, 5, 9, 100 if code != 1 else 400)
    first = pool.step_host([0, 0], [20, 3])
    pool.step(kb, [0, 0], [20, 3])
    pool.compare(first)
    want = pool.step_host(lens, fresh)
    assert want["info"][3] & code == code
    pool.step(kb, lens, fresh)
    assert int(pool.info[3]) & code == code
    want["info"] = pool.info.tolist()
    assert want["info"][:3] == [0, 0, 0]
    pool.compare(want)
    again = pool.step_host([20, 3], [5, 5])                          # and the next step goes on from the state before
    pool.step(kb, [20, 3], [5, 5])
    pool.compare(again)


def test_damaged_state_is_refused(kb):
    for name, value in (("owned", 9), ("owned", -1), ("count", 10), ("count", -1)):
        pool = Pool(2, 16, 5, 9, 100)
        getattr(pool, name)[0] = value
        before = pool.table.clone(), pool.free.clone()
        pool.step(kb, [0, 0], [5, 5])
        assert pool.info.tolist() == [0, 0, 0, 8]
        assert torch.equal(pool.table, before[0]) and torch.equal(pool.free, before[1]) and int(getattr(pool, name)[0]) == value


def test_no_rows_wanted_and_refusals(kb):
    pool = Pool(2, 16, 5, 9, 0)
    pool.step(kb, [40, 3], [0, 0])
    assert pool.info.tolist() == [0, 4, 0, 0]
    args = lambda p: (torch.zeros(2, dtype=torch.int32, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda"), p.owned, p.table, p.free, p.count)  # noqa: E731
    rest = lambda p: (p.start, p.request, p.pos, p.slot, p.info)  # noqa: E731
    for page in (0, 8, 24):
        with pytest.raises(kb.KnnssdError) as e:
            kb.knnssd_page_tables(*args(pool), page, *rest(pool))
        assert e.value.status == (1 if page == 0 else 2)
    with pytest.raises(kb.KnnssdError) as e:
        kb.knnssd_page_tables(*args(pool), 2 ** 28, *rest(pool))
    assert e.value.status == 3
    with pytest.raises(ValueError):
        kb.knnssd_page_tables(*args(pool), 16, pool.start[:2].contiguous(), *rest(pool)[1:])
    big = Pool(8193, 16, 1, 4, 4)
    with pytest.raises(kb.KnnssdError) as e:
        big.step(kb, [0] * 8193, [0] * 8193)
    assert e.value.status == 3
    most = Pool(8192, 16, 2, 100, 50)
    fresh = [1 if b % 300 == 299 else 0 for b in range(8192)]
    want = most.step_host([0] * 8192, fresh)
    most.step(kb, [0] * 8192, fresh)
    most.compare(want)


# ---- rotary embedding and store ---------------------------------------------------------------------------------------
def _store64(qkv, cs, pos, slot, k, v):
    """64-bit values; what is not written stays."""
    n_pages, KV, page, hd = k.shape
    x = qkv.double().view(qkv.shape[0], -1, hd)
    H = x.shape[1] - 2 * KV
    k, v = k.double().clone(), v.double().clone()
    q = torch.zeros(qkv.shape[0], H, hd, dtype=torch.float64, device="cuda")
    size = torch.zeros_like(q), torch.zeros_like(k)
    for r in range(qkv.shape[0]):
        p, s = int(pos[r]), int(slot[r])
        if p < 0 or p >= cs.shape[0]:
            continue
        c, sn = cs[p, :, 0].double(), cs[p, :, 1].double()
        a, b = x[r, :H + KV, :hd // 2], x[r, :H + KV, hd // 2:]
        turned = torch.cat([a * c - b * sn, b * c + a * sn], -1)
        most = torch.cat([(a * c).abs() + (b * sn).abs(), (b * c).abs() + (a * sn).abs()], -1)
        q[r], size[0][r] = turned[:H], most[:H]
        if 0 <= s < n_pages * page:
            k[s // page, :, s % page], size[1][s // page, :, s % page] = turned[H:], most[H:]
            v[s // page, :, s % page] = x[r, H + KV:]
    return q, k, v, size


@pytest.mark.parametrize("dtype,cache", [("fp32", "fp32"), ("fp32", "bf16"), ("bf16", "bf16")])
@pytest.mark.parametrize("H,KV,hd", [(4, 4, 64), (40, 8, 128), (3, 1, 128), (8, 2, 64)])
@pytest.mark.parametrize("rows,page", [(1, 16), (5, 32), (61, 16)])
def test_rotary_store(kb, dtype, cache, H, KV, hd, rows, page):
    g = torch.Generator(device="cuda").manual_seed(rows + H)
    n_pages = -(-rows // page) + 2
    wide = torch.randn(rows, (H + 2 * KV) * hd + 16, generator=g, device="cuda").to(TYPES[dtype])
    qkv = wide[:, 8:8 + (H + 2 * KV) * hd] if dtype == "bf16" else wide[:, 4:4 + (H + 2 * KV) * hd]
    rng = np.random.default_rng(rows)
    pos = torch.tensor(rng.integers(0, 5000, rows), dtype=torch.int32, device="cuda")
    slot = torch.tensor(rng.permutation(n_pages * page)[:rows], dtype=torch.int32, device="cuda")
    if rows > 8:
        pos[3], pos[4], slot[5], slot[6] = -1, 5000, -1, n_pages * page      # padding, outside the table, no slot, outside the pool
    cs = kb.rotary_table(5000, hd, 10000.0)
    k, v = (torch.randn(n_pages, KV, page, hd, generator=g, device="cuda").to(TYPES[cache]) for _ in range(2))
    wq, wk, wv, size = _store64(qkv.contiguous(), cs, pos, slot, k, v)
    q = kb.knnssd_rotary_store(qkv, cs, pos, slot, k, v)
    # two products and a sum in fp32: 3 roundings of the larger term; then the type's own rounding
    eps = lambda t: 3 * 2.0 ** -24 + (2.0 ** -8 if t == "bf16" else 0.0)  # noqa: E731
    assert ((q.double() - wq).abs() <= eps(dtype) * size[0] * (1 + 2.0 ** -8)).all()
    assert ((k.double() - wk).abs() <= eps(cache) * size[1] * (1 + 2.0 ** -8)).all()
    assert torch.equal(v, wv.to(v.dtype))
    if rows > 8:
        assert q[3:5].abs().max() == 0 and q[5:7].abs().max() > 0


def test_rotary_store_refusals(kb):
    k, v = (torch.zeros(3, 2, 16, 64, device="cuda") for _ in range(2))
    cs = kb.rotary_table(10, 64, 10000.0)
    i32 = lambda n: torch.zeros(n, dtype=torch.int32, device="cuda")  # noqa: E731
    qkv = torch.zeros(4, 8 * 64, device="cuda")
    with pytest.raises(ValueError):
        kb.knnssd_rotary_store(qkv[:, :4 * 64], cs, i32(4), i32(4), k, v)    # no q heads
    with pytest.raises(ValueError):
        kb.knnssd_rotary_store(qkv, cs[:, :16], i32(4), i32(4), k, v)
    with pytest.raises(ValueError):
        kb.knnssd_rotary_store(qkv, cs, i32(3), i32(4), k, v)
    with pytest.raises(ValueError):
        kb.knnssd_rotary_store(qkv, cs, i32(4), i32(4), k, v, q=torch.zeros(4, 4, 64, device="cuda").bfloat16())
    with pytest.raises(kb.KnnssdError) as e:
        kb.knnssd_rotary_store(qkv.bfloat16(), cs, i32(4), i32(4), k, v)     # bf16 rows, fp32 cache
    assert e.value.status == 2
    assert kb.knnssd_rotary_store(qkv[:0], cs, i32(0), i32(0), k, v).shape == (0, 4, 64)


def test_slots_beyond_32_bits_of_elements(kb):
    KV, hd, page = 8, 128, 64
    n_pages = 2 ** 31 // (KV * hd * page) + 5
    k, v = (torch.empty((n_pages, KV, page, hd), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    k[-1], v[-1] = 0, 0
    qkv = torch.randn(2, 24 * hd, device="cuda").bfloat16()
    cs = kb.rotary_table(4, hd, 10000.0)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    kb.knnssd_rotary_store(qkv, cs, i32([0, 0]), i32([n_pages * page - 1, n_pages * page - 2]), k, v)
    assert torch.equal(k[-1, :, -1], qkv[0].view(24, hd)[8:16]) and torch.equal(v[-1, :, -2], qkv[1].view(24, hd)[16:])


@pytest.mark.parametrize("dtype,cache,H,KV,hd", [("fp32", "bf16", 4, 2, 64), ("bf16", "bf16", 40, 8, 128), ("fp32", "fp32", 3, 1, 128)])
def test_rotated_k_by_rows(kb, dtype, cache, H, KV, hd):
    rows, page = 37, 16
    g = torch.Generator(device="cuda").manual_seed(H)
    qkv = torch.randn(rows, (H + 2 * KV) * hd, generator=g, device="cuda").to(TYPES[dtype])
    pos = torch.arange(100, 100 + rows, dtype=torch.int32, device="cuda")
    slot = torch.arange(rows, dtype=torch.int32, device="cuda")
    pos[3], pos[4], slot[5] = -1, 5000, -1                                   # no position twice, a position without a slot
    cs = kb.rotary_table(5000, hd, 10000.0)
    k, v = (torch.zeros(3, KV, page, hd, device="cuda", dtype=TYPES[cache]) for _ in range(2))
    k0, v0 = k.clone(), v.clone()
    q0 = kb.knnssd_rotary_store(qkv, cs, pos, slot, k0, v0)
    got = torch.full((rows, KV, hd), float("nan"), device="cuda", dtype=TYPES[dtype])
    q = kb.knnssd_rotary_store(qkv, cs, pos, slot, k, v, k_rows=got)
    assert torch.equal(q, q0) and torch.equal(k, k0) and torch.equal(v, v0)  # nothing else changes by it
    assert got[3:5].abs().max() == 0 and got[5].abs().max() > 0
    by_slot = k.permute(0, 2, 1, 3).reshape(-1, KV, hd)                      # [slot][head][dim]
    live = [r for r in range(rows) if r not in (3, 4, 5)]
    assert torch.equal(got[live].to(TYPES[cache]), by_slot[live])
    with pytest.raises(ValueError):
        kb.knnssd_rotary_store(qkv, cs, pos, slot, k, v, k_rows=got[:, :, :32])
    with pytest.raises(ValueError):
        kb.knnssd_rotary_store(qkv, cs, pos, slot, k, v, k_rows=got.double())
