"""Several requests on one paged K/V cache, as cases that can be timed and compared.

The decode path of this library serves one request from one contiguous cache.  The four operators here are what a
program needs that keeps the caches of many requests in pages of one pool and drafts and verifies for all of them at
once (k drafts and the pending token: k + 1 new rows per request and pass), or reads their prompts packed one behind
the other:

  tables   block tables and slot maps made on the GPU from the requests' lengths (knnssd_page_tables)
  rotary   rotary embedding of the new rows' q and k, K and V into their pages (knnssd_rotary_store)
  paged    attention of the new rows of every request over its pages (knnssd_paged_attention)
  packed   causal attention over whole prompts, packed (knnssd_packed_attention)

A case holds plain values.  Head counts and widths are those of the model shapes this repository names: 32 heads (7B),
40 heads (13B), 40 query heads on 8 K/V heads (Qwen 14B), head dimension 128; 4 heads of 64 in fp32 (tiny).  `dtype` is
that of q, the new rows and the outputs, `cache` that of the pages.  Lengths are spread around the numbers a case
gives, by its seed.

While `own` is false, run() computes the operators in elementary torch operations; where it is true, it calls the library.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}


def listed():
    return [
        # the plan of one verification round of 24 requests, k = 4: pure latency, once per round
        {"name": "tables-24x5", "op": "tables", "requests": 24, "context": 1280, "rows": 5, "prompt": 0, "page": 16},
        # a large server's step: 1024 requests, one in sixteen ends and makes room for a prompt
        {"name": "tables-1024-mixed", "op": "tables", "requests": 1024, "context": 4096, "rows": 5, "prompt": 700, "page": 16},
        # the new rows of that round, 13B widths, fp32 activations and a bf16 cache as the decode passes keep them
        {"name": "rotary-13b-120", "op": "rotary", "rows": 120, "heads": 40, "kv_heads": 40, "hd": 128, "page": 16, "dtype": "fp32", "cache": "bf16"},
        # the rows of a few prompts at once, grouped heads, all bf16
        {"name": "rotary-qwen14b-8192", "op": "rotary", "rows": 8192, "heads": 40, "kv_heads": 8, "hd": 128, "page": 16, "dtype": "bf16", "cache": "bf16"},
        # one draft token of one request of the small fp32 model: the smallest call
        {"name": "paged-tiny-fp32-1x1", "op": "paged", "requests": 1, "context": 96, "rows": 1, "long": 0, "heads": 4, "kv_heads": 4, "hd": 64, "page": 16,
         "dtype": "fp32", "cache": "fp32"},
        # verification of k = 4 drafts of eight requests in mid-generation, 13B, fp32 activations
        {"name": "paged-13b-fp32-8x5", "op": "paged", "requests": 8, "context": 1280, "rows": 5, "long": 0, "heads": 40, "kv_heads": 40, "hd": 128, "page": 16,
         "dtype": "fp32", "cache": "bf16"},
        # plain decoding of 64 requests, grouped heads: single tokens
        {"name": "paged-qwen14b-64x1", "op": "paged", "requests": 64, "context": 2304, "rows": 1, "long": 0, "heads": 40, "kv_heads": 8, "hd": 128, "page": 16,
         "dtype": "bf16", "cache": "bf16"},
        # two requests with very long contexts: few rows, the work is along the positions
        {"name": "paged-qwen14b-2x5-long", "op": "paged", "requests": 2, "context": 120000, "rows": 5, "long": 0, "heads": 40, "kv_heads": 8, "hd": 128, "page": 64,
         "dtype": "bf16", "cache": "bf16"},
        # a step that carries chunks of three prompts among thirteen requests' verification rows
        {"name": "paged-7b-chunks", "op": "paged", "requests": 16, "context": 3000, "rows": 5, "long": 512, "heads": 32, "kv_heads": 32, "hd": 128, "page": 16,
         "dtype": "bf16", "cache": "bf16"},
        # short questions packed: 24 prompts of about 100 tokens
        {"name": "packed-7b-24-short", "op": "packed", "prompts": 24, "total": 2309, "longest": 0.08, "heads": 32, "kv_heads": 32, "hd": 128, "dtype": "bf16"},
        # prompts of the small fp32 model
        {"name": "packed-tiny-fp32", "op": "packed", "prompts": 9, "total": 3001, "longest": 0.3, "heads": 4, "kv_heads": 4, "hd": 64, "dtype": "fp32"},
        # long prompts, grouped heads: the largest call, bound by products
        {"name": "packed-qwen14b-12000", "op": "packed", "prompts": 4, "total": 12000, "longest": 0.68, "heads": 40, "kv_heads": 8, "hd": 128, "dtype": "bf16"},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["tables", "rotary", "paged", "paged", "paged", "packed", "packed"])
    page = rng.choice([16, 16, 32, 64, 128])
    heads, kv_heads, hd = rng.choice([(32, 32, 128), (40, 40, 128), (40, 8, 128), (32, 4, 128), (8, 1, 64), (6, 2, 128), (8, 2, 64), (4, 4, 64)])
    dtype, cache = rng.choice([("bf16", "bf16"), ("bf16", "bf16"), ("fp32", "bf16"), ("fp32", "fp32")])
    if op == "tables":
        return {"op": op, "requests": _log_int(rng, 1, 1024), "context": _log_int(rng, 1, 4096), "rows": rng.randint(1, 16), "prompt": rng.choice([0, _log_int(rng, 8, 700)]),
                "page": page}
    if op == "rotary":
        return {"op": op, "rows": _log_int(rng, 1, 8192), "heads": heads, "kv_heads": kv_heads, "hd": hd, "page": page, "dtype": dtype, "cache": cache}
    case = {"op": op, "heads": heads, "kv_heads": kv_heads, "hd": hd, "dtype": dtype}
    if op == "paged":
        rows = rng.choice([1, 1, rng.randint(2, 9), rng.randint(2, 16)])
        long = rng.choice([0, 0, _log_int(rng, 20, 700)])
        most = 100000 if kv_heads < heads and not long else 6000         # positions of all requests: what the listed ones hold
        context = _log_int(rng, 1, most)
        requests = min(_log_int(rng, 1, 64), max(1, 2 * most // (context + max(rows, long))))
        return {**case, "requests": requests, "context": context, "rows": rows, "long": long, "page": page, "cache": cache}
    total = _log_int(rng, 1, 9000 if dtype == "bf16" else 4000)
    return {**case, "prompts": min(total, _log_int(rng, 1, 40)), "total": total, "longest": round(rng.uniform(0.1, 0.95), 2)}


# ---- lengths and inputs -------------------------------------------------------------------------------------------
def _cdiv(a, b):
    return -(-a // b)


def _spread(rng, n, middle):
    """n lengths from half to one and a half times `middle`."""
    return np.maximum(1, np.round(middle * rng.uniform(0.5, 1.5, n))).astype(np.int64) if middle else np.zeros(n, np.int64)


def _paged_lens(case, seed):
    """(lengths held, new rows) of the requests: every fifth request gets a chunk of `long` rows where the case has one."""
    rng = np.random.default_rng(seed)
    n = case["requests"]
    lens = _spread(rng, n, case["context"])
    fresh = np.full(n, case["rows"], np.int64)
    if case["long"]:                                                  # the same numbers of rows whatever the seed
        fresh[2::5] = np.maximum(1, np.round(case["long"] * np.random.default_rng(n).uniform(0.8, 1.0, len(fresh[2::5]))))
        if n < 3:
            fresh[0] = case["long"]
    return lens, fresh


def _packed_lens(case, seed):
    """One prompt with the share `longest` of the tokens, the others ragged; the last of four or more has one token."""
    rng = np.random.default_rng(seed)
    n, total = case["prompts"], case["total"]
    first = max(1, min(total - (n - 1), int(round(case["longest"] * total)))) if n > 1 else total
    left, rest = total - first, n - 1
    lens = [first]
    if rest:
        part = rng.uniform(0.3, 1.0, rest)
        if n >= 4:
            part[-1] = 1e-9
        more = np.maximum(1, np.floor(part / part.sum() * left)).astype(np.int64)
        more[0] += left - more.sum()
        while more[0] < 1:                                            # more prompts than tokens are left for
            more[0] += 1
            more[int(more[1:].argmax()) + 1] -= 1
        lens += more.tolist()
    return np.array(lens, np.int64)


def _table_steps(case, seed):
    """Two steps of a server that follow one another in turn, as (lens, fresh).  In the first some requests end (fresh = -1); in the second
    their places are taken by new prompts while the others are a few accepted tokens further."""
    rng = np.random.default_rng(seed)
    n = case["requests"]
    lens = _spread(rng, n, case["context"])
    one, two = np.full(n, case["rows"], np.int64), np.full(n, case["rows"], np.int64)
    further = lens + rng.integers(1, case["rows"] + 1, n)
    if case["prompt"]:
        ends = np.arange(n) % 16 == 7
        one[ends] = -1
        further[ends] = 0
        two[ends] = _spread(rng, int(ends.sum()), case["prompt"])
    return [(lens, one), (further, two)]


def _table_sizes(case):
    """Pages of the pool, columns of the table and rows the maps have room for: enough for every draw of the lengths."""
    n, prompts = case["requests"], (case["requests"] + 8) // 16 if case["prompt"] else 0
    width = _cdiv(max(int(1.5 * case["context"]) + 2 * case["rows"], 2 * case["prompt"]), case["page"]) + 3
    return n * width, width, n * case["rows"] + prompts * 2 * case["prompt"] + 7


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _normal(g, shape, dtype, spread=1.0):
    return (spread * torch.randn(shape, generator=g, device="cuda")).to(TYPES[dtype])


def _pool(case, lens, seed):
    """Block tables of requests that hold `lens` positions, their pages anywhere in the pool, unused entries -1."""
    page = case["page"]
    held = _cdiv(lens, page)
    n_pages, width = int(held.sum()) + 3, int(held.max()) + 2
    ids = np.random.default_rng(seed + 1).permutation(n_pages)
    table = np.full((len(lens), width), -1, np.int64)
    table[np.arange(width)[None] < held[:, None]] = ids[:held.sum()]
    return n_pages, held, table, ids


def _i32(a):
    return torch.as_tensor(np.ascontiguousarray(a), dtype=torch.int32, device="cuda")


def _angles(n, hd):
    """(cos, sin) of n positions, as the decode passes use them: formed in 64 bits, kept in 32."""
    a = torch.arange(n, device="cuda", dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(hd // 2, device="cuda", dtype=torch.float64) / (hd // 2))
    return torch.stack([a.cos(), a.sin()], dim=-1).float().contiguous()


def prepare(case, seed):
    g, op = _gen(seed), case["op"]
    st = {"case": case}
    if op == "tables":
        steps = _table_steps(case, seed)
        page = case["page"]
        n_pages, width, rows = _table_sizes(case)
        held = _cdiv(steps[0][0], page)
        ids = np.random.default_rng(seed + 1).permutation(n_pages)
        table = np.full((len(held), width), -1, np.int64)
        table[np.arange(width)[None] < held[:, None]] = ids[:held.sum()]
        free = np.zeros(n_pages, np.int64)
        left = ids[held.sum():]
        free[:len(left)] = left
        n = len(held)
        st.update(steps=[(_i32(a), _i32(b)) for a, b in steps], turn=0, owned=_i32(held), table=_i32(table), free=_i32(free), count=_i32([len(left)]),
                  start=_i32(np.zeros(n + 1)), request=_i32(np.zeros(rows)), pos=_i32(np.zeros(rows)), slot=_i32(np.zeros(rows)), info=_i32(np.zeros(4)))
        return st
    H, KV, hd = case["heads"], case["kv_heads"], case["hd"]
    if op == "rotary":
        R, page = case["rows"], case["page"]
        rng = np.random.default_rng(seed)
        n_pages = _cdiv(R, page) + 9
        pos = rng.integers(0, 4096, R)
        slot = rng.permutation(n_pages * page)[:R]
        st.update(qkv=_normal(g, (R, (H + 2 * KV) * hd), case["dtype"]), angles=_angles(4096, hd), pos=_i32(pos), slot=_i32(slot),
                  k=torch.zeros((n_pages, KV, page, hd), dtype=TYPES[case["cache"]], device="cuda"), v=torch.zeros((n_pages, KV, page, hd), dtype=TYPES[case["cache"]], device="cuda"))
        return st
    if op == "paged":
        lens, fresh = _paged_lens(case, seed)
        n_pages, _, table, _ = _pool(case, lens + fresh, seed)
        start = np.concatenate([[0], np.cumsum(fresh)])
        R = int(start[-1])
        st.update(q=_normal(g, (R, H, hd), case["dtype"], 1.5), k=_normal(g, (n_pages, KV, case["page"], hd), case["cache"]),
                  v=_normal(g, (n_pages, KV, case["page"], hd), case["cache"]), table=_i32(table), lens=_i32(lens), start=_i32(start),
                  most=int(fresh.max()), width=_cdiv(int((lens + fresh).max()), case["page"]))
        return st
    lens = _packed_lens(case, seed)
    qkv = _normal(g, (case["total"], (H + 2 * KV) * hd), case["dtype"], 1.2)       # one map's output: q, k and v are views of it
    st.update(q=qkv[:, :H * hd].unflatten(1, (H, hd)), k=qkv[:, H * hd:(H + KV) * hd].unflatten(1, (KV, hd)), v=qkv[:, (H + KV) * hd:].unflatten(1, (KV, hd)),
              start=_i32(np.concatenate([[0], np.cumsum(lens)])))
    return st


# ---- the operators ------------------------------------------------------------------------------------------------
def run(st):
    op = st["case"]["op"]
    if op == "tables":
        st["turn"] ^= 1
        lens, fresh = st["steps"][1 - st["turn"]]
        (_tables_own if own else _tables_plain)(st, lens, fresh)
        return {k: st[k] for k in ("owned", "table", "free", "count", "start", "request", "pos", "slot", "info")}
    if op == "rotary":
        q = (_rotary_own if own else _rotary_plain)(st)
        return {"q": q, "k": st["k"], "v": st["v"]}
    if op == "paged":
        return (_paged_own if own else _paged_plain)(st)
    return (_packed_own if own else _packed_plain)(st)


def _tables_own(st, lens, fresh):
    from paper_2505_16162_b200 import binding as kb
    kb.knnssd_page_tables(lens, fresh, st["owned"], st["table"], st["free"], st["count"], st["case"]["page"], st["start"], st["request"], st["pos"], st["slot"], st["info"])


def _rotary_own(st):
    from paper_2505_16162_b200 import binding as kb
    return kb.knnssd_rotary_store(st["qkv"], st["angles"], st["pos"], st["slot"], st["k"], st["v"])


def _paged_own(st):
    from paper_2505_16162_b200 import binding as kb
    return kb.knnssd_paged_attention(st["q"], st["k"], st["v"], st["table"], st["lens"], st["start"], max_fresh=st["most"])


def _packed_own(st):
    from paper_2505_16162_b200 import binding as kb
    return kb.knnssd_packed_attention(st["q"], st["k"], st["v"], st["start"])


def _tables_plain(st, lens, fresh):
    """A request holds exactly the pages of its len + fresh positions (none where fresh is -1).  Surplus pages go onto the free stack in request
    and page order, then pages come from its top in the same order."""
    page, owned, table, free, count = st["case"]["page"], st["owned"], st["table"], st["free"], st["count"]
    n = fresh.clamp(min=0)
    need = torch.where(fresh < 0, 0, (lens + n + page - 1) // page)
    give, take = (owned - need).clamp(min=0), (need - owned).clamp(min=0)
    given, taken = give.cumsum(0, dtype=torch.int32), take.cumsum(0, dtype=torch.int32)
    col = torch.arange(table.shape[1], device="cuda", dtype=torch.int32)
    back = (col >= need[:, None]) & (col < owned[:, None])
    spare = torch.cat([free, free[:1]])                                # the last entry takes what has no place
    at = torch.where(back, count + (given - give - need)[:, None] + col, free.shape[0])
    spare.scatter_(0, at.flatten().long(), table.flatten())
    free.copy_(spare[:-1])
    top = count + given[-1:]
    new = (col >= owned[:, None]) & (col < need[:, None])
    at = (top - 1 - (taken - take - owned)[:, None] - col).clamp(0, free.shape[0] - 1)
    table.copy_(torch.where(new, free[at.long()], torch.where(back, -1, table)))
    owned.copy_(need)
    count.copy_(top - taken[-1:])
    end = n.cumsum(0, dtype=torch.int32)
    st["start"][1:] = end
    r = torch.arange(st["pos"].shape[0], device="cuda", dtype=torch.int32)
    b = torch.searchsorted(end, r, right=True).clamp(max=n.shape[0] - 1)
    live = r < end[-1]
    pos = lens[b] + r - (end - n)[b]
    st["request"].copy_(torch.where(live, b, -1))
    st["pos"].copy_(torch.where(live, pos, -1))
    st["slot"].copy_(torch.where(live, table[b, (pos // page).clamp(0, table.shape[1] - 1).long()] * page + pos % page, -1))
    st["info"].copy_(torch.stack([end[-1], taken[-1], given[-1], torch.zeros_like(end[-1])]))


def _rotary_plain(st):
    """Dimension i of a head and dimension i + hd / 2 are turned by the angle of position and i."""
    k, v = st["k"], st["v"]
    _, KV, page, hd = k.shape
    H = st["qkv"].shape[1] // hd - 2 * KV
    x = st["qkv"].float().unflatten(1, (H + 2 * KV, hd))
    cs = st["angles"][st["pos"].long()][:, None]
    a, b = x[:, :H + KV, :hd // 2], x[:, :H + KV, hd // 2:]
    turned = torch.cat([a * cs[..., 0] - b * cs[..., 1], b * cs[..., 0] + a * cs[..., 1]], dim=-1)
    slot = st["slot"].long()
    k[slot // page, :, slot % page] = turned[:, H:].to(k.dtype)
    v[slot // page, :, slot % page] = x[:, H + KV:].to(v.dtype)
    return turned[:, :H].to(st["qkv"].dtype)


def _softmax(s, hide):
    """In place over the last axis, nothing where `hide`."""
    s.masked_fill_(hide, -math.inf)
    s.sub_(s.amax(dim=-1, keepdim=True)).exp_()
    return s.div_(s.sum(dim=-1, keepdim=True))


def _paged_plain(st):
    q, start, lens = st["q"], st["start"].long(), st["lens"].long()
    R, H, hd = q.shape
    _, KV, page, _ = st["k"].shape
    B, most, G = lens.shape[0], st["most"], H // KV
    pages = st["table"][:, :st["width"]].long().clamp(min=0)
    k, v = (t[pages].float().transpose(1, 2).flatten(2, 3) for t in (st["k"], st["v"]))          # [request][kv head][position][dim]
    row = torch.arange(R, device="cuda")
    b = torch.searchsorted(start[1:], row, right=True)
    i = row - start[b]
    x = torch.zeros(B, most, H, hd, device="cuda")
    x[b, i] = q.float()
    x = x.unflatten(2, (KV, G)).permute(0, 2, 3, 1, 4).reshape(B, KV, G * most, hd)
    s = (x / math.sqrt(hd)) @ k.transpose(-1, -2)
    last = (lens[:, None] + torch.arange(most, device="cuda")).repeat(1, G)[:, None, :, None]   # the position a row is at
    o = _softmax(s, torch.arange(k.shape[2], device="cuda") > last) @ v
    return o.unflatten(2, (G, most)).permute(0, 3, 1, 2, 4).flatten(2, 3)[b, i].to(q.dtype)


def _packed_plain(st):
    q, start = st["q"], st["start"].long()
    R, H, hd = q.shape
    KV = st["k"].shape[1]
    row = torch.arange(R, device="cuda")
    b = torch.searchsorted(start[1:], row, right=True)
    hide = (b[:, None] != b[None]) | (row[None] > row[:, None])
    x = (q.float() / math.sqrt(hd)).unflatten(1, (KV, H // KV)).permute(1, 2, 0, 3)              # [kv head][group][row][dim]
    k, v = (t.float().transpose(0, 1)[:, None] for t in (st["k"], st["v"]))
    o = _softmax(x @ k.transpose(-1, -2), hide) @ v
    return o.permute(2, 0, 1, 3).flatten(1, 2).to(q.dtype)


# ---- what a pass cannot do without ---------------------------------------------------------------------------------
def work(case):
    op = case["op"]
    if op == "tables":
        (lens, fresh), _ = _table_steps(case, 0)
        n, rows, page = len(lens), int(np.maximum(fresh, 0).sum()), case["page"]
        new = int(np.maximum(_cdiv(lens + np.maximum(fresh, 0), page) - _cdiv(lens, page), 0).sum())
        return {"bytes": 4 * (5 * n + 2 * new + 3 * rows), "flops": 4 * (n + rows)}
    H, KV, hd = case["heads"], case["kv_heads"], case["hd"]
    b = 4 if case["dtype"] == "fp32" else 2
    if op == "rotary":
        R, c = case["rows"], 4 if case["cache"] == "fp32" else 2
        return {"bytes": R * hd * (b * (2 * H + 2 * KV) + 2 * KV * c + 4) + 8 * R, "flops": 3 * R * (H + KV) * hd}
    if op == "paged":
        lens, fresh = _paged_lens(case, 0)
        c = 4 if case["cache"] == "fp32" else 2
        seen = int((fresh * lens + fresh * (fresh + 1) // 2).sum())
        return {"bytes": int((lens + fresh).sum()) * 2 * KV * hd * c + int(fresh.sum()) * 2 * H * hd * b, "flops": 4 * H * hd * seen}
    lens = _packed_lens(case, 0)
    return {"bytes": case["total"] * hd * b * (2 * H + 2 * KV), "flops": 4 * H * hd * int((lens * (lens + 1) // 2).sum())}


# ---- the same in 64 bits -------------------------------------------------------------------------------------------
def _attend64(q, k, v, first):
    """Rows [n][H][hd] at positions first .. over keys [m][KV][hd]: row i looks at positions up to first + i."""
    n, H, hd = q.shape
    m, KV, _ = k.shape
    out = torch.empty(n, H, hd, dtype=torch.float64, device="cuda")
    unseen = torch.ones(n, m, dtype=torch.bool, device="cuda").triu(first + 1)
    for h in range(H):
        kv = h * KV // H
        w = torch.softmax((q[:, h].double() @ k[:, kv].double().T * hd ** -0.5).masked_fill(unseen, -math.inf), dim=1)
        out[:, h] = w @ v[:, kv].double()
    return out


def exact(case, seed):
    op = case["op"]
    if op == "tables":
        return None
    st = prepare(case, seed)
    if op == "rotary":
        KV, hd = case["kv_heads"], case["hd"]
        rows = st["qkv"].double().view(case["rows"], -1, hd)
        z = torch.view_as_complex(torch.stack(rows.chunk(2, dim=-1), dim=-1).contiguous())
        turn = torch.view_as_complex(st["angles"].double().contiguous())[st["pos"].long()]
        z[:, :-KV] *= turn[:, None]
        rows = torch.cat([z.real, z.imag], dim=-1)
        pages = [t.double().transpose(1, 2).reshape(-1, KV, hd) for t in (st["k"], st["v"])]          # [slot][kv head][dim]
        pages[0][st["slot"].long()] = rows[:, -2 * KV:-KV]
        pages[1][st["slot"].long()] = rows[:, -KV:]
        k, v = (t.view(-1, case["page"], KV, hd).transpose(1, 2) for t in pages)
        return {"q": rows[:, :-2 * KV], "k": k.contiguous(), "v": v.contiguous()}
    out = []
    if op == "paged":
        lens, fresh = _paged_lens(case, seed)
        start, page = st["start"].tolist(), case["page"]
        for i, (a, n) in enumerate(zip(lens.tolist(), fresh.tolist())):
            ids = st["table"][i, :_cdiv(a + n, page)].long()
            k, v = (t[ids].transpose(1, 2).flatten(0, 1)[:a + n] for t in (st["k"], st["v"]))
            out.append(_attend64(st["q"][start[i]:start[i + 1]], k, v, a))
    else:
        at = 0
        for n in _packed_lens(case, seed).tolist():
            out.append(_attend64(st["q"][at:at + n], st["k"][at:at + n], st["v"][at:at + n], 0))
            at += n
    return torch.cat(out)
