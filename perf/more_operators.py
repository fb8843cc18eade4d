"""Drafts that branch, for several requests on one paged K/V cache, as cases that can be timed and compared.

A request's new rows are a tree of tokens: row 0 is the pending token, row i > 0 a drafted token that follows the row parent[i] < i.  One verification
round takes four operators besides the maps, the rotary store and the page tables that the library has for chains:

  tables   positions of the rows and which of the rows before it each one sees (knnssd_tree_tables)
  attend   attention of the rows over the pages: the committed positions and the row's own ancestors (knnssd_tree_attention)
  accept   which drafts the full model's distributions keep, and the token after them (knnssd_tree_accept)
  keep     K and V of the rows on the kept path moved together in the pages of all layers (knnssd_keep_rows)

A case holds plain values.  Head counts, widths, layers and vocabularies are those of the model shapes this repository names: 32 heads and 32 layers
(7B), 40 heads and 40 layers (13B), 40 query heads on 8 K/V heads, 48 layers and 152064 tokens (Qwen 14B), head dimension 128, 32000 tokens; 4 heads of 64
in fp32 (tiny).  `rows` is the most rows of a request, `width` how far back a row's parent may lie (1: a chain).  Lengths held are spread around
`context` by the seed; the numbers of rows follow from the case alone.

While `own` is false, run() computes the operators in elementary torch operations; where it is true, it calls the library.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
LAYERS = {"tiny": (4, 4, 64, 4), "7b": (32, 32, 128, 32), "13b": (40, 40, 128, 40), "qwen14b": (40, 8, 128, 48)}     # heads, K/V heads, head dimension, layers


def listed():
    return [
        # the trees of one round of 24 requests: pure latency, once per round
        {"name": "tables-24x25", "op": "tables", "requests": 24, "context": 1280, "rows": 25, "width": 6, "prompt": 0},
        # a large server's step: 1024 requests, one in sixteen brings a chunk of its prompt instead (a chain)
        {"name": "tables-1024-mixed", "op": "tables", "requests": 1024, "context": 4096, "rows": 33, "width": 8, "prompt": 700},
        # two trees of the small fp32 model: the smallest attention
        {"name": "attend-tiny-fp32-2x13", "op": "attend", "requests": 2, "context": 96, "rows": 13, "width": 4, "heads": 4, "kv_heads": 4, "hd": 64, "page": 16,
         "dtype": "fp32", "cache": "fp32"},
        # eight requests in mid-generation, 13B widths, fp32 activations and a bf16 cache as the decode passes keep them
        {"name": "attend-13b-fp32-8x25", "op": "attend", "requests": 8, "context": 1280, "rows": 25, "width": 5, "heads": 40, "kv_heads": 40, "hd": 128, "page": 16,
         "dtype": "fp32", "cache": "bf16"},
        # a full server, grouped heads, small trees
        {"name": "attend-qwen14b-64x16", "op": "attend", "requests": 64, "context": 2304, "rows": 16, "width": 4, "heads": 40, "kv_heads": 8, "hd": 128, "page": 16,
         "dtype": "bf16", "cache": "bf16"},
        # two requests with very long contexts: the work is along the positions
        {"name": "attend-qwen14b-2x48-long", "op": "attend", "requests": 2, "context": 120000, "rows": 48, "width": 12, "heads": 40, "kv_heads": 8, "hd": 128, "page": 64,
         "dtype": "bf16", "cache": "bf16"},
        # as large trees as there are, a K/V head for every query head: the largest call
        {"name": "attend-7b-24x64", "op": "attend", "requests": 24, "context": 3000, "rows": 64, "width": 16, "heads": 32, "kv_heads": 32, "hd": 128, "page": 16,
         "dtype": "bf16", "cache": "bf16"},
        # one request, a chain of five drafts drawn from the draft model: what a single user's round waits for
        {"name": "accept-1x6-v32000", "op": "accept", "requests": 1, "rows": 6, "width": 1, "vocab": 32000, "drawn": True},
        # the trees of 24 requests, drafts drawn
        {"name": "accept-24x25-v32000", "op": "accept", "requests": 24, "rows": 25, "width": 5, "vocab": 32000, "drawn": True},
        # drafts chosen by rank instead, on the largest vocabulary
        {"name": "accept-32x26-v152064-ranked", "op": "accept", "requests": 32, "rows": 26, "width": 6, "vocab": 152064, "drawn": False},
        # all 48 layers of a few requests, grouped heads
        {"name": "keep-qwen14b-4x16", "op": "keep", "requests": 4, "context": 300, "rows": 16, "width": 3, "model": "qwen14b", "page": 16, "cache": "bf16"},
        # 32 layers of 32 heads for 24 requests
        {"name": "keep-7b-24x40", "op": "keep", "requests": 24, "context": 130, "rows": 40, "width": 4, "model": "7b", "page": 32, "cache": "bf16"},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["tables", "attend", "attend", "attend", "accept", "accept", "keep"])
    page = rng.choice([16, 16, 32, 64, 128])
    rows = rng.choice([rng.randint(2, 12), rng.randint(2, 64)])
    width = rng.choice([1, rng.randint(2, 6), rng.randint(2, 20)])
    if op == "tables":
        return {"op": op, "requests": _log_int(rng, 1, 1024), "context": _log_int(rng, 1, 4096), "rows": min(rows, 33), "width": width, "prompt": rng.choice([0, _log_int(rng, 8, 700)])}
    if op == "attend":
        heads, kv_heads, hd = rng.choice([(32, 32, 128), (40, 40, 128), (40, 8, 128), (32, 4, 128), (8, 1, 64), (6, 2, 128), (8, 2, 64), (4, 4, 64)])
        dtype, cache = rng.choice([("bf16", "bf16"), ("bf16", "bf16"), ("fp32", "bf16"), ("fp32", "fp32")])
        most = 100000 if kv_heads < heads and dtype == "bf16" else 8000       # positions of all requests
        context = _log_int(rng, 1, most)
        return {"op": op, "requests": min(_log_int(rng, 1, 48), max(1, 2 * most // (context + rows))), "context": context, "rows": rows, "width": width, "heads": heads,
                "kv_heads": kv_heads, "hd": hd, "page": page, "dtype": dtype, "cache": cache}
    if op == "accept":
        vocab = _log_int(rng, 1000, 152064)
        most = 32 * 26 * 152064 // (vocab * rows) // 2
        return {"op": op, "requests": min(_log_int(rng, 1, 64), max(1, most)), "rows": rows, "width": width, "vocab": vocab, "drawn": rng.random() < 0.6}
    return {"op": op, "requests": _log_int(rng, 1, 20), "context": _log_int(rng, 1, 130), "rows": min(rows, 40), "width": width, "model": rng.choice(["7b", "qwen14b", "tiny"]),
            "page": page, "cache": rng.choice(["bf16", "bf16", "fp32"])}


# ---- lengths, trees and inputs ------------------------------------------------------------------------------------
def _cdiv(a, b):
    return -(-a // b)


def _fresh(case):
    """New rows of the requests: two thirds of `rows` up to all of them, every seventh request the pending token alone, chunks of prompts where the
    case has them.  The same whatever the seed."""
    n = case["requests"]
    rng = np.random.default_rng(n)
    fresh = np.maximum(1, np.round(case["rows"] * rng.uniform(2 / 3, 1.0, n))).astype(np.int64)
    fresh[0] = case["rows"]
    fresh[6::7] = 1
    if case.get("prompt"):
        fresh[7::16] = np.maximum(1, np.round(case["prompt"] * rng.uniform(0.5, 1.0, len(fresh[7::16]))))
    return fresh


def _lens(case, seed):
    rng = np.random.default_rng(seed)
    return np.maximum(1, np.round(case["context"] * rng.uniform(0.5, 1.5, case["requests"]))).astype(np.int64)


def _parents(case, seed):
    """[request] of parents of its rows: each among the `width` rows before it; those of a chunk of a prompt form a chain."""
    rng = np.random.default_rng(seed + 2)
    out = []
    for n in _fresh(case).tolist():
        i = np.arange(n)
        back = np.ones(n, np.int64) if n > 64 else rng.integers(1, case["width"] + 1, n)
        out.append(np.maximum(i - back, np.minimum(i - 1, 0)))
    return out


def _start(fresh):
    return np.concatenate([[0], np.cumsum(fresh)])


def _ancestors(parent):
    """[row][row]: whether the first one sees the second, that is itself and what it follows."""
    sees = np.zeros((len(parent), len(parent)), bool)
    for i, p in enumerate(parent.tolist()):
        if p >= 0:
            sees[i] = sees[p]
        sees[i, i] = True
    return sees


def _seen_words(parent):
    """64 bits a row: bit d says whether it sees the position d before its own; all that lies before the tree is seen."""
    n = len(parent)
    sees = np.concatenate([np.ones((n, 64), bool), _ancestors(parent)], axis=1)
    at = np.arange(n)[:, None] + 64 - np.arange(64)
    bits = np.take_along_axis(sees, at, axis=1).astype(np.uint64)
    return (bits << np.arange(64, dtype=np.uint64)).sum(axis=1, dtype=np.uint64).view(np.int64)


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _normal(g, shape, dtype, spread=1.0):
    return (spread * torch.randn(shape, generator=g, device="cuda")).to(TYPES[dtype])


def _pool(case, lens, seed):
    """Block tables of requests that hold `lens` positions, their pages anywhere in the pool, unused entries -1.  The pool has room for any lengths that
    the seed may give."""
    held = _cdiv(lens, case["page"])
    width = _cdiv(int(1.5 * case["context"]) + 1 + case["rows"], case["page"])
    n_pages = len(lens) * width + 3
    ids = np.random.default_rng(seed + 1).permutation(n_pages)
    table = np.full((len(lens), width), -1, np.int64)
    table[np.arange(width)[None] < held[:, None]] = ids[:held.sum()]
    return n_pages, table


def _i32(a):
    return torch.as_tensor(np.ascontiguousarray(a), dtype=torch.int32, device="cuda")


def _distributions(z, off):
    """Softmax of the values, nothing below a ten-thousandth of the largest; rows sum to 1."""
    p = torch.softmax(z + off, dim=-1)
    p.masked_fill_(p < 1e-4 * p.amax(dim=-1, keepdim=True), 0.0)
    return p.div_(p.sum(dim=-1, keepdim=True))


def _walk(parent, rng):
    """A path from row 0 down: rows of a kept path."""
    path = [0]
    while rng.random() < 0.75:
        below = np.flatnonzero(parent == path[-1])
        below = below[below > path[-1]]
        if len(below) == 0:
            break
        path.append(int(rng.choice(below)))
    return path


def prepare(case, seed):
    g, op = _gen(seed), case["op"]
    fresh, parents = _fresh(case), _parents(case, seed)
    start = _start(fresh)
    st = {"case": case, "start": _i32(start), "parent": _i32(np.concatenate(parents)), "most": int(fresh.max())}
    R = int(start[-1])
    if op == "tables":
        st.update(lens=_i32(_lens(case, seed)), pos=_i32(np.zeros(R)), seen=torch.zeros(R, dtype=torch.int64, device="cuda"), state=_i32(np.zeros(len(fresh))))
        return st
    if op == "accept":
        # the drafts: each drawn from its parent's distribution of the draft model, or the parent's most probable tokens in their order
        V = case["vocab"]
        z = 2.5 * torch.randn(R, V, generator=g, device="cuda")
        q = _distributions(z, 0.0)
        p = _distributions(z, 0.8 * torch.randn(R, V, generator=g, device="cuda"))
        above = torch.as_tensor(np.concatenate([np.maximum(x, 0) + s for x, s in zip(parents, start)]), device="cuda")
        if case["drawn"]:
            token = torch.cat([torch.multinomial(q[above[i:i + 64]], 1, generator=g)[:, 0] for i in range(0, R, 64)])
        else:
            rank = np.concatenate([[(x[:i] == x[i]).sum() for i in range(len(x))] for x in parents])
            best = torch.cat([q[i:i + 64].topk(21, dim=-1).indices for i in range(0, R, 64)])
            token = best[above, torch.as_tensor(rank, device="cuda")]
        n = len(fresh)
        st.update(p=p, q=q if case["drawn"] else None, token=token.int(), u=torch.rand(R, generator=g, device="cuda"), u_final=torch.rand(n, generator=g, device="cuda"),
                  path=_i32(np.zeros(R)), accepted=_i32(np.zeros(n)), next=_i32(np.zeros(n)))
        return st
    lens = _lens(case, seed)
    n_pages, table = _pool(case, lens + fresh, seed)
    st.update(lens=_i32(lens), table=_i32(table), width=_cdiv(int((lens + fresh).max()), case["page"]))
    if op == "attend":
        H, KV, hd = case["heads"], case["kv_heads"], case["hd"]
        st.update(q=_normal(g, (R, H, hd), case["dtype"], 1.5), k=_normal(g, (n_pages, KV, case["page"], hd), case["cache"]),
                  v=_normal(g, (n_pages, KV, case["page"], hd), case["cache"]), seen=torch.as_tensor(np.concatenate([_seen_words(x) for x in parents]), device="cuda"))
        return st
    _, KV, hd, layers = LAYERS[case["model"]]
    rng = np.random.default_rng(seed + 3)
    path = np.full(R, -1, np.int64)
    for s, x in zip(start, parents):
        kept = _walk(x, rng)
        path[s:s + len(kept)] = kept
    k, v = (torch.empty((layers, n_pages, KV, case["page"], hd), dtype=TYPES[case["cache"]], device="cuda") for _ in range(2))
    for pool in (*k, *v):
        pool.normal_(generator=g)
    st.update(path=_i32(path), k=k, v=v)
    if own:
        from paper_2505_16162_b200 import binding as kb
        st["pools"] = kb.PagePools(list(k), list(v))
    return st


# ---- the operators ------------------------------------------------------------------------------------------------
def run(st):
    op = st["case"]["op"]
    if op == "tables":
        (_tables_own if own else _tables_plain)(st)
        return {"pos": st["pos"], "seen": st["seen"], "state": st["state"]}
    if op == "attend":
        return (_attend_own if own else _attend_plain)(st)
    if op == "accept":
        (_accept_own if own else _accept_plain)(st)
        return {"path": st["path"], "accepted": st["accepted"], "next": st["next"]}
    (_keep_own if own else _keep_plain)(st)
    return {"k": st["k"], "v": st["v"]}


def _tables_own(st):
    from paper_2505_16162_b200 import binding as kb
    kb.knnssd_tree_tables(st["lens"], st["start"], st["parent"], st["pos"], st["seen"], st["state"])


def _attend_own(st):
    from paper_2505_16162_b200 import binding as kb
    return kb.knnssd_tree_attention(st["q"], st["k"], st["v"], st["table"], st["lens"], st["start"], st["seen"], max_fresh=st["most"])


def _accept_own(st):
    from paper_2505_16162_b200 import binding as kb
    kb.knnssd_tree_accept(st["p"], st["q"], st["token"], st["parent"], st["start"], st["u"], st["u_final"], st["path"], st["accepted"], st["next"])


def _keep_own(st):
    from paper_2505_16162_b200 import binding as kb
    kb.knnssd_keep_rows(st["pools"], st["table"], st["lens"], st["start"], st["path"])


def _requests_of(st):
    """Request and number within it of every row."""
    row = torch.arange(st["parent"].shape[0], device="cuda")
    b = torch.searchsorted(st["start"][1:].long(), row, right=True)
    return row, b, row - st["start"].long()[b]


def _tables_plain(st):
    """Up from every row at once, a parent at a time: 64 steps at most where the tree is, and a chain's rows see all before them."""
    row, b, i = _requests_of(st)
    start = st["start"].long()[b]
    parent = st["parent"].long()
    n_chain = torch.full((st["lens"].shape[0],), 1 << 30, device="cuda", dtype=torch.int64)         # rows of the chain that a request begins with
    n_chain.scatter_reduce_(0, b, torch.where(parent != i - 1, i, 1 << 30), "amin")
    chain = i < n_chain[b]
    bit = torch.ones((), dtype=torch.int64, device="cuda")
    seen, depth, at = torch.where(i >= 63, 0, torch.bitwise_left_shift(-bit, (i + 1).clamp(max=63))), torch.zeros_like(i), i
    good = torch.ones_like(chain)
    for _ in range(64):
        inside = (at >= 0) & (i - at < 64)
        seen = torch.where(inside, seen | torch.bitwise_left_shift(bit, (i - at).clamp(0, 63)), seen)
        depth = depth + (inside & (at < i))
        up = parent[(start + at.clamp(min=0))]
        good &= ~inside | ((up >= -1) & (up < at))
        at = torch.where(inside, up.clamp(min=-1), at)
    far = i - 63                                                                                    # rows that lie 64 or more before this one: all are its ancestors
    good &= (far <= 0) | ((at == far - 1) & (far <= n_chain[b]))
    depth = torch.where(chain, i, depth + far.clamp(min=0))
    seen = torch.where(chain, -bit, seen)
    bad = torch.zeros_like(st["state"]).scatter_reduce_(0, b, (~(chain | good)).int(), "amax")
    st["state"].copy_(bad)
    wrong = bad[b] != 0
    st["pos"].copy_(torch.where(wrong, -1, st["lens"][b] + depth))
    st["seen"].copy_(torch.where(wrong, 0, seen))


def _attend_plain(st):
    q, lens = st["q"], st["lens"].long()
    R, H, hd = q.shape
    _, KV, page, _ = st["k"].shape
    B, most, G = lens.shape[0], st["most"], H // KV
    pages = st["table"][:, :st["width"]].long().clamp(min=0)
    k, v = (t[pages].float().transpose(1, 2).flatten(2, 3) for t in (st["k"], st["v"]))          # [request][kv head][position][dim]
    _, b, i = _requests_of(st)
    x = torch.zeros(B, most, H, hd, device="cuda")
    x[b, i] = q.float()
    words = torch.zeros(B, most, dtype=torch.int64, device="cuda")
    words[b, i] = st["seen"]
    x = x.unflatten(2, (KV, G)).permute(0, 2, 3, 1, 4).reshape(B, KV, G * most, hd)
    s = (x / math.sqrt(hd)) @ k.transpose(-1, -2)
    before = (lens[:, None] + torch.arange(most, device="cuda"))[:, :, None] - torch.arange(k.shape[2], device="cuda")   # how far a position lies before the row's own
    hide = (before < 0) | ((before < 64) & ((words[:, :, None] >> before.clamp(0, 63)) & 1 == 0))
    s = s.unflatten(2, (G, most)).masked_fill_(hide[:, None, None], -math.inf)
    top = s.amax(dim=-1, keepdim=True)
    s.sub_(torch.where(top == -math.inf, 0.0, top)).exp_()
    total = s.sum(dim=-1, keepdim=True)
    o = (s / torch.where(total == 0, 1.0, total)).flatten(2, 3) @ v
    return o.unflatten(2, (G, most)).permute(0, 3, 1, 2, 4).flatten(2, 3)[b, i].to(q.dtype)


def _accept_plain(st):
    """All requests go through their rows in order together: a row whose parent is the last one kept is tested.  In 64 bits: a test or a draw that
    lies next to a border is to fall on the same side whatever the order of the sums."""
    p, q, token, parent, V = st["p"], st["q"], st["token"].long(), st["parent"].long(), st["case"]["vocab"]
    start, n = st["start"].long()[:-1], st["start"].long().diff()
    R, B = token.shape[0], n.shape[0]
    node = torch.zeros(B, dtype=torch.int64, device="cuda")
    accepted = torch.zeros_like(node)
    path = torch.full((R + 1,), -1, dtype=torch.int32, device="cuda")                              # the last entry takes what has no place
    path[start] = 0
    w, z = p[start].double(), torch.ones(B, 1, dtype=torch.float64, device="cuda")
    for i in range(1, st["most"]):
        r = (start + i).clamp(max=R - 1)
        x = token[r][:, None]
        tested = ((i < n) & (parent[r] == node))[:, None]
        of_draft = 1.0 if q is None else q[start + node].gather(1, x).double()
        kept = tested & (st["u"][r].double()[:, None] * z * of_draft < w.gather(1, x))
        lost = tested & ~kept
        if q is None:
            left = w.scatter(1, x, 0.0)
        else:
            left = (w / torch.where(z > 0, z, 1.0) - q[start + node]).clamp_(min=0.0)
        w = torch.where(lost, left, w)
        z = torch.where(lost, w.sum(dim=1, keepdim=True), z)
        node = torch.where(kept[:, 0], i, node)
        accepted = accepted + kept[:, 0]
        path[torch.where(kept[:, 0], start + accepted, R)] = i
        w = torch.where(kept, p[start + node], w)
        z = torch.where(kept, 1.0, z)
    w = torch.where(w.sum(dim=1, keepdim=True) > 0, w, p[start + node])
    upto = w.cumsum(dim=1)
    st["next"].copy_(torch.searchsorted(upto, st["u_final"].double()[:, None] * upto[:, -1:], right=True)[:, 0].clamp(max=V - 1))
    st["accepted"].copy_(accepted)
    st["path"].copy_(path[:-1])


def _keep_plain(st):
    """What is not on a path is moved from the first row's place to itself."""
    page, lens = st["case"]["page"], st["lens"].long()
    _, b, j = _requests_of(st)
    on = st["path"] >= 0
    src, dst = (lens[b] + torch.where(on, a, 0) for a in (st["path"].long(), j))
    sp, dp = (st["table"].long()[b, a // page] for a in (src, dst))
    for pool in (*st["k"], *st["v"]):
        pool[dp, :, dst % page] = pool[sp, :, src % page]


# ---- what a pass cannot do without ---------------------------------------------------------------------------------
def work(case):
    op, fresh = case["op"], _fresh(case)
    n, rows = len(fresh), int(fresh.sum())
    if op == "tables":
        return {"bytes": 16 * rows + 12 * n, "flops": rows}
    if op == "accept":                                                # where a request's round ends it needs a row of p whole, and of q
        return {"bytes": 4 * n * case["vocab"] * (2 if case["drawn"] else 1) + 16 * rows, "flops": 2 * n * case["vocab"]}
    if op == "attend":
        H, KV, hd = case["heads"], case["kv_heads"], case["hd"]
        b, c = (4 if case[t] == "fp32" else 2 for t in ("dtype", "cache"))
        lens = _lens(case, 0)
        seen = sum(int(m) * len(x) + int(_ancestors(x).sum()) for m, x in zip(lens, _parents(case, 0)))
        return {"bytes": int((lens + fresh).sum()) * 2 * KV * hd * c + rows * (2 * H * hd * b + 8), "flops": 4 * H * hd * seen}
    _, KV, hd, layers = LAYERS[case["model"]]
    rng = np.random.default_rng(3)
    moved = sum(sum(j != r for j, r in enumerate(_walk(x, rng))) for x in _parents(case, 0))
    return {"bytes": 2 * 2 * layers * KV * hd * (4 if case["cache"] == "fp32" else 2) * moved + 4 * rows, "flops": 0}


# ---- the same in 64 bits -------------------------------------------------------------------------------------------
def exact(case, seed):
    op = case["op"]
    if op == "tables" or (op == "accept" and case["requests"] * case["rows"] > 1000):
        return None
    st = prepare(case, seed)
    parents, start = _parents(case, seed), _start(_fresh(case)).tolist()
    if op == "accept":
        return _exact_accept(st, parents, start)
    lens, table, page = st["lens"].tolist(), st["table"].long(), case["page"]
    if op == "keep":
        for b, m in enumerate(lens):
            path = [r for r in st["path"].tolist()[start[b]:start[b + 1]] if r >= 0]
            src, dst = (torch.tensor([m + x for x in a], device="cuda") for a in (path, range(len(path))))
            for pool in (*st["k"], *st["v"]):
                pool[table[b, dst // page], :, dst % page] = pool[table[b, src // page], :, src % page].clone()
        return {"k": st["k"], "v": st["v"]}
    out = torch.empty(st["q"].shape, dtype=torch.float64, device="cuda")
    H, KV, hd = case["heads"], case["kv_heads"], case["hd"]
    for b, m in enumerate(lens):
        n = len(parents[b])
        ids = table[b, :_cdiv(m + n, page)]
        k, v = (t[ids].transpose(1, 2).flatten(0, 1)[:m + n] for t in (st["k"], st["v"]))
        sees = torch.cat([torch.ones(n, m, dtype=torch.bool), torch.as_tensor(_ancestors(parents[b]))], dim=1).cuda()
        for h in range(H):
            kv = h * KV // H
            s = st["q"][start[b]:start[b + 1], h].double() @ k[:, kv].double().T * hd ** -0.5
            out[start[b]:start[b + 1], h] = torch.softmax(s.masked_fill(~sees, -math.inf), dim=1) @ v[:, kv].double()
    return out


def _exact_accept(st, parents, start):
    """Request by request, node by node, on the host."""
    p, q, V = st["p"], st["q"], st["case"]["vocab"]
    token, u, u_final = st["token"].tolist(), st["u"].double().tolist(), st["u_final"].double().tolist()
    path, accepted, nexts = [-1] * len(token), [], []
    for b, parent in enumerate(parents):
        s, kept = start[b], [0]
        while True:
            full = p[s + kept[-1]].double().cpu().numpy()
            left, mass, go = full.copy(), 1.0, None
            for c in np.flatnonzero(parent == kept[-1]).tolist():
                if c <= kept[-1]:
                    continue
                x = token[s + c]
                draft = None if q is None else q[s + kept[-1]].double().cpu().numpy()
                if u[s + c] * mass * (1.0 if draft is None else draft[x]) < left[x]:
                    go = c
                    break
                if draft is None:
                    left[x] = 0.0
                elif mass > 0:
                    left = np.maximum(left / mass - draft, 0.0)
                mass = math.fsum(left[left > 0])
            if go is None:
                break
            kept.append(go)
        left = left if left.any() else full
        upto = np.cumsum(left)
        nexts.append(min(V - 1, int(np.searchsorted(upto, u_final[b] * upto[-1], side="right"))))
        accepted.append(len(kept) - 1)
        path[s:s + len(kept)] = kept
    return {"path": torch.tensor(path, device="cuda"), "accepted": torch.tensor(accepted, device="cuda"), "next": torch.tensor(nexts, device="cuda")}
