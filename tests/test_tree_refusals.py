"""The operators for drafts that branch refuse what they cannot do before anything is enqueued (no GPU: statuses of the C ABI)."""
import ctypes as C

import pytest


@pytest.fixture(scope="module")
def kb():
    from paper_2505_16162_b200 import build
    build.build()
    from paper_2505_16162_b200 import binding
    return binding


A = 1 << 20                                                          # an address that nothing is read from
GOOD = {
    "knnssd_tree_tables": dict(lens=A, row_start=A, parent=A, n_requests=2, n_rows=5, pos=A, seen=A, state=A, stream=None),
    "knnssd_tree_attention": dict(q=A, dtype=1, n_rows=5, q_stride=512, n_heads=8, n_kv_heads=2, head_dim=64, k=A, v=A, cache=1, page=16, n_pages=9, table=A, max_pages=4, lens=A,
                                  row_start=A, seen=A, n_requests=2, max_fresh=0, scale=0.1, out=A, stream=None),
    "knnssd_tree_accept": dict(p=A, q=A, vocab=100, token=A, parent=A, row_start=A, n_requests=2, n_rows=5, u=A, u_final=A, path=A, accepted=A, next=A, stream=None),
    "knnssd_tree_agree": dict(best=A, token=A, parent=A, row_start=A, n_requests=2, n_rows=5, path=A, accepted=A, next=A, stream=None),
    "knnssd_keep_rows": dict(pools=None, n_pools=2, cache=1, n_kv_heads=2, head_dim=64, page=16, n_pages=9, table=A, max_pages=4, lens=A, row_start=A, path=A, n_requests=2, n_rows=5,
                             stream=None),
}
CASES = [
    *[("knnssd_tree_tables", {n: None}, 1) for n in ("lens", "row_start", "parent", "pos", "seen", "state")],
    ("knnssd_tree_tables", {"n_requests": 0}, 1), ("knnssd_tree_tables", {"n_rows": -1}, 1), ("knnssd_tree_tables", {"seen": A + 4}, 2),
    *[("knnssd_tree_attention", {n: None}, 1) for n in ("q", "k", "v", "table", "lens", "row_start", "seen", "out")],
    *[("knnssd_tree_attention", {n: A + 8}, 2) for n in ("q", "k", "v", "out")],
    ("knnssd_tree_attention", {"seen": A + 4}, 2), ("knnssd_tree_attention", {"cache": 0}, 2), ("knnssd_tree_attention", {"dtype": 2}, 1),
    ("knnssd_tree_attention", {"n_heads": 7}, 2), ("knnssd_tree_attention", {"head_dim": 96}, 2), ("knnssd_tree_attention", {"page": 24}, 2), ("knnssd_tree_attention", {"page": 8}, 2),
    ("knnssd_tree_attention", {"q_stride": 511}, 2), ("knnssd_tree_attention", {"max_fresh": -1}, 1), ("knnssd_tree_attention", {"scale": float("inf")}, 1),
    ("knnssd_tree_attention", {"scale": -1.0}, 1), ("knnssd_tree_attention", {"n_pages": 1 << 28}, 3), ("knnssd_tree_attention", {"n_requests": 0}, 1),
    ("knnssd_tree_attention", {"n_rows": 1 << 29}, 3),
    *[("knnssd_tree_accept", {n: None}, 1) for n in ("p", "token", "parent", "row_start", "u", "u_final", "path", "accepted", "next")],
    ("knnssd_tree_accept", {"vocab": 0}, 1), ("knnssd_tree_accept", {"vocab": (1 << 24) + 1}, 3), ("knnssd_tree_accept", {"n_requests": 8193}, 3),
    ("knnssd_tree_accept", {"n_requests": 0}, 1), ("knnssd_tree_accept", {"n_rows": -1}, 1),
    *[("knnssd_tree_agree", {n: None}, 1) for n in ("best", "token", "parent", "row_start", "path", "accepted", "next")],
    ("knnssd_tree_agree", {"n_requests": 0}, 1), ("knnssd_tree_agree", {"n_rows": -1}, 1),
    *[("knnssd_keep_rows", {n: None}, 1) for n in ("table", "lens", "row_start", "path")],
    ("knnssd_keep_rows", {"pools": (A, None)}, 1), ("knnssd_keep_rows", {"pools": (A, A + 8)}, 2), ("knnssd_keep_rows", {"pools": "NULL"}, 1), ("knnssd_keep_rows", {"n_pools": 0}, 1),
    ("knnssd_keep_rows", {"cache": 2}, 1), ("knnssd_keep_rows", {"head_dim": 32}, 2), ("knnssd_keep_rows", {"page": 20}, 2), ("knnssd_keep_rows", {"max_pages": 1 << 28}, 3),
    ("knnssd_keep_rows", {"n_requests": 0}, 1), ("knnssd_keep_rows", {"n_kv_heads": 0}, 1),
]


@pytest.mark.parametrize("name,change,status", CASES)
def test_a_call_that_is_refused(kb, name, change, status):
    args = {**GOOD[name], **change}
    if name == "knnssd_keep_rows":
        pools = args["pools"] or (A, A)
        args["pools"] = None if pools == "NULL" else (C.c_void_p * 2)(*pools)
    assert getattr(kb._lib, name)(*args.values()) == status


def test_no_rows_are_nothing_to_do(kb):
    none = {**GOOD["knnssd_tree_attention"], "n_rows": 0, "q": None, "out": None, "seen": None}
    assert kb._lib.knnssd_tree_attention(*none.values()) == 0
    none = {**GOOD["knnssd_keep_rows"], "n_rows": 0, "path": None, "pools": (C.c_void_p * 2)(A, A)}
    assert kb._lib.knnssd_keep_rows(*none.values()) == 0
