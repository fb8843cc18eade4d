"""Which way the attention of trees takes: whole items in one launch, or positions shared out over launches with scratch.  Either gives the same result."""
import ctypes

import numpy as np
import pytest
import torch

from test_gpu_tree_attention import Trees, _check, _parents, _wider, kb  # noqa: F401

pytestmark = pytest.mark.gpu


def _nodes(call):
    """Nodes of the graph that a capture of the call gives: one for the way that is a launch alone."""
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph(keep_graph=True)
    with torch.cuda.graph(graph):
        call()
    n = ctypes.c_size_t()
    assert ctypes.CDLL("libcuda.so.1").cuGraphGetNodes(ctypes.c_void_p(graph.raw_cuda_graph()), None, ctypes.byref(n)) == 0
    return n.value


# (requests, rows, heads, K/V heads, dimensions, positions that the table has room for, whether one launch is the sooner way): fp32 rows over fp32 pages
WAYS = [(2, 13, 4, 4, 64, 112, True), (22, 64, 8, 2, 64, 80, True), (3, 48, 32, 4, 128, 480, True), (1, 8, 40, 40, 128, 1472, False), (5, 2, 32, 32, 128, 1424, False), (6, 3, 4, 4, 64, 1216, False)]


@pytest.mark.parametrize("B,n,H,KV,hd,room,whole", WAYS)
def test_fp32_pages_go_the_sooner_way(kb, B, n, H, KV, hd, room, whole):  # noqa: F811
    rng = np.random.default_rng(room)
    p = Trees(kb, B, [room - n] * B, [_parents(rng, n, 5) for _ in range(B)], KV, hd, 16, "fp32")
    p.table = p.table[:, :room // 16].contiguous()
    q = p.q(H, hd, "fp32")
    out = torch.empty_like(q)
    assert (_nodes(lambda: p.run(kb, q, out=out)) == 1) == whole
    want, tol = p.want(q)
    _check(p.run(kb, q), want, tol)
    p.table = _wider(p.table, 200)                                   # room for more than the short way takes
    assert _nodes(lambda: p.run(kb, q, out=out)) > 1
    _check(p.run(kb, q), want, tol)
