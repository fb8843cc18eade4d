"""The operators for many requests under a capture, from the first call of a process on: what a call sets up once must not end the capture."""
import os
import subprocess
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

FIRST_CALLS = """
import sys
sys.path[:0] = [%r, %r]
import torch
from paper_2505_16162_b200 import binding as kb
from test_gpu_paged_attention import Paged, _check, _packed, _packed_want
i32 = dict(dtype=torch.int32, device="cuda")
p = Paged(5, [40, 300], [3, 2], 2, 64, 16, "bf16")
qkv = torch.randn(5, 8 * 64, device="cuda").bfloat16()
q = p.q(4, 64, "bf16")
cs = kb.rotary_table(400, 64, 10000.0)
lens, fresh = torch.tensor([0, 17], **i32), torch.tensor([20, 3], **i32)
owned, table, free, count = torch.zeros(2, **i32), torch.full((2, 4), -1, **i32), torch.arange(9, **i32), torch.full((1,), 9, **i32)
start, request, pos, slot, info = (torch.full((n,), 77, **i32) for n in (3, 5000, 5000, 5000, 4))
k, v = (torch.zeros(9, 2, 16, 64, device="cuda", dtype=torch.bfloat16) for _ in range(2))
at = torch.arange(5, **i32)
pq, pk, pv, ps = _packed(7, [70, 30], 4, 2, 64, "bf16")
calls = {
    "store": lambda: kb.knnssd_rotary_store(qkv, cs, at, at, k, v),
    "tables": lambda: kb.knnssd_page_tables(lens, fresh, owned, table, free, count, 16, start, request, pos, slot, info),
    "packed": lambda: kb.knnssd_packed_attention(pq, pk, pv, ps),
    "paged": lambda: p.run(kb, q),
    "fp32": lambda: kb.knnssd_packed_attention(pq.float(), pk.float(), pv.float(), ps),
}
torch.cuda.synchronize()
for name in %r:
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = calls[name]()
    graph.replay()
    torch.cuda.synchronize()
    if name == "store":
        assert torch.equal(v[0].transpose(0, 1)[:5].reshape(5, -1), qkv[:, 6 * 64:])
    elif name == "tables":
        assert info.tolist() == [23, 4, 0, 0] and table.tolist() == [[8, 7, -1, -1], [6, 5, -1, -1]] and start.tolist() == [0, 20, 23] and slot[20:24].tolist() == [5 * 16 + 1, 5 * 16 + 2, 5 * 16 + 3, -1]
    elif name == "paged":
        _check(got, *p.want(q))
    else:
        t = (lambda x: x.float()) if name == "fp32" else (lambda x: x)
        _check(got, *_packed_want(t(pq), t(pk), t(pv), [70, 30]))
print("captured")
"""


@pytest.mark.parametrize("first", ["packed", "fp32", "paged", "tables", "store"])
def test_the_first_call_of_a_process_under_a_capture(first):
    if not torch.cuda.is_available():
        pytest.fail("the gpu tests need a CUDA device")
    from paper_2505_16162_b200 import build
    build.build()
    order = [first] + [n for n in ("store", "tables", "packed", "paged", "fp32") if n != first]
    r = subprocess.run([sys.executable, "-c", FIRST_CALLS % (ROOT, os.path.join(ROOT, "tests"), order)], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "captured" in r.stdout, r.stderr[-2000:]
