"""The greedy acceptance under a capture: its own buffers, its own results, as a process's first call as well."""
import os
import subprocess
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

CODE = """
import sys
sys.path[:0] = [%r]
import torch
from oracle import trees as ot
from paper_2505_16162_b200 import binding as kb
i32 = dict(dtype=torch.int32, device="cuda")
parents = [[-1, 0, 0, 1, 1, 2, 2, 5, 7], [-1, 0, 1, 1, 3], []]
start = [1, 10, 15, 15]
token, parent = torch.tensor([9, 4, 5, 6, 7, 8, 1, 2, 3, 4, 4, 6, 7, 8, 9, 3], **i32), torch.tensor([0] + [x for p in parents for x in p] + [0], **i32)
best, at = torch.zeros(16, **i32), torch.tensor(start, **i32)
path, accepted, nxt = (torch.full((n,), 77, **i32) for n in (16, 3, 3))
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    kb.knnssd_tree_agree(best, token, parent, at, path, accepted, nxt)
assert path.tolist() == [77] * 16 and accepted.tolist() == nxt.tolist() == [77] * 3
for choices in ([6, 1, 1, 4, 1, 1, 2, 1, 1], [0] * 9), ([5, 1, 1, 1, 1, 1, 1, 1, 1], [6, 8, 1, 9, 2]), ([1] * 9, [6, 7, 3, 3, 3]):
    best.copy_(torch.tensor([4] + choices[0] + choices[1][:5] + [4]))
    for x in (path, accepted, nxt):
        x.fill_(77)
    graph.replay()
    torch.cuda.synchronize()
    want, kept, tokens = [-1] * 16, [], []
    for b, p in enumerate(parents):
        rows = slice(start[b], start[b + 1])
        k, t = ot.agree(best[rows].tolist(), token[rows].tolist(), p) if p else ([], -1)
        want[start[b]:start[b] + len(k)] = k
        kept.append(max(0, len(k) - 1))
        tokens.append(t)
    assert [path.tolist(), accepted.tolist(), nxt.tolist()] == [want, kept, tokens], (path, accepted, nxt, want, kept, tokens)
    print("kept", kept)
print("captured")
"""


def test_the_greedy_form_under_a_capture():
    if not torch.cuda.is_available():
        pytest.fail("the gpu tests need a CUDA device")
    from paper_2505_16162_b200 import build
    build.build()
    r = subprocess.run([sys.executable, "-c", CODE % ROOT], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "captured" in r.stdout, r.stderr[-2000:]
    assert max(int(x) for line in r.stdout.splitlines() if line.startswith("kept") for x in line[6:-1].split(",")) >= 2
