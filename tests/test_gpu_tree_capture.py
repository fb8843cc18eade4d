"""The operators for drafts that branch under a capture, from the first call of a process on, and from several threads at once."""
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
import numpy as np
import torch
from paper_2505_16162_b200 import binding as kb
from test_gpu_tree_attention import Trees, _check, _parents
from test_gpu_tree_accept import Round, _moved, _pools
i32 = dict(dtype=torch.int32, device="cuda")
rng = np.random.default_rng(1)
words = [[(1 << 64) - 1] * 9, [1] * 4]
t = Trees(kb, 5, [40, 300], [[-1] * 9, [-1] * 4], 2, 64, 16, "bf16", words=words)
q = t.q(4, 64, "bf16")
r = Round(3, [_parents(rng, 12, 3) for _ in range(2)], 70000, True, zeros=0.5)          # enough ids for clusters of sixteen
out = [torch.zeros(n, **i32) for n in (24, 2, 2)]
args = r.on_device()
pools, table = _pools(4, 2, [30], [6], 2, 64, 16, torch.bfloat16)
want = _moved(pools, table, [30], [0, 6], [0, 2, 5, -1, -1, -1], 16)
handle, moved = kb.PagePools(pools[:1], pools[1:]), [torch.tensor(x, **i32) for x in ([30], [0, 6], [0, 2, 5, -1, -1, -1])]
parent, start, lens = torch.tensor([-1, 0, 0, 1], **i32), torch.tensor([0, 4], **i32), torch.tensor([7], **i32)
pos, seen, state = torch.zeros(4, **i32), torch.zeros(4, dtype=torch.int64, device="cuda"), torch.zeros(1, **i32)
calls = {
    "tables": lambda: kb.knnssd_tree_tables(lens, start, parent, pos, seen, state),
    "bf16": lambda: t.run(kb, q),
    "fp32": lambda: t.run(kb, q.float()),
    "accept": lambda: kb.knnssd_tree_accept(*args, *out),
    "agree": lambda: kb.knnssd_tree_agree(args[2], args[2], args[3], args[4], *out),
    "keep": lambda: kb.knnssd_keep_rows(handle, table, *moved),
}
torch.cuda.synchronize()
for name in %r:
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = calls[name]()
    graph.replay()
    torch.cuda.synchronize()
    if name == "tables":
        assert pos.tolist() == [7, 8, 8, 9] and seen.tolist() == [-1, -1, -3, -3] and state.tolist() == [0]      # rows 2 and 3 do not see the row before them
    elif name in ("bf16", "fp32"):
        _check(got, *t.want(q if name == "bf16" else q.float()))
    elif name == "accept":
        assert tuple(x.tolist() for x in out) == r.want()
    elif name == "agree":
        assert out[1].max() <= 11 and out[0][::12].tolist() == [0, 0]
    else:
        assert all(torch.equal(a, b) for a, b in zip(pools, want))
print("captured")
"""


@pytest.mark.parametrize("first", ["tables", "bf16", "fp32", "accept", "agree", "keep"])
def test_the_first_call_of_a_process_under_a_capture(first):
    if not torch.cuda.is_available():
        pytest.fail("the gpu tests need a CUDA device")
    from paper_2505_16162_b200 import build
    build.build()
    order = [first] + [n for n in ("keep", "accept", "tables", "bf16", "agree", "fp32") if n != first]
    r = subprocess.run([sys.executable, "-c", FIRST_CALLS % (ROOT, os.path.join(ROOT, "tests"), order)], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "captured" in r.stdout, r.stderr[-2000:]


def test_threads_with_streams_of_their_own():
    import threading
    import numpy as np
    from paper_2505_16162_b200 import build
    build.build()
    from paper_2505_16162_b200 import binding as kb
    from test_gpu_tree_accept import Round, _parents
    from test_gpu_tree_attention import Trees
    rng = np.random.default_rng(2)
    jobs = []
    for i in range(4):
        dtype = ("bf16", "fp32")[i % 2]
        t = Trees(kb, 30 + i, [200 * i, 30], [_parents(rng, 20, 4), _parents(rng, 9, 3)], 2, 128, (16, 64)[i // 2], "bf16")
        r = Round(40 + i, [_parents(rng, 15, 4) for _ in range(3)], 5000 * (i + 1), i % 2 == 0)
        jobs.append((t, t.q(6, 128, dtype), r, r.on_device()))
    want = [(t.run(kb, q), r.want()) for t, q, r, _ in jobs]
    torch.cuda.synchronize()
    wrong = []

    def work(i):
        t, q, r, args = jobs[i]
        s = torch.cuda.Stream()
        with torch.cuda.stream(s):
            for _ in range(30):
                got = t.run(kb, q)
                out = [torch.empty(n, dtype=torch.int32, device="cuda") for n in (len(r.token), 3, 3)]
                kb.knnssd_tree_accept(*args, *out)
            s.synchronize()
            if not torch.equal(got, want[i][0]) or tuple(x.tolist() for x in out) != want[i][1]:
                wrong.append(i)

    threads = [threading.Thread(target=work, args=(i,)) for i in range(4)]
    for x in threads:
        x.start()
    for x in threads:
        x.join()
    assert not wrong
