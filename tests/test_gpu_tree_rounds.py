"""Whole rounds of token trees on a bf16 cache, drafted level by level by a model and verified by it: greedy tokens against a plain pass, sampled ones against the oracle.

Tolerance of the logits: those of bf16 shapes lie within 2e-2 of a Session's whichever operators form them (``test_gpu_many_requests``), two ways of forming them within twice that of one another, so a
choice by the one is at most four times 2e-2 below the other's largest.
"""
import os
import sys

import pytest
import torch

import synthetic_inputs as si
from oracle import trees as ot
from test_gpu_tree_accept import _moved

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.fixture(scope="module")
def tt():
    if not torch.cuda.is_available():
        pytest.fail("the gpu tests need a CUDA device")
    from paper_2505_16162_b200 import build
    build.build()
    import token_trees
    return token_trees


def _model(shape_name):
    shape = si.SHAPES[shape_name]
    mask = si.skip_mask(1, 2 * shape.n_layers, shape.n_layers)
    return shape, mask, si.make_model_weights(shape, 3, device="cuda", damp={j: 0.05 for j in range(2 * shape.n_layers) if mask[j]}, gain_spread=0.1)


@pytest.mark.parametrize("shape_name,widths", [("gqa-bf16", [3, 2, 1]), ("stream-bf16", [1, 1, 1]), ("stream-bf16", [4, 2, 2]), ("ragged-bf16", [2, 2, 1, 1])])
def test_greedy_tokens_over_a_bf16_cache(tt, shape_name, widths):
    shape, mask, w = _model(shape_name)
    prompts = [si.uniform_tokens(3, b, n, shape.vocab).tolist() for b, n in enumerate([1, 37, 16, 70])]
    max_new = [20, 7, 13, 9]
    n_pages = 4 * 16
    batch = tt.TreeBatch(shape, w, 4, 256, n_pages, mask, widths)
    got = tt.mr.decode(batch, prompts, max_new, None)
    assert int(batch.count) == n_pages and [len(t) for t in got] == max_new
    plain = tt.mr.Batch(shape, w, 4, 256, n_pages, mask)
    texts = [p + t[:-1] for p, t in zip(prompts, got)]
    n = torch.tensor([len(t) for t in texts], dtype=torch.int32, device="cuda")
    s = plain.step(plain.lens, n, int(n.sum()))
    logits = plain.logits(plain.forward(torch.tensor([x for t in texts for x in t], device="cuda"), s, whole_prompts=True))
    for b, (p, t) in enumerate(zip(prompts, got)):
        rows = logits[int(s["start"][b]) + len(p) - 1:int(s["start"][b + 1])]
        below = rows.max(1).values - rows[torch.arange(len(t)), torch.tensor(t, device="cuda")]
        assert len(rows) == len(t) and below.max() <= 8e-2


@pytest.mark.parametrize("shape_name,widths", [("gqa-bf16", [3, 2]), ("stream-bf16", [2, 2, 1]), ("gqa-fp32", [3, 2, 1])])
def test_sampled_rounds_are_the_oracles(tt, monkeypatch, shape_name, widths):
    """What the model and the random numbers gave a round goes to the oracle as well: the same rows kept, the same token behind them, their K and V in their places."""
    shape, mask, w = _model(shape_name)
    prompts = [si.uniform_tokens(7, b, n, shape.vocab).tolist() for b, n in enumerate([9, 40, 15])]
    batch = tt.TreeBatch(shape, w, 3, 256, 48, mask, widths, temperature=0.7, top_p=0.9, seed=4)
    pending = batch.read(prompts)
    accept, keep, calls = tt.kb.knnssd_tree_accept, tt.kb.knnssd_keep_rows, []

    def accepted(*args):
        accept(*args)
        calls.append([a.clone() for a in args])

    def kept(pools, table, lens, start, path):
        flat = [x for pool in batch.pools for x in pool]
        want = _moved(flat, table, lens.tolist(), start.tolist(), path.tolist(), tt.mr.PAGE)
        keep(pools, table, lens, start, path)
        assert all(torch.equal(a, b) for a, b in zip(flat, want))

    monkeypatch.setattr(tt.kb, "knnssd_tree_accept", accepted)
    monkeypatch.setattr(tt.kb, "knnssd_keep_rows", kept)
    drafts_kept = 0
    for live in ([True] * 3, [True] * 3, [True, False, True], [True] * 3, [False, True, False]):
        before = batch.lens.tolist()
        new = batch.round(pending, live)
        p, q, token, parent, start, u, last, path, n_accepted, nxt = (a.cpu().numpy() for a in calls.pop())
        for b in range(3):
            rows = slice(int(start[b]), int(start[b + 1]))
            if not live[b]:
                assert rows.start == rows.stop and not new[b] and int(batch.lens[b]) == before[b]
                continue
            k, t = ot.accept(p[rows], q[rows], token[rows].tolist(), parent[rows].tolist(), u[rows], float(last[b]))
            assert path[rows].tolist() == k + [-1] * (rows.stop - rows.start - len(k)) and (n_accepted[b], nxt[b]) == (len(k) - 1, t)
            assert new[b] == [int(token[rows][i]) for i in k[1:]] + [t] and int(batch.lens[b]) == before[b] + len(k)
            drafts_kept += len(k) - 1
        pending = torch.tensor([n[-1] if n else int(x) for n, x in zip(new, pending)], device="cuda")
    assert drafts_kept > 0
