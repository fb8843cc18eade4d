"""A verification round of token trees, all operators together: the example against one Session a request, and a round under a capture."""
import os
import sys

import numpy as np
import pytest
import torch

import synthetic_inputs as si
from oracle import trees as ot

pytestmark = pytest.mark.gpu
I32 = dict(dtype=torch.int32, device="cuda")

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


@pytest.mark.parametrize("shape_name,widths", [("tiny", [3, 2, 1]), ("gqa-fp32", [1, 1, 1]), ("gqa-fp32", [4, 3, 2, 1]), ("gqa-fp32", [])])
def test_requests_decode_as_they_do_alone(tt, shape_name, widths):
    shape, mask, w = _model(shape_name)
    prompts = [si.uniform_tokens(3, b, n, shape.vocab).tolist() for b, n in enumerate([1, 37, 16, 70])]
    max_new = [20, 7, 13, 1]
    n_pages = 4 * 16
    batch = tt.TreeBatch(shape, w, 4, 256, n_pages, mask, widths)
    got = tt.mr.decode(batch, prompts, max_new, None)
    assert int(batch.count) == n_pages and sorted(batch.free.tolist()) == list(range(n_pages))
    for p, m, tokens in zip(prompts, max_new, got):
        sess = tt.kb.Session.from_shape(shape, w, 256, max_draft=1)
        sess.set_skipmask(mask)
        assert sess.generate(p, m, 1)["tokens"].tolist() == tokens
        sess.close()


def test_kept_rows_leave_the_cache_of_a_plain_pass(tt):
    """After some rounds K and V of every request are what reading its tokens at once leaves: nothing of the rows that were dropped, everything in its place."""
    shape, mask, w = _model("gqa-fp32")
    prompts = [si.uniform_tokens(5, b, n, shape.vocab).tolist() for b, n in enumerate([20, 33])]
    batch = tt.TreeBatch(shape, w, 2, 256, 32, mask, [3, 2, 2])
    first = batch.read(prompts)
    texts, pending = [p + [int(t)] for p, t in zip(prompts, first)], first
    for _ in range(5):
        for t, new in zip(texts, batch.round(pending, [True, True])):
            t += new
        pending = torch.tensor([t[-1] for t in texts], device="cuda")
    assert batch.lens.tolist() == [len(t) - 1 for t in texts]
    plain = tt.TreeBatch(shape, w, 2, 256, 32, mask, [])
    plain.read([t[:-1] for t in texts])
    for b, n in enumerate(batch.lens.tolist()):
        at = torch.arange(n, device="cuda")
        for (k, v), (pk, pv) in zip(batch.pools, plain.pools):
            for x, y in ((k, pk), (v, pv)):
                x, y = x[batch.table[b, at // 16].long(), :, at % 16], y[plain.table[b, at // 16].long(), :, at % 16]
                assert (x - y).abs().max() <= 2e-4 * y.abs().max()   # fp32 maps and attention in other orders, layer on layer


@pytest.mark.parametrize("widths", [[2, 2], [1, 1, 1, 1]])
def test_sampled_rounds_run(tt, widths):
    shape, mask, w = _model("tiny")
    prompts = [si.uniform_tokens(7, b, n, shape.vocab).tolist() for b, n in enumerate([9, 40])]
    batch = tt.TreeBatch(shape, w, 2, 256, 32, mask, widths, temperature=0.7, top_p=0.9)
    got = tt.mr.decode(batch, prompts, [12, 9], None)
    assert [len(t) for t in got] == [12, 9] and all(0 <= x < shape.vocab for t in got for x in t)


def test_a_round_under_a_capture(tt):
    """Tables, attention, acceptance and the move as one graph, replayed with other trees, lengths and distributions in the same buffers; eager calls on another stream in between."""
    kb = tt.kb
    B, n, V, H, KV, hd, page = 3, 20, 700, 4, 2, 64, 16
    R = B * n
    start = torch.tensor([0, n, 2 * n, R], **I32)
    lens, parent, token = torch.zeros(B, **I32), torch.zeros(R, **I32), torch.zeros(R, **I32)
    table = torch.arange(B * 8, **I32).view(B, 8).flip(0).contiguous()
    pools = [torch.zeros(B * 8, KV, page, hd, device="cuda", dtype=torch.bfloat16) for _ in range(4)]
    handle = kb.PagePools(pools[:2], pools[2:])
    q = torch.zeros(R, H, hd, device="cuda", dtype=torch.bfloat16)
    p, dq, u, last = torch.zeros(R, V, device="cuda"), torch.zeros(R, V, device="cuda"), torch.zeros(R, device="cuda"), torch.zeros(B, device="cuda")
    pos, seen, state = torch.zeros(R, **I32), torch.zeros(R, dtype=torch.int64, device="cuda"), torch.zeros(B, **I32)
    path, accepted, nxt, o = torch.zeros(R, **I32), torch.zeros(B, **I32), torch.zeros(B, **I32), torch.zeros_like(q)

    def calls():
        kb.knnssd_tree_tables(lens, start, parent, pos, seen, state)
        kb.knnssd_tree_attention(q, pools[0], pools[2], table, lens, start, seen, out=o)
        kb.knnssd_tree_accept(p, dq, token, parent, start, u, last, path, accepted, nxt)
        kb.knnssd_keep_rows(handle, table, lens, start, path)

    def fill(seed):
        rng = np.random.default_rng(seed)
        t = lambda x, like: like.copy_(torch.as_tensor(x, device="cuda").to(like.dtype))  # noqa: E731
        t(rng.integers(0, 90, B), lens)
        trees = [[max(0, i - int(rng.integers(1, 6))) if i else -1 for i in range(n)] for _ in range(B)]
        t([x for tr in trees for x in tr], parent)
        w = rng.random((R, V)) ** 30
        t(w / w.sum(1, keepdims=True), dq)
        v = 0.7 * w + 0.3 * rng.random((R, V)) ** 30
        t(v / v.sum(1, keepdims=True), p)
        t(rng.random(R), u)
        t(rng.random(B), last)
        t([int(dq[b * n + max(trees[b][i], 0)].argmax()) for b in range(B) for i in range(n)], token)
        q.normal_()
        for x in pools:
            x.normal_()
        return trees

    graph = torch.cuda.CUDAGraph()
    fill(0)
    calls()
    with torch.cuda.graph(graph):
        calls()
    for seed in (1, 2, 3):
        trees = fill(seed)
        before = [x.clone() for x in pools]
        graph.replay()
        torch.cuda.synchronize()
        got = [x.clone() for x in (pos, seen, o, path, accepted, nxt, *pools)]
        for x, y in zip(pools, before):
            x.copy_(y)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            calls()
        side.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, (pos, seen, o, path, accepted, nxt, *pools)))
        for b in range(B):
            rows = slice(b * n, b * n + n)
            kept, t = ot.accept(p[rows].cpu().numpy(), dq[rows].cpu().numpy(), token[rows].tolist(), trees[b], u[rows].cpu().numpy(), float(last[b]))
            assert path[rows].tolist() == kept + [-1] * (n - len(kept)) and int(accepted[b]) == len(kept) - 1 and int(nxt[b]) == t
