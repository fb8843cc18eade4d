"""The example that serves many requests with the paged operators, against one Session a request."""
import os
import sys

import pytest
import torch

import synthetic_inputs as si

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.fixture(scope="module")
def mr():
    if not torch.cuda.is_available():
        pytest.fail("the gpu tests need a CUDA device")
    from paper_2505_16162_b200 import build
    build.build()
    import many_requests
    return many_requests


@pytest.mark.parametrize("shape_name,k", [("tiny", 4), ("gqa-fp32", 3), ("gqa-fp32", 0)])
def test_requests_decode_as_they_do_alone(mr, shape_name, k):
    shape = si.SHAPES[shape_name]
    mask = si.skip_mask(1, 2 * shape.n_layers, shape.n_layers)
    w = si.make_model_weights(shape, 3, device="cuda", damp={j: 0.05 for j in range(2 * shape.n_layers) if mask[j]}, gain_spread=0.1)
    prompts = [si.uniform_tokens(3, b, n, shape.vocab).tolist() for b, n in enumerate([1, 37, 16, 70])]
    max_new = [20, 7, 13, 1]
    n_pages = 4 * 8
    batch = mr.Batch(shape, w, 4, 128, n_pages, mask)
    got = mr.decode(batch, prompts, max_new, k)
    assert int(batch.count) == n_pages and sorted(batch.free.tolist()) == list(range(n_pages))
    for p, m, tokens in zip(prompts, max_new, got):
        sess = mr.kb.Session.from_shape(shape, w, 128, max_draft=max(k, 1))
        sess.set_skipmask(mask)
        assert sess.generate(p, m, k)["tokens"].tolist() == tokens
        sess.close()


def test_logits_of_a_bf16_model(mr):
    """Prompt, then k + 1 rows a request: logits of all against the Session's, within the tolerance that the bf16 shapes have elsewhere."""
    shape = si.SHAPES["stream-bf16"]
    w = si.make_model_weights(shape, 5, device="cuda")
    prompts = [si.uniform_tokens(5, b, n, shape.vocab).tolist() for b, n in enumerate([33, 18, 50])]
    drafts = [si.uniform_tokens(6, b, 3, shape.vocab).tolist() for b in range(3)]
    batch = mr.Batch(shape, w, 3, 96, 18, None)
    first = batch.read(prompts)
    s = batch.step(batch.lens, torch.full((3,), 4, dtype=torch.int32, device="cuda"), 12)
    want = []
    for p, d in zip(prompts, drafts):
        sess = mr.kb.Session.from_shape(shape, w, 96, max_draft=4)
        t = sess.prefill(p)
        want.append((t, sess.verify(d, want_logits=True)["logits"]))
        sess.close()
    tokens = [x for (t, _), d in zip(want, drafts) for x in [t] + d]
    got = batch.logits(batch.forward(torch.tensor(tokens, device="cuda"), s)).view(3, 4, -1)
    for b, (t, logits) in enumerate(want):
        assert (got[b] - logits).abs().max() <= 2e-2
    assert first.shape == (3,)
