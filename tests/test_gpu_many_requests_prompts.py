"""The example that serves many requests: its prompts attend to what later passes read, the cache's values."""
import pytest
import torch

import synthetic_inputs as si
from test_gpu_many_requests import mr  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("shape_name", ["stream-bf16", "gqa-fp32"])
def test_prompts_attend_to_the_cached_values(mr, monkeypatch, shape_name):  # noqa: F811
    shape = si.SHAPES[shape_name]
    w = si.make_model_weights(shape, 5, device="cuda")
    prompts = [si.uniform_tokens(5, b, n, shape.vocab).tolist() for b, n in enumerate([1, 33, 18])]
    batch = mr.Batch(shape, w, 3, 64, 12, None)
    seen, steps = [], []
    attention, step = mr.kb.knnssd_packed_attention, batch.step
    monkeypatch.setattr(mr.kb, "knnssd_packed_attention", lambda q, k, v, start: seen.append((k.clone(), v.clone())) or attention(q, k, v, start))
    monkeypatch.setattr(batch, "step", lambda *a: steps.append(step(*a)) or steps[-1])
    batch.read(prompts)
    assert len(seen) == shape.n_layers
    slot = steps[0]["slot"].long()
    for rows, pools in zip(seen, batch.pools):
        for x, pool in zip(rows, pools):
            assert torch.equal(x, pool.transpose(1, 2).reshape(-1, shape.n_kv_heads, shape.head_dim)[slot].float())
