"""Many requests at once on one paged K/V cache: prompts read together, then drafted and verified together.

    python examples/many_requests.py [--shape gqa-fp32] [--requests 5] [--max-new 24] [--k 4]

The library's Session decodes one request.  This example serves several with the operators for a paged cache:

  1. `knnssd_page_tables` finds pages and slots for the step's rows (and takes back those of rejected drafts and ended requests),
  2. a pass over all rows: per layer q, k, v by the linear maps, `knnssd_rotary_store`, attention, output map, MLP,
  3. prompts attend by `knnssd_packed_attention`, drafts (one row a request, masked sublayers left out) and verifications (k + 1 rows a
     request) by `knnssd_paged_attention`.

It prints each request's tokens and whether a Session of its own decodes the same.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import synthetic_inputs as si  # noqa: E402
from paper_2505_16162_b200 import binding as kb  # noqa: E402

PAGE = 16


def linear(W, x):
    """x W^T in fp32: by the prompt pass's contraction where it serves the sizes, else sixteen rows at a time."""
    if W.dtype == torch.bfloat16 and x.shape[0] > 16 and W.shape[1] % 64 == 0 and W.shape[0] % 8 == 0:
        return kb.knnssd_gemm_split(W, x.contiguous())
    return torch.cat([kb.knnssd_linear(W, x[i:i + 16].contiguous()) for i in range(0, x.shape[0], 16)])


class Batch:
    """The decoder of `shape` with `weights` for up to n_requests requests of up to max_seq positions."""

    def __init__(self, shape, weights, n_requests, max_seq, n_pages, mask):
        self.shape, self.w, self.mask, self.B = shape, weights, mask, n_requests
        i32 = dict(dtype=torch.int32, device="cuda")
        self.cos_sin = kb.rotary_table(max_seq, shape.head_dim, shape.rope_theta)
        cache = torch.float32 if shape.dtype == "fp32" else torch.bfloat16
        self.pools = [tuple(torch.zeros(n_pages, shape.n_kv_heads, PAGE, shape.head_dim, dtype=cache, device="cuda") for _ in range(2)) for _ in range(shape.n_layers)]
        self.wqkv = [torch.cat([q, k, v]) for q, k, v in zip(weights["wq"], weights["wk"], weights["wv"])]
        self.lens, self.owned = torch.zeros(n_requests, **i32), torch.zeros(n_requests, **i32)
        self.table = torch.full((n_requests, -(-max_seq // PAGE)), -1, **i32)
        self.free, self.count = torch.arange(n_pages, **i32), torch.full((1,), n_pages, **i32)

    def norm(self, x, g):
        return x * torch.rsqrt(x.square().mean(-1, keepdim=True) + self.shape.rms_eps) * g

    def step(self, lens, fresh, rows):
        """Pages for fresh rows behind lens positions of each request (-1: ended); the step's maps."""
        i32 = dict(dtype=torch.int32, device="cuda")
        s = {n: torch.empty(m, **i32) for n, m in (("start", self.B + 1), ("request", rows), ("pos", rows), ("slot", rows), ("info", 4))}
        s["lens"] = lens
        kb.knnssd_page_tables(lens, fresh, self.owned, self.table, self.free, self.count, PAGE, s["start"], s["request"], s["pos"], s["slot"], s["info"])
        info = s["info"].tolist()
        if info[3] != 0 or info[0] != rows:
            raise RuntimeError(f"no room for the step: {info}")
        return s

    def attend(self, q, k_pages, v_pages, s):
        return kb.knnssd_paged_attention(q, k_pages, v_pages, self.table, s["lens"], s["start"])

    def forward(self, tokens, s, mask=None, whole_prompts=False):
        """Last hidden states of the rows.  mask: sublayers left out (drafting)."""
        sh, w = self.shape, self.w
        x = w["tok_embed"][tokens].float()
        for l in range(sh.n_layers):
            if mask is None or not mask[2 * l]:
                qkv = linear(self.wqkv[l], self.norm(x, w["attn_norm"][l]))
                k_pages, v_pages = self.pools[l]
                if whole_prompts:
                    k = torch.empty(len(tokens), sh.n_kv_heads, sh.head_dim, device="cuda")
                    q = kb.knnssd_rotary_store(qkv, self.cos_sin, s["pos"], s["slot"], k_pages, v_pages, k_rows=k)
                    v = qkv.view(len(tokens), -1, sh.head_dim)[:, -sh.n_kv_heads:]
                    k, v = (t.to(k_pages.dtype).float() for t in (k, v))             # what later passes read from the pages
                    o = kb.knnssd_packed_attention(q, k, v, s["start"])
                else:
                    q = kb.knnssd_rotary_store(qkv, self.cos_sin, s["pos"], s["slot"], k_pages, v_pages)
                    o = self.attend(q, k_pages, v_pages, s)
                x = x + linear(w["wo"][l], o.view(len(tokens), -1))
            if mask is None or not mask[2 * l + 1]:
                y = self.norm(x, w["mlp_norm"][l])
                x = x + linear(w["w_down"][l], torch.nn.functional.silu(linear(w["w_gate"][l], y)) * linear(w["w_up"][l], y))
        return x

    def logits(self, x):
        return linear(self.w["lm_head"], self.norm(x, self.w["final_norm"]))

    def read(self, prompts):
        """All prompts in one pass; the first token of each."""
        n = torch.tensor([len(p) for p in prompts], dtype=torch.int32, device="cuda")
        s = self.step(self.lens, n, int(n.sum()))
        x = self.forward(torch.tensor([t for p in prompts for t in p], device="cuda"), s, whole_prompts=True)
        self.lens = n
        return self.logits(x[(s["start"][1:] - 1).long()]).argmax(-1)

    def round(self, pending, live, k):
        """Drafts k tokens for each live request and verifies them; [(accepted + 1) tokens] of each, the next pending ones last."""
        rows = [b for b in range(self.B) if live[b]]
        idx = torch.tensor(rows, device="cuda")
        fresh = lambda n: torch.tensor([n if a else -1 for a in live], dtype=torch.int32, device="cuda")  # noqa: E731
        tokens, drafts = pending[idx], []
        for i in range(k):
            s = self.step(self.lens + i * (fresh(1) > 0).int(), fresh(1), len(rows))
            tokens = self.logits(self.forward(tokens, s, mask=self.mask)).argmax(-1)
            drafts.append(tokens)
        candidates = torch.stack([pending[idx]] + drafts, dim=1)                     # [live][k + 1]
        s = self.step(self.lens, fresh(k + 1), candidates.numel())
        best = self.logits(self.forward(candidates.flatten(), s)).argmax(-1).view(len(rows), k + 1)
        agree = (candidates[:, 1:] == best[:, :k]).long().cumprod(1).sum(1)         # drafts accepted
        self.lens[idx] += (agree + 1).int()
        out = [[] for _ in range(self.B)]
        for b, a, t in zip(rows, agree.tolist(), best.tolist()):
            out[b] = t[:a + 1]
        return out


def decode(batch, prompts, max_new, k):
    """Greedy tokens of each request."""
    pending = batch.read(prompts)
    out = [[int(t)] for t in pending]
    while any(len(o) < m for o, m in zip(out, max_new)):
        live = [len(o) < m for o, m in zip(out, max_new)]
        for o, new in zip(out, batch.round(pending, live, k)):
            o += new
        pending = torch.tensor([o[-1] for o in out], device="cuda")
    end = torch.full((batch.B,), -1, dtype=torch.int32, device="cuda")              # all pages back
    batch.step(batch.lens, end, 0)
    return [o[:m] for o, m in zip(out, max_new)]


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--shape", default="gqa-fp32", choices=sorted(si.SHAPES))
    ap.add_argument("--requests", type=int, default=5)
    ap.add_argument("--max-new", type=int, default=24)
    ap.add_argument("--k", type=int, default=4)
    a = ap.parse_args()
    shape = si.SHAPES[a.shape]
    mask = si.skip_mask(0, 2 * shape.n_layers, shape.n_layers)
    weights = si.make_model_weights(shape, 0, device="cuda", damp={j: 0.05 for j in range(2 * shape.n_layers) if mask[j]})
    prompts = [si.uniform_tokens(0, b, n, shape.vocab).tolist() for b, n in enumerate(si.prompt_lengths(0, a.requests, 5, 90))]
    max_new = [a.max_new - 3 * (b % 3) for b in range(a.requests)]
    max_seq = max(map(len, prompts)) + a.max_new + 2 * a.k + 2
    batch = Batch(shape, weights, a.requests, max_seq, a.requests * -(-max_seq // PAGE), mask)
    same = 0
    for b, tokens in enumerate(decode(batch, prompts, max_new, a.k)):
        sess = kb.Session.from_shape(shape, weights, max_seq, max_draft=max(a.k, 1))
        sess.set_skipmask(mask)
        alone = sess.generate(prompts[b], max_new[b], a.k)["tokens"].tolist()
        sess.close()
        same += alone == tokens
        print(f"request {b}: {len(prompts[b])} prompt tokens, {len(tokens)} new, {'the same as' if alone == tokens else 'NOT as'} alone: {tokens}")
    print(f"{same} of {a.requests} requests as alone; {int(batch.count)} of {batch.free.numel()} pages free")


if __name__ == "__main__":
    main()
