"""Drafts that branch, for many requests on one paged K/V cache: a round drafts a tree of tokens for each request and verifies all of them in one pass.

    python examples/token_trees.py [--shape gqa-fp32] [--requests 5] [--max-new 24] [--widths 3,2,1] [--temperature 0]

The decoder, its cache and the reading of prompts are those of `many_requests.py`; a round is

  1. pages for the tree's rows (`knnssd_page_tables`), their positions and what each sees (`knnssd_tree_tables`),
  2. the draft model (masked sublayers left out) level by level: the rows of a level attend with their words of the whole tree's, the rows before them
     counted as held (`knnssd_tree_attention`); behind each row the next level gets its `widths` most probable tokens, or as many drawn ones,
  3. the full model over the whole tree in one pass,
  4. `knnssd_tree_agree` (greedy) or `knnssd_tree_accept` (sampled) finds the rows to keep and the token after them, `knnssd_keep_rows` moves their K and V together.

Greedy tokens are compared with one Session each.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import many_requests as mr  # noqa: E402

kb, si = mr.kb, mr.si
I32 = dict(dtype=torch.int32, device="cuda")


def tree_of(widths):
    """(parents of the rows, rows at which each level begins) of a tree whose rows of level l have widths[l] children each."""
    parents, levels = [-1], [0, 1]
    for w in widths:
        parents += [p for p in range(levels[-2], levels[-1]) for _ in range(w)]
        levels.append(len(parents))
    return parents, levels


class TreeBatch(mr.Batch):
    """A batch whose rounds draft the tree of `widths`.  temperature 0: greedy, drafts by rank; else sampled at top_p, drafts drawn."""

    def __init__(self, shape, weights, n_requests, max_seq, n_pages, mask, widths, temperature=0.0, top_p=1.0, seed=0):
        super().__init__(shape, weights, n_requests, max_seq, n_pages, mask)
        self.widths, self.temperature, self.top_p = list(widths), temperature, top_p
        self.parents, self.levels = tree_of(widths)
        self.page_pools = kb.PagePools([k for k, _ in self.pools], [v for _, v in self.pools])
        self.g = torch.Generator(device="cuda").manual_seed(seed)

    def attend(self, q, k_pages, v_pages, s):
        if "seen" not in s:
            return super().attend(q, k_pages, v_pages, s)
        return kb.knnssd_tree_attention(q, k_pages, v_pages, self.table, s["lens"], s["start"], s["seen"])

    def part(self, s, live, a, z):
        """The step's maps for rows a .. z - 1 of every live request, the rows before them counted as held."""
        n, L = len(self.parents), len(live)
        rows = (torch.arange(L, device="cuda")[:, None] * n + torch.arange(a, z, device="cuda")).flatten()
        fresh = torch.zeros(self.B, **I32)
        fresh[live] = z - a
        start = torch.cat([torch.zeros(1, **I32), fresh.cumsum(0, dtype=torch.int32)])
        return {"lens": s["lens"] + a, "start": start, "pos": s["pos"][rows], "slot": s["slot"][rows], "seen": s["seen"][rows]}

    def probabilities(self, logits):
        return kb.knnssd_filtered_probs(logits.contiguous(), self.temperature, self.top_p)

    def round(self, pending, live, k=None):
        """One round of the live requests; [tokens of each], the next pending ones last."""
        where = torch.tensor([b for b in range(self.B) if live[b]], device="cuda")
        n, L = len(self.parents), len(where)
        fresh = torch.tensor([n if a else -1 for a in live], **I32)
        s = self.step(self.lens, fresh, n * L)
        parent = torch.tensor(self.parents, **I32).repeat(L)
        s["seen"], state = torch.empty(n * L, dtype=torch.int64, device="cuda"), torch.empty(self.B, **I32)
        kb.knnssd_tree_tables(self.lens, s["start"], parent, s["pos"], s["seen"], state)
        # the draft model, a level of all trees at a time
        tokens, drafted = torch.zeros(L, n, dtype=torch.int64, device="cuda"), [None] * n
        tokens[:, 0] = pending[where]
        q = torch.zeros(L, n, self.shape.vocab, device="cuda") if self.temperature > 0 else None
        for w, a, z in zip(self.widths, self.levels, self.levels[1:]):
            logits = self.logits(self.forward(tokens[:, a:z].flatten(), self.part(s, where, a, z), mask=self.mask))
            if q is None:
                best = logits.topk(w, dim=-1).indices
            else:
                p = self.probabilities(logits)
                q[:, a:z] = p.view(L, z - a, -1)
                best = torch.multinomial(p, w, replacement=True, generator=self.g)
            tokens[:, z:z + (z - a) * w] = best.view(L, -1)
        # the full model over all rows, then what it keeps
        logits = self.logits(self.forward(tokens.flatten(), s))
        flat = tokens.flatten().int()
        path, accepted, nxt = torch.empty(n * L, **I32), torch.empty(self.B, **I32), torch.empty(self.B, **I32)
        if q is None:
            kb.knnssd_tree_agree(logits.argmax(-1).int(), flat, parent, s["start"], path, accepted, nxt)
        else:
            u, last = torch.rand(n * L, generator=self.g, device="cuda"), torch.rand(self.B, generator=self.g, device="cuda")
            kb.knnssd_tree_accept(self.probabilities(logits), q.flatten(0, 1), flat, parent, s["start"], u, last, path, accepted, nxt)
        kb.knnssd_keep_rows(self.page_pools, self.table, self.lens, s["start"], path)
        self.lens = self.lens + torch.where(fresh > 0, accepted + 1, 0).int()
        out = [[] for _ in range(self.B)]
        for b, row, p, m in zip(where.tolist(), tokens.tolist(), path.view(L, n).tolist(), nxt[where].tolist()):
            out[b] = [row[i] for i in p[1:] if i > 0] + [m]
        return out


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--shape", default="gqa-fp32", choices=sorted(si.SHAPES))
    ap.add_argument("--requests", type=int, default=5)
    ap.add_argument("--max-new", type=int, default=24)
    ap.add_argument("--widths", default="3,2,1")
    ap.add_argument("--temperature", type=float, default=0.0)
    ap.add_argument("--top-p", type=float, default=0.85)
    a = ap.parse_args()
    shape, widths = si.SHAPES[a.shape], [int(w) for w in a.widths.split(",")]
    mask = si.skip_mask(0, 2 * shape.n_layers, shape.n_layers)
    weights = si.make_model_weights(shape, 0, device="cuda", damp={j: 0.05 for j in range(2 * shape.n_layers) if mask[j]})
    prompts = [si.uniform_tokens(0, b, n, shape.vocab).tolist() for b, n in enumerate(si.prompt_lengths(0, a.requests, 5, 90))]
    max_new = [a.max_new - 3 * (b % 3) for b in range(a.requests)]
    rows = len(tree_of(widths)[0])
    max_seq = max(map(len, prompts)) + a.max_new + 2 * rows
    batch = TreeBatch(shape, weights, a.requests, max_seq, a.requests * -(-max_seq // mr.PAGE), mask, widths, a.temperature, a.top_p)
    same = 0
    for b, tokens in enumerate(mr.decode(batch, prompts, max_new, None)):
        if a.temperature > 0:
            print(f"request {b}: {len(prompts[b])} prompt tokens, {len(tokens)} new, sampled: {tokens}")
            continue
        sess = kb.Session.from_shape(shape, weights, max_seq, max_draft=1)
        sess.set_skipmask(mask)
        alone = sess.generate(prompts[b], max_new[b], 1)["tokens"].tolist()
        sess.close()
        same += alone == tokens
        print(f"request {b}: {len(prompts[b])} prompt tokens, {len(tokens)} new, {'the same as' if alone == tokens else 'NOT as'} alone: {tokens}")
    if a.temperature == 0:
        print(f"{same} of {a.requests} requests as alone; {int(batch.count)} of {batch.free.numel()} pages free")


if __name__ == "__main__":
    main()
