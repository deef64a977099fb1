"""Prompts taken to a paged KV cache in chunks, next to the blocks that a decoding loop verifies over it.

A few layers of random weights (a layer here is its attention: the packed projection, qkv_append, attention over the
pages, the output projection) run over a ragged batch: prompts in chunks of `chunk` tokens, all sequences in one call a
layer; then one drafted block of every sequence through the verify pass (qkv_append and block_attention_paged over the
same pages) and the drafter's pass over contiguous keys of its own (qk_norm_rope, block_attention).

    python examples/chunked_prefill.py
"""
from __future__ import annotations

import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2606_31315_gb300 as bp  # noqa: E402


def offsets(lengths) -> torch.Tensor:
    return torch.tensor([0, *torch.tensor(lengths).cumsum(0).tolist()], dtype=torch.int32, device="cuda")


def rotary_table(positions: int, dim: int, base: float = 1e6) -> torch.Tensor:
    angle = torch.arange(positions, dtype=torch.float64)[:, None] * base ** (-torch.arange(dim // 2, dtype=torch.float64) * 2 / dim)
    return torch.cat([angle.cos(), angle.sin()], 1).float().cuda()


class Model:
    """Layers of attention with random weights, and the pages of their caches."""

    def __init__(self, layers=2, hq=32, hkv=8, dim=128, page=64, capacity=(1000, 700, 90), seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        bf = torch.bfloat16
        self.hq, self.hkv, self.dim, self.page, self.hidden = hq, hkv, dim, page, hq * dim
        rand = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
        self.qkv = [(rand((hq + 2 * hkv) * dim, self.hidden) / math.sqrt(self.hidden)).to(bf) for _ in range(layers)]
        self.out = [(rand(self.hidden, self.hidden) / math.sqrt(self.hidden)).to(bf) for _ in range(layers)]
        self.norm = [[(1 + 0.1 * rand(dim)).to(bf) for _ in range(2)] for _ in range(layers)]
        need = [-(-n // page) for n in capacity]
        order = torch.randperm(sum(need), generator=torch.Generator().manual_seed(seed)).to(torch.int32)
        table = torch.zeros(len(need), max(need), dtype=torch.int32)
        for s, n in enumerate(need):
            table[s, :n] = order[sum(need[:s]):sum(need[:s]) + n]
        self.pages = table.cuda()
        # (zeros: the verify pass's attention wants every row of its pages finite)
        self.caches = [[torch.zeros(sum(need) * page, hkv, dim, device="cuda", dtype=bf) for _ in range(2)] for _ in range(layers)]
        self.table = rotary_table(max(need) * page, dim)
        self.small = bp.workspace(256, "cuda")
        self.ws = {}

    def step(self, x, new, held, block=False):
        """One pass of new[s] tokens of every sequence, held[s] keys before them, through all layers; x [sum(new), hidden]."""
        cu_new, cu_kv = offsets(new), offsets([h + n for h, n in zip(held, new)])
        longest = max(h + n for h, n in zip(held, new))
        size = (len(new), x.shape[0], self.hq, self.hkv, self.dim)
        if block:
            ws = bp.workspace(bp.block_attention_workspace_size(len(new), max(new), self.hq, self.hkv, self.dim), "cuda")
        else:
            need = bp.chunk_attention_workspace_size(*size)
            ws = self.ws.setdefault(need, bp.workspace(need, "cuda"))
        for (k, v), wqkv, wo, (qn, kn) in zip(self.caches, self.qkv, self.out, self.norm):
            packed = (x @ wqkv.t()).view(x.shape[0], self.hq + 2 * self.hkv, self.dim)
            q = bp.qkv_append(packed, k, v, cu_new, cu_kv, self.pages, self.page, self.table, q_weight=qn, k_weight=kn,
                              ws=self.small)
            if block:  # a drafted block: the verify pass's kernel (at most 64 positions)
                o, _ = bp.block_attention_paged(q, k, v, cu_new, cu_kv, self.pages, self.page, int(cu_kv[-1]), max(new),
                                                longest, ws=ws)
            else:
                o, _ = bp.chunk_attention_paged(q, k, v, cu_new, cu_kv, self.pages, self.page, max(new), longest, ws=ws)
            x = x + o.view(x.shape[0], self.hidden) @ wo.t()
        assert bp.get_status(self.small) == 0 and bp.get_status(ws) == 0
        return x

    def prefill(self, prompts, chunk):
        """prompts: embeddings [length, hidden] of every sequence; returns their last layer's rows, as given."""
        done = [0] * len(prompts)
        rows = [[] for _ in prompts]
        while any(d < len(p) for d, p in zip(done, prompts)):
            new = [min(chunk, len(p) - d) for d, p in zip(done, prompts)]
            x = self.step(torch.cat([p[d:d + n] for p, d, n in zip(prompts, done, new)]), new, done)
            for s, part in enumerate(x.split(new)):
                rows[s].append(part)
            done = [d + n for d, n in zip(done, new)]
        return [torch.cat(r) for r in rows]

    def draft(self, x, keys, values, held):
        """A drafter's pass: a block of mask tokens over contiguous keys of its own that it norms and rotates itself."""
        b = x.shape[0]
        packed = (x @ self.qkv[0].t()).view(b, self.hq + 2 * self.hkv, self.dim)
        q, k, v = packed.split([self.hq, self.hkv, self.hkv], 1)
        pos = torch.arange(held, held + b, device="cuda", dtype=torch.int32)
        q, k = bp.qk_norm_rope(q, k, self.table, pos, q_weight=self.norm[0][0], k_weight=self.norm[0][1], ws=self.small)
        o, _ = bp.block_attention(q, torch.cat([keys, k]), torch.cat([values, v]), offsets([b]), offsets([held + b]), b,
                                  held + b, mask=bp.MASK_BIDIR)
        return o


def main():
    bp.build()
    lengths, block = (900, 333, 40), 16
    model = Model()
    g = torch.Generator(device="cuda").manual_seed(1)
    prompts = [torch.randn(n, model.hidden, device="cuda", generator=g).to(torch.bfloat16) for n in lengths]
    whole = model.prefill(prompts, max(lengths))
    parts = model.prefill(prompts, 128)
    off = max(float((a.float() - b.float()).norm() / b.float().norm()) for a, b in zip(parts, whole))
    print(f"prompts of {lengths} tokens in chunks of 128 against all at once: rows differ by {off:.1e} of their size")
    x = torch.randn(block * len(lengths), model.hidden, device="cuda", generator=g).to(torch.bfloat16)
    checked = model.step(x, [block] * len(lengths), list(lengths), block=True)
    again = model.step(x, [block] * len(lengths), list(lengths))
    near = float((checked.float() - again.float()).norm() / again.float().norm())
    print(f"a block of {block} over them, by the verify pass and as a chunk: {near:.1e}")
    keys, values = (torch.randn(100, model.hkv, model.dim, device="cuda", generator=g).to(torch.bfloat16) for _ in range(2))
    o = model.draft(x[:block], keys, values, 100)
    print("a drafter's block over keys of its own:", tuple(o.shape))
    return off, near, bool(torch.isfinite(o.float()).all())


if __name__ == "__main__":
    main()
