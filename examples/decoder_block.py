#!/usr/bin/env python3
"""A decoder block's step on the library's kernels, for decode and for fine-tuning.

    python examples/decoder_block.py [--steps 24] [--budget 16]

Random weights, quantized to 4 bits with weak columns.  Decode: a few sequences take one token at a time through a stack of blocks - norm,
query / key / value projections in one launch, rotation and append to the paged cache, attention over it with its weights accumulated, output projection,
norm with the residual addition, gate / up, down - and caches that have grown over the budget drop the tokens of least accumulated weight.  Fine-tuning:
forward and backward of a block's second half, with the gradients of its norms and weak columns.  PyTorch does what is not the library's: memory, SiLU,
the bookkeeping of lengths.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2410_08661_amd import binding as B  # noqa: E402


def rotation(positions, dim, device="cuda"):
    """[position][cosines, sines] of dim / 2 frequencies, angles in 64 bits."""
    f = 10000.0 ** (-torch.arange(0, dim, 2, dtype=torch.float64, device=device) / dim)
    a = torch.arange(positions, dtype=torch.float64, device=device)[:, None] * f
    return torch.cat([a.cos(), a.sin()], 1).float()


class Linear:
    def __init__(self, out_features, in_features, n_weak, gen):
        self.desc = B.make_desc(out_features, in_features, n_weak, 4, 128)
        w = torch.randn((out_features, in_features), generator=gen, device="cuda") * in_features ** -0.5
        self.weight = B.qeft_pack(self.desc, w.half())


class Block:
    """The layers of one block and the cache of its keys and values."""

    def __init__(self, hidden, heads, kv_heads, ffn, n_weak, gen, pages, page_size, seqs, table_pages):
        self.heads, self.kv, self.d = heads, kv_heads, hidden // heads
        mk = lambda o, i: Linear(o, i, n_weak, gen)  # noqa: E731
        self.q, self.k, self.v = mk(hidden, hidden), mk(kv_heads * self.d, hidden), mk(kv_heads * self.d, hidden)
        self.o, self.gate, self.up, self.down = mk(hidden, hidden), mk(ffn, hidden), mk(ffn, hidden), mk(hidden, ffn)
        self.w_attn, self.w_mlp = ((1 + 0.1 * torch.randn(hidden, generator=gen, device="cuda")).half() for _ in range(2))
        self.cache = B.Cache(B.make_cache_desc(pages, page_size, kv_heads, self.d))
        tokens = table_pages * page_size
        self.score = torch.zeros((seqs, kv_heads, tokens), device="cuda")
        self.pos = torch.zeros((seqs, kv_heads, tokens), dtype=torch.int32, device="cuda")

    def decode(self, norm, h, x, table, lens, longest, seen, rot, w_next):
        """One token of every sequence: residual stream h, its norm x; returns both for the next block.  lens: the tokens in the cache before this one, fewer than
        `longest`, which is what the caller knows of them."""
        if longest > self.score.shape[2]:
            raise ValueError(f"a sequence of {longest} tokens in a table for {self.score.shape[2]}")
        q, k, v = B.qeft_linear_fwd_group([l.desc for l in (self.q, self.k, self.v)], [l.weight for l in (self.q, self.k, self.v)], x)
        B.qeft_cache_append(self.cache, table, k, v, lens, q=q, q_out=q, rot=rot, pos=seen)
        at = lens.long()[:, None, None].expand(-1, self.kv, 1)      # the new token's weight starts at zero
        self.score.scatter_(2, at, 0.0)
        self.pos.scatter_(2, at, seen[:, None, None].expand(-1, self.kv, 1))
        a = B.qeft_attn_decode(self.cache, table, lens + 1, longest, q, score=self.score, accumulate=True)
        y = B.qeft_linear_fwd(self.o.desc, self.o.weight, a)
        h, x = B.qeft_norm_fwd(norm, h, self.w_mlp, y=y, h=h)
        g, u = B.qeft_linear_fwd_group([self.gate.desc, self.up.desc], [self.gate.weight, self.up.weight], x)
        y = B.qeft_linear_fwd(self.down.desc, self.down.weight, torch.nn.functional.silu(g) * u)
        return B.qeft_norm_fwd(norm, h, w_next, y=y, h=h)

    def evict(self, table, lens, longest, budget, seen, keep_first, keep_last):
        return B.qeft_cache_evict(self.cache, table, lens, longest, budget, self.score, self.pos, seen, keep_first=keep_first, keep_last=keep_last)[2]


def decode(blocks, w_last, h, table, lens, longest, seen, rot):
    """One token of every sequence through the stack: the last norm's output."""
    norm = B.make_norm_desc(h.shape[1], torch.float32)
    _, x = B.qeft_norm_fwd(norm, h, blocks[0].w_attn)
    for i, b in enumerate(blocks):
        h, x = b.decode(norm, h, x, table, lens, longest, seen, rot, blocks[i + 1].w_attn if i + 1 < len(blocks) else w_last)
    return x


def tune_mlp(block, r, y, dh):
    """A block's second half, forward and backward: residual r (fp32) and attention's output y (fp16) in, h' = h + down(silu(gate x) up x) with h = r + y,
    x = norm(h) out; dh is the gradient of h'.  Returns h', the gradients of r, y and the norm's weights, and those of the three layers' weak columns."""
    norm = B.make_norm_desc(r.shape[1], torch.float32)
    h, x = B.qeft_norm_fwd(norm, r, block.w_mlp, y=y)
    g, u = B.qeft_linear_fwd_group([block.gate.desc, block.up.desc], [block.gate.weight, block.up.weight], x)
    s = torch.sigmoid(g.float())
    m = (g.float() * s * u.float()).half()
    out = h + B.qeft_linear_fwd(block.down.desc, block.down.weight, m).float()
    weak = lambda layer, a: a[:, layer.desc.in_features - layer.desc.n_weak:]  # noqa: E731
    dm, dw_down = B.qeft_linear_bwd(block.down.desc, block.down.weight, dh.half(), weak(block.down, m))
    dm = dm.float()
    dg = (dm * u.float() * s * (1 + g.float() * (1 - s))).half()
    du = (dm * g.float() * s).half()
    dx_g, dw_gate = B.qeft_linear_bwd(block.gate.desc, block.gate.weight, dg, weak(block.gate, x))
    dx_u, dw_up = B.qeft_linear_bwd(block.up.desc, block.up.weight, du, weak(block.up, x))
    dr, dy, dw_norm, _, _ = B.qeft_norm_bwd(norm, dx_g + dx_u, h, block.w_mlp, dh=dh, y=y)
    return out, dr, dy, dw_norm, dw_gate, dw_up, dw_down


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--steps", type=int, default=24)
    ap.add_argument("--budget", type=int, default=16)
    args = ap.parse_args()
    if args.steps < 1 or args.budget < 1:
        ap.error("--steps and --budget are 1 or more")
    gen = torch.Generator(device="cuda").manual_seed(0)
    hidden, heads, kv, ffn, page, seqs = 512, 8, 2, 1408, 8, 3
    cols = -(-min(args.steps, args.budget + 1) // page)   # pages for the most tokens that a sequence has before an eviction
    blocks = [Block(hidden, heads, kv, ffn, 8, gen, seqs * cols, page, seqs, cols) for _ in range(2)]
    w_last = torch.ones(hidden, dtype=torch.float16, device="cuda")
    table = torch.randperm(seqs * cols, generator=gen, device="cuda").int().view(seqs, cols)
    rot = rotation(args.steps, hidden // heads)
    lens, seen = torch.zeros(seqs, dtype=torch.int32, device="cuda"), torch.zeros(seqs, dtype=torch.int32, device="cuda")
    longest = 0
    for step in range(args.steps):
        h = torch.randn((seqs, hidden), generator=gen, device="cuda")
        x = decode(blocks, w_last, h, table, lens, longest + 1, seen, rot)
        lens, seen, longest = lens + 1, seen + 1, longest + 1
        if longest > args.budget:
            lens = [b.evict(table, lens, longest, args.budget, seen, 2, args.budget // 4) for b in blocks][0]
            longest = args.budget
    torch.cuda.synchronize()
    print(f"decode: {args.steps} tokens of {seqs} sequences, {lens.tolist()} kept of {seen.tolist()}, output rms {float(x.float().square().mean().sqrt()):.3f}")
    r, dh = torch.randn((64, hidden), generator=gen, device="cuda"), torch.randn((64, hidden), generator=gen, device="cuda") * 0.1
    y = torch.randn((64, hidden), generator=gen, device="cuda").half()
    out = tune_mlp(blocks[0], r, y, dh)
    torch.cuda.synchronize()
    print("fine-tune: gradient norms " + ", ".join(f"{n} {float(t.float().norm()):.3f}" for n, t in zip(("dr", "dy", "norm", "gate", "up", "down"), out[1:])))


if __name__ == "__main__":
    main()
