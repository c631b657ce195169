"""The example's decoder blocks against the same computation in 64 bits, token by token with evictions, and its fine-tuning step against automatic differentiation."""
import importlib.util
import os
import sys

import pytest
import torch

import block_util as U

pytestmark = pytest.mark.gpu
PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "decoder_block.py")
EPS = 1e-5


def load():
    spec = importlib.util.spec_from_file_location("decoder_block", PATH)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def dense(layer):
    """The stored weight in 64 bits."""
    from paper_2410_08661_amd import binding as B
    codes, scales, zeros, weak = B.qeft_unpack(layer.desc, layer.weight)
    g = torch.arange(codes.shape[1], device="cuda") // layer.desc.group_size
    return torch.cat([scales.double()[:, g] * (codes.double() - zeros.double()[:, g]), weak.double()], 1)


def test_decode_with_evictions():
    ex = load()
    gen = torch.Generator(device="cuda").manual_seed(1)
    hidden, heads, kv, ffn, page, seqs, cols, budget = 256, 4, 2, 640, 8, 2, 3, 12
    d = hidden // heads
    blocks = [ex.Block(hidden, heads, kv, ffn, 8, gen, seqs * cols, page, seqs, cols) for _ in range(2)]
    w_last = torch.ones(hidden, dtype=torch.float16, device="cuda")
    table = torch.randperm(seqs * cols, generator=gen, device="cuda").int().view(seqs, cols)
    rot = ex.rotation(64, d)
    W = [{n: dense(getattr(b, n)) for n in ("q", "k", "v", "o", "gate", "up", "down")} for b in blocks]
    # the same in 64 bits: every head's list of (key, value, weight, position)
    held = [[[[] for _ in range(kv)] for _ in range(seqs)] for _ in blocks]
    lens = torch.zeros(seqs, dtype=torch.int32, device="cuda")
    seen, longest, moved = lens.clone(), 0, 0
    for step in range(16):
        h = torch.randn((seqs, hidden), generator=gen, device="cuda")
        got = ex.decode(blocks, w_last, h.clone(), table, lens, longest + 1, seen, rot)
        z = h.double()
        for i, b in enumerate(blocks):
            x = U.unit(z, EPS) * b.w_attn.double()
            q, k, v = (x @ W[i][n].t() for n in ("q", "k", "v"))
            q, k = (U.rotated(t, n, rot, seen, d)[0] for t, n in ((q, heads), (k, kv)))
            a = torch.zeros((seqs, hidden), dtype=torch.float64, device="cuda")
            for s in range(seqs):
                for c in range(kv):
                    mine = held[i][s][c]
                    mine.append([k[s, c * d: (c + 1) * d], v[s, c * d: (c + 1) * d], 0.0, step])
                    K, V = (torch.stack([t[n] for t in mine]) for n in (0, 1))
                    g = heads // kv
                    p = torch.softmax(q[s, c * g * d: (c + 1) * g * d].view(g, d) @ K.t() * d ** -0.5, 1)
                    a[s, c * g * d: (c + 1) * g * d] = (p @ V).view(-1)
                    for t, w in zip(mine, p.sum(0).tolist()):
                        t[2] += w
            z = z + a @ W[i]["o"].t()
            x = U.unit(z, EPS) * b.w_mlp.double()
            z = z + (torch.nn.functional.silu(x @ W[i]["gate"].t()) * (x @ W[i]["up"].t())) @ W[i]["down"].t()
        want = U.unit(z, EPS)
        # some twenty roundings to fp16 on the way, each of a step's values relative to a row of unit size
        assert float((got.double() - want).abs().max()) <= 40 * U.HALF * float(want.abs().max()), step
        lens, seen, longest = lens + 1, seen + 1, longest + 1
        for i, b in enumerate(blocks):
            for s in range(seqs):
                for c in range(kv):
                    n = len(held[i][s][c])
                    have = b.score[s, c, :n].double().cpu()
                    wants = torch.tensor([t[2] for t in held[i][s][c]], dtype=torch.float64)
                    assert float((have - wants).abs().max()) <= 0.02 * (step + 1), (step, i, s, c)
                    assert b.pos[s, c, :n].tolist() == [t[3] for t in held[i][s][c]]
        if longest > budget:
            new = []
            for i, b in enumerate(blocks):
                score, pos = b.score.clone(), b.pos.clone()
                new.append(b.evict(table, lens, longest, budget, seen, 1, 3))
                for s in range(seqs):
                    for c in range(kv):   # by the library's own weights: near ties are its to decide
                        to = U.evicted(score[s, c].tolist(), pos[s, c].tolist(), longest, int(seen[s]), budget, 1, 3)
                        moved += sum(x != y for x, y in enumerate(to))
                        held[i][s][c] = [held[i][s][c][t] for t in to]
            lens, longest = new[0], budget
            assert all(n.tolist() == [budget] * seqs for n in new)
    assert moved > 0


def test_tune_mlp():
    ex = load()
    gen = torch.Generator(device="cuda").manual_seed(2)
    b = ex.Block(256, 4, 4, 640, 8, gen, 4, 8, 1, 4)
    r, dh = torch.randn((40, 256), generator=gen, device="cuda"), torch.randn((40, 256), generator=gen, device="cuda") * 0.1
    y = torch.randn((40, 256), generator=gen, device="cuda").half()
    got = ex.tune_mlp(b, r, y, dh)
    leaves = [t.double().requires_grad_() for t in (r, y, b.w_mlp, dense(b.gate), dense(b.up), dense(b.down))]
    R, Y, w, G, Up, D = leaves
    h = R + Y
    x = U.unit(h, EPS) * w
    out = h + (torch.nn.functional.silu(x @ G.t()) * (x @ Up.t())) @ D.t()
    grads = torch.autograd.grad((out * dh.double()).sum(), leaves)
    want = [out.detach(), *grads[:3], *(g[:, g.shape[1] - 8:] for g in grads[3:])]
    for name, a, e in zip(("out", "dr", "dy", "norm", "gate", "up", "down"), got, want):
        # fp16 products, activations and gradients on the way: relative to the whole, some ten roundings
        assert float((a.double() - e).norm() / e.norm()) <= 12 * U.HALF, name


def test_the_example_runs(monkeypatch, capsys):
    monkeypatch.setattr(sys, "argv", [PATH, "--steps", "20"])
    load().main()
    said = capsys.readouterr().out
    assert "[16, 16, 16] kept of [20, 20, 20]" in said and "fine-tune" in said
