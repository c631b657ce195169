"""Whole fine-tuning steps of the example's decoder - norms of heads and rotation, loss, their gradients, the gradients' norm and the optimizer beside the
library's other calls - against the same in 64 bits by automatic differentiation."""
import math

import pytest
import torch

import block_util as U
import ends_util as V
from test_gpu_block_example import dense, load

pytestmark = pytest.mark.gpu


def make(ex, gen, head_norms, bits=8):
    blocks = [ex.Block(256, 4, 2, 640, 8, gen, 1, 8, 1, 1, head_norms=head_norms) for _ in range(2)]
    w_last = (1 + 0.1 * torch.randn(256, generator=gen, device="cuda")).half()
    return ex.Tuner(blocks, w_last, ex.Linear(512, 256, 8, gen), bits=bits)


def reference(ex, tuner, h, token, rot):
    """The loss and its gradients by every trained tensor, in 64 bits."""
    leaves = {}
    for name, w in tuner.weights.items():
        if w.dim() == 1:
            leaves[name] = w.double().requires_grad_()
    layer = {("head", "weak"): tuner.head, **{(i, n): getattr(b, n) for i, b in enumerate(tuner.blocks) for n in tuner.LAYERS}}
    leaves.update({name: dense(x).requires_grad_() for name, x in layer.items()})
    n = h.shape[0]
    pos = torch.arange(n, device="cuda")
    z = h.double()
    for i, b in enumerate(tuner.blocks):
        W = lambda name: leaves[i, name]  # noqa: E731
        x = U.unit(z, 1e-5) * W("w_attn")
        q, k, v = (x @ W(name).t() for name in ("q", "k", "v"))
        q, k = (V.heads_forward(t, heads, leaves.get((i, w)), 1e-6, rot, pos, b.d)[0].view(n, heads, b.d).transpose(0, 1) for t, heads, w in ((q, b.heads, "w_q"), (k, b.kv, "w_k")))
        v = v.view(n, b.kv, b.d).transpose(0, 1)
        k, v = (t.repeat_interleave(b.heads // b.kv, 0) for t in (k, v))
        s = (q @ k.transpose(1, 2) * b.d ** -0.5).masked_fill(torch.ones((n, n), dtype=torch.bool, device="cuda").triu(1), -math.inf)
        z = z + (torch.softmax(s, -1) @ v).transpose(0, 1).reshape(n, -1) @ W("o").t()
        x = U.unit(z, 1e-5) * W("w_mlp")
        z = z + (torch.nn.functional.silu(x @ W("gate").t()) * (x @ W("up").t())) @ W("down").t()
    lp = torch.log_softmax((U.unit(z, 1e-5) * leaves["head", "norm"]) @ leaves["head", "weak"].t(), -1)
    has = token >= 0
    loss = -lp.gather(1, token.clamp(min=0).long()[:, None])[has].mean()
    grads = dict(zip(leaves, torch.autograd.grad(loss, list(leaves.values()))))
    return loss.detach(), {name: g[:, -8:] if g.dim() == 2 else g for name, g in grads.items()}


@pytest.mark.parametrize("head_norms", [True, False])
def test_a_step_against_automatic_differentiation(head_norms):
    ex = load()
    gen = torch.Generator(device="cuda").manual_seed(3)
    t = make(ex, gen, head_norms, 32)
    h = torch.randn((48, 256), generator=gen, device="cuda")
    token = torch.randint(0, 512, (48,), generator=gen, device="cuda").int()
    token[:10] = -1
    rot = ex.rotation(48, 64)
    want, grads = reference(ex, t, h, token, rot)
    before = {n: w.clone() for n, w in t.weights.items()}
    loss, norm = t.step(h, token, rot, 1e-2)
    # forward: two blocks of some ten fp16 roundings each before the logits, which are of the order of one: the mean loss moves by less than a logit
    assert abs(float(loss - want)) <= 40 * U.HALF
    total = 0.0
    for name, g in grads.items():
        got = t.grads[name].double() / t.loss_scale
        total += float(g.square().sum())
        # fp16 activations and gradients on the way there and back, some forty roundings in a chain: relative to the whole
        assert float((got - g).norm() / g.norm()) <= 40 * U.HALF, name
    mine = math.sqrt(sum(float((g.double() / t.loss_scale).square().sum()) for g in t.grads.values()))
    assert abs(float(norm[0]) - mine) <= 4 * V.U * mine and abs(mine - math.sqrt(total)) <= 40 * U.HALF * math.sqrt(total)
    assert abs(float(norm[1]) * t.loss_scale - min(1.0, 1 / mine)) <= 4 * V.U
    # the step itself, from the gradients as they are: moments of zero before it
    for name, w in before.items():
        zero = torch.zeros(w.numel(), dtype=torch.float64, device="cuda")
        (new, bound), _, _ = V.adamw(w.reshape(-1), t.grads[name].reshape(-1), zero, zero, 1e-2, 1, 0.1 if w.dim() == 2 else 0.0, 0.9, 0.999, 1e-8, float(norm[1]))
        step = torch.exp2(torch.floor(torch.log2(new.abs().clamp(min=2.0 ** -14))) - 10)      # stochastic: to one of two neighbours
        assert bool(((t.weights[name].reshape(-1).double() - new).abs() <= bound + step * (1 + 1e-9)).all()), name
        assert not torch.equal(t.weights[name], w)
    assert int(t.steps) == 1


def test_steps_repeat_and_leave_out_what_is_not_finite():
    ex = load()
    runs = []
    for _ in range(2):
        gen = torch.Generator(device="cuda").manual_seed(4)
        t = make(ex, gen, True)
        h = torch.randn((33, 256), generator=gen, device="cuda")
        token = torch.randint(0, 512, (33,), generator=gen, device="cuda").int()
        rot = ex.rotation(33, 64)
        losses = [t.step(h, token, rot, 1e-2, seed=i)[0] for i in range(3)]
        held = {n: w.clone() for n, w in t.weights.items()}
        states = [x.clone() for k in ("m", "v", "m_scale", "v_scale") for x in t.plan.tensors[k]]
        bad = h.clone()
        bad[5, 7] = math.inf
        t.step(bad, token, rot, 1e-2)
        assert int(t.steps) == 3 and math.isnan(float(t.norm[1]))
        assert all(torch.equal(held[n], w) for n, w in t.weights.items())
        assert all(torch.equal(a, b) for a, b in zip(states, [x for k in ("m", "v", "m_scale", "v_scale") for x in t.plan.tensors[k]]))
        losses.append(t.step(h, token, rot, 1e-2, seed=3)[0])
        runs.append([*losses, *t.weights.values()])
    for a, b in zip(*runs):
        assert torch.equal(a, b)


def test_decode_with_head_norms():
    """Two tokens of a sequence through a block whose heads are normed, against the same in 64 bits."""
    ex = load()
    gen = torch.Generator(device="cuda").manual_seed(5)
    b = ex.Block(256, 4, 2, 640, 8, gen, 4, 8, 2, 2, head_norms=True)
    w_last, rot = torch.ones(256, dtype=torch.float16, device="cuda"), ex.rotation(8, 64)
    table = torch.arange(4, device="cuda").int().view(2, 2)
    W = {n: dense(getattr(b, n)) for n in ("q", "k", "v", "o", "gate", "up", "down")}
    kept = []
    for t in range(3):
        lens = torch.full((2,), t, dtype=torch.int32, device="cuda")
        h = torch.randn((2, 256), generator=gen, device="cuda")
        got = ex.decode([b], w_last, h.clone(), table, lens, t + 1, lens, rot)
        x = U.unit(h.double(), 1e-5) * b.w_attn.double()
        q, k, v = (x @ W[n].t() for n in ("q", "k", "v"))
        q, k = (V.heads_forward(a, n, w, 1e-6, rot, lens, 64)[0].view(2, n, 64) for a, n, w in ((q, 4, b.w_q), (k, 2, b.w_k)))
        kept.append((k, v.view(2, 2, 64)))
        K, Vs = (torch.stack([r[i] for r in kept], 2).repeat_interleave(2, 1) for i in (0, 1))
        p = torch.softmax((q[:, :, None] * K).sum(-1) * 64 ** -0.5, -1)
        z = h.double() + (p[..., None] * Vs).sum(2).reshape(2, -1) @ W["o"].t()
        x = U.unit(z, 1e-5) * b.w_mlp.double()
        z = z + (torch.nn.functional.silu(x @ W["gate"].t()) * (x @ W["up"].t())) @ W["down"].t()
        want = U.unit(z, 1e-5)
        assert float((got.double() - want).abs().max()) <= 40 * U.HALF * float(want.abs().max()), t


