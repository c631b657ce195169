"""qeft_adamw_step and qeft_grad_norm against the formulas in 64 bits; 8-bit states on their grid, with the stated random numbers."""
import math

import pytest
import torch

import ends_util as V
from paper_2410_08661_amd import binding as B

pytestmark = pytest.mark.gpu
SIZES = [1, 128, 7, 1000, 0, 127, 129, 8192, 20000, 2048, 8191, 33, 100003]
KW = dict(beta1=0.9, beta2=0.999, eps=1e-8)


def tensors(sizes, half=False, bits=32, weight=True, master=True, seed=0, std=1e-3):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    new = lambda n, s: torch.randn(n, generator=gen, device="cuda") * s  # noqa: E731
    p = dict(grads=[(new(n, std) * torch.exp(new(n, 1.0))).to(torch.float16 if half else torch.float32) for n in sizes])
    w = [new(n, 0.02) for n in sizes]
    if weight:
        p["weights"] = [x.half() for x in w]
    if master:
        p["masters"] = w
    if bits == 32:
        p.update(m=[new(n, std / 3) for n in sizes], v=[new(n, std).square() for n in sizes])
    else:
        for name, limit in (("m", 0x7F), ("v", 0x7C)):
            p[name], p[name + "_scales"] = [], []
            for n in sizes:
                c = torch.randint(0, limit, (n,), generator=gen, device="cuda")
                if name == "m":
                    c |= torch.randint(0, 2, (n,), generator=gen, device="cuda") << 7
                p[name].append(c.to(torch.uint8))
                b = -(-n // B.QEFT_STATE_BLOCK)
                p[name + "_scales"].append((torch.randint(100, 108, (b,), generator=gen, device="cuda") if name == "m" else torch.randint(80, 90, (b,), generator=gen, device="cuda")).to(torch.uint8))
    return p


def held(p):
    return {k: [t.clone() for t in ts] for k, ts in p.items()}


def check_step(p, before, lr, step, decays, stochastic=False, seed=0, factor=1.0, **kw):
    """Every tensor of p after the step from `before`."""
    first = 0
    bits = 8 if "m_scales" in p else 32
    for i, g in enumerate(before["grads"]):
        n = g.numel()
        old = {name: before[name][i].double() if bits == 32 else V.state_values(before[name][i], before[name + "_scales"][i], name, n) for name in ("m", "v")}
        w = before["masters"][i] if "masters" in p else before["weights"][i]
        (new, ew), (m, em), (v, ev) = V.adamw(w, g, old["m"], old["v"], lr, step, decays[i], kw["beta1"], kw["beta2"], kw["eps"], factor)
        dice = V.dice(first, n, step, seed)
        first += -(-n // B.QEFT_STATE_BLOCK) * B.QEFT_STATE_BLOCK
        if "masters" in p:
            V.close("master", p["masters"][i], new, ew, V.U)
            if "weights" in p:
                assert torch.equal(p["weights"][i], p["masters"][i].half())
        elif not stochastic:
            V.close("weight", p["weights"][i], new, ew, V.HALF)
        else:
            u = ((dice * 0x5C3C9CCD) % (1 << 32) >> 19).double() / 8192
            got = p["weights"][i].double() * new.sign()
            ok = V.rounded_within(got, new.abs(), ew, u, 2.0 ** -13, 10, 2.0 ** -14) | (new.abs() < ew)
            bad = (~ok).nonzero()[:3, 0]
            assert not len(bad), (i, bad.tolist(), got[bad].tolist(), new[bad].tolist(), ew[bad].tolist(), u[bad].tolist())
        if bits == 32:
            V.close("m", p["m"][i], m, em, V.U)
            V.close("v", p["v"][i], v, ev, V.U)
            continue
        for name, x, e, mant, least, top, u in (("m", m, em, 3, 2.0 ** -6, 7, dice >> 16), ("v", v, ev, 2, 2.0 ** -14, 14, dice % 65536)):
            blocks = -(-n // B.QEFT_STATE_BLOCK)
            flat = torch.zeros(blocks * B.QEFT_STATE_BLOCK, dtype=torch.float64, device="cuda")
            flat[:n] = x.abs()
            most = flat.view(-1, B.QEFT_STATE_BLOCK).amax(1)
            power = torch.where(most > 0, torch.floor(torch.log2(most)) - top, -127.0).clamp(min=-127)
            sure = (most * (1 + 1e-6)).log2().floor() == (most * (1 - 1e-6)).log2().floor()      # (not within a rounding of a power of two)
            assert torch.equal(p[name + "_scales"][i].double()[sure] - 127, power[sure]) and int((~sure).sum()) <= blocks // 100, (name, i)
            scale = torch.exp2(p[name + "_scales"][i].double() - 127).repeat_interleave(B.QEFT_STATE_BLOCK)[:n]
            got = V.state_values(p[name][i], p[name + "_scales"][i], name, n) / scale
            got = got * torch.where(x < 0, -1.0, 1.0) if name == "m" else got
            a = x.abs() / scale
            ok = V.rounded_within(got, a, e / scale, u.double() / 65536, 0.0, mant, least)
            if name == "v":
                ok |= (got == 2.0 ** -16) & (a < 2.0 ** -15)
                assert bool((got > 0)[x > 0].all())
            bad = (~ok).nonzero()[:3, 0]
            assert not len(bad), (name, i, bad.tolist(), got[bad].tolist(), a[bad].tolist(), (e / scale)[bad].tolist(), u[bad].tolist())


@pytest.mark.parametrize("half", [False, True])
@pytest.mark.parametrize("weight,master", [(True, True), (True, False), (False, True)])
@pytest.mark.parametrize("bits", [32, 8])
def test_steps(bits, weight, master, half):
    p = tensors(SIZES, half, bits, weight, master)
    decays = [0.1 * (i % 3) for i in range(len(SIZES))]
    plan = B.TensorList(decay=decays, **p)
    for step, lr, stochastic, seed in ((1, 1e-3, False, 0), (2, 2e-2, True, 7), (1000, 1e-4, True, (1 << 40) + 3)):
        before = held(p)
        B.qeft_adamw_step(plan, lr, step, stochastic=stochastic, seed=seed, **KW)
        check_step(p, before, lr, step, decays, stochastic and not master, seed, **KW)
        assert all(torch.equal(a, b) for a, b in zip(p["grads"], before["grads"]))


def test_other_betas_and_eps():
    for kw in (dict(beta1=0.0, beta2=0.0, eps=1e-3), dict(beta1=0.95, beta2=0.9999, eps=1e-15), dict(beta1=0.5, beta2=0.5, eps=1.0)):
        p = tensors(SIZES, bits=32)
        before = held(p)
        B.qeft_adamw_step(B.TensorList(**p), 0.1, 3, **kw)
        check_step(p, before, 0.1, 3, [0.0] * len(SIZES), **kw)


@pytest.mark.parametrize("bits", [32, 8])
def test_lr_step_and_factor_on_the_device(bits):
    p, q = tensors(SIZES, bits=bits, master=False), tensors(SIZES, bits=bits, master=False)
    a, b = B.TensorList(decay=0.1, **p), B.TensorList(decay=0.1, **q)
    lr, step, factor = torch.tensor([3e-3], device="cuda"), torch.tensor([5], dtype=torch.int32, device="cuda"), torch.tensor([0.25], device="cuda")
    before = held(p)
    B.qeft_adamw_step(a, lr, step, factor=factor, stochastic=True, seed=3, **KW)
    check_step(p, before, float(lr), 5, [0.1] * len(SIZES), True, 3, 0.25, **KW)
    B.qeft_adamw_step(b, float(lr), 5, factor=factor, stochastic=True, seed=3, **KW)
    for name in ("m", "v"):
        for x, y in zip(p[name], q[name]):
            assert torch.equal(x, y)
    for bad in (math.nan, math.inf, -math.inf):
        before = held(p)
        B.qeft_adamw_step(a, lr, step, factor=torch.tensor([bad], device="cuda"), **KW)
        assert all(torch.equal(x, y) for k in p for x, y in zip(p[k], before[k]))
    step.fill_(-3)                            # counts as 1
    before = held(p)
    B.qeft_adamw_step(a, lr, step, stochastic=True, **KW)
    check_step(p, before, float(lr), 1, [0.1] * len(SIZES), True, 0, **KW)


def test_zero_states_and_gradients():
    w = [torch.randn(300, device="cuda").half(), torch.randn(128, device="cuda").half()]
    g = [torch.zeros(300, device="cuda"), torch.zeros(128, device="cuda")]
    for bits in (8, 32):
        s = B.make_adamw_states(w, bits)
        before = [t.clone() for t in w]
        B.qeft_adamw_step(B.TensorList(g, weights=w, **s), 0.1, 1)
        assert all(torch.equal(a, b) for a, b in zip(w, before)) and not any(bool(t.any()) for ts in s.values() for t in ts)


def test_8_bit_states_are_rounded_by_16_bits():
    """From moments that fp32 holds exactly (halves of fp16 gradients and of their squares), every code is the definition's."""
    n, step, seed = 1 << 21, 3, 11
    gen = torch.Generator(device="cuda").manual_seed(5)
    g = (torch.randn(n, generator=gen, device="cuda") * torch.exp2(torch.randint(-8, 3, (n,), generator=gen, device="cuda").float())).half()
    p = dict(grads=[g], weights=[torch.zeros(n, dtype=torch.float16, device="cuda")])
    p["m"], p["v"] = ([torch.zeros(n, dtype=torch.uint8, device="cuda")] for _ in range(2))
    p["m_scales"], p["v_scales"] = ([torch.zeros(n // B.QEFT_STATE_BLOCK, dtype=torch.uint8, device="cuda")] for _ in range(2))
    B.qeft_adamw_step(B.TensorList(**p), 1e-3, step, beta1=0.5, beta2=0.5, seed=seed)
    dice, g = V.dice(0, n, step, seed), g.double()
    for name, x, mant, least, u in (("m", 0.5 * g, 3, 2.0 ** -6, dice >> 16), ("v", 0.5 * g * g, 2, 2.0 ** -14, dice % 65536)):
        scale = torch.exp2(p[name + "_scales"][0].double() - 127).repeat_interleave(B.QEFT_STATE_BLOCK)
        want = V.on_grid(x.abs() / scale, u.double() / 65536, mant, least)
        if name == "v":
            want = torch.where((want == 0) & (x > 0), 2.0 ** -16, want)
        got = V.state_values(p[name][0], p[name + "_scales"][0], name, n) / scale
        assert torch.equal(got.abs(), want) and bool((got * x >= 0).all())


def test_8_bit_states_keep_the_mean():
    """1000 steps of a constant gradient: second moments move by a thousandth a step; the mean over 64 Ki values follows 1 - beta2^t."""
    n, steps = 1 << 16, 1000
    g = [torch.full((n,), 1e-3, device="cuda")]
    s = B.make_adamw_states(g, 8)
    m = [torch.zeros(n, device="cuda")]
    plan = B.TensorList(g, masters=m, **s)
    for t in range(1, steps + 1):
        B.qeft_adamw_step(plan, 0.0, t, seed=11, **KW)
    v = V.state_values(s["v"][0], s["v_scales"][0], "v", n).mean()
    want = 1e-6 * (1 - 0.999 ** steps)
    # a value's variance: a step of a code is at most a quarter of it, taken with probability p = change / step: p step^2 = change * step, 1e-3 * 1/4 of v^2 a step at
    # most, half of it left over the memory of 1000 steps: 0.125 v^2; the mean of n: v sqrt(0.125 / n), seven of these
    assert abs(float(v) - want) < 7 * want * math.sqrt(0.125 / n), (float(v), want)
    first = V.state_values(s["m"][0], s["m_scales"][0], "m", n).mean()
    # (change a tenth, step an eighth, memory of ten steps: 1/16)
    assert abs(float(first) - 1e-3) < 7 * 1e-3 * math.sqrt(0.0625 / n)


def test_16_bit_weights_keep_the_mean():
    """An update of a hundredth of a weight's step arrives in the mean."""
    n = 1 << 16
    w = [torch.ones(n, dtype=torch.float16, device="cuda")]
    g = [torch.full((n,), -1.0, device="cuda")]
    plan = B.TensorList(g, weights=w, **B.make_adamw_states(w))
    for t in range(1, 101):
        B.qeft_adamw_step(plan, 2.0 ** -10 / 100, t, stochastic=True, seed=5, **KW)
    moved = float((w[0].double() - 1).mean()) * 1024
    # 100 steps of 0.01 +- sqrt(0.01): 1 step in the mean, seven deviations of sqrt(1 / n) and the 13 bits' truncation (2^-13 of a step each)
    assert abs(moved - 1) < 7 / math.sqrt(n) + 100 * 2.0 ** -13, moved
    w[0].fill_(1)
    B.qeft_adamw_step(plan, 2.0 ** -10 / 100, 101, **KW)
    assert bool((w[0] == 1).all())            # to nearest it does not


def test_values_at_the_ends_of_fp16_and_not_finite_gradients():
    w = [torch.tensor([65504.0, -65504.0, 6e-8, -6e-8, 3e-5, 0.0, -0.0, 1.0], device="cuda").half()]
    for stochastic in (False, True):
        x = [w[0].clone()]
        B.qeft_adamw_step(B.TensorList([torch.zeros(8, device="cuda")], weights=x, **B.make_adamw_states(w)), 0.1, 1, stochastic=stochastic)
        assert torch.equal(x[0], w[0])        # values that fp16 has stay what they are
        big = [torch.full((8,), 65504.0, device="cuda").half()]
        B.qeft_adamw_step(B.TensorList([torch.full((8,), -1.0, device="cuda")], weights=big, **B.make_adamw_states(big)), 1e4, 1, stochastic=stochastic)
        assert bool((big[0] == math.inf).all())
    for bits in (8, 32):
        g = [torch.ones(300, device="cuda") * 0.01]
        g[0][130], g[0][200] = math.inf, math.nan
        x = [torch.ones(300, device="cuda")]
        s = B.make_adamw_states(x, bits)
        B.qeft_adamw_step(B.TensorList(g, masters=x, **s), 0.1, 1)
        values = {k: V.state_values(s[k][0], s[k + "_scales"][0], k, 300) if bits == 8 else s[k][0] for k in ("m", "v")}
        for t in values.values():
            assert bool(t[:128].isfinite().all()) and bool(t[256:].isfinite().all()) and not bool(t[130].isfinite()) and bool(t[200].isnan())
            if bits == 8:
                assert bool(t[128:256].isnan().all())
        assert bool(x[0][:128].isfinite().all()) and bool(x[0][131:200].isfinite().all()) and bool(x[0][200].isnan())


@pytest.mark.parametrize("half", [False, True])
@pytest.mark.parametrize("sizes", [[1], [5, 0, 3], SIZES, [9_000_001, 17], []])
def test_norm(sizes, half):
    p = tensors(sizes, half)
    plan = B.TensorList(p["grads"]) if sizes else B.TensorList([])
    true = math.sqrt(sum(float(g.double().square().sum()) for g in p["grads"]))
    steps = torch.tensor([4], dtype=torch.int32, device="cuda")
    for scale, most in ((1.0, math.inf), (0.5, 1e-3), (2.0, 1e9)):
        out = B.qeft_grad_norm(plan, max_norm=most, scale=scale, steps=steps).double()
        # fp64 sums: what is left are the roundings of the results
        assert abs(float(out[0]) - scale * true) <= 2 * V.U * scale * true
        want = scale * min(1.0, most / (scale * true)) if true else scale
        assert abs(float(out[1]) - want) <= 2 * V.U * want
    assert int(steps) == 7


def test_norm_of_large_small_and_not_finite_gradients():
    steps = torch.zeros(1, dtype=torch.int32, device="cuda")
    for x in (1e30, 1e-30):
        out = B.qeft_grad_norm(B.TensorList([torch.full((400,), x, device="cuda")]), steps=steps)
        assert abs(float(out[0]) - 20 * x) < 1e-6 * 20 * x
    for x in (math.inf, math.nan, 3e38):      # (a norm beyond fp32 is not finite either)
        g = torch.full((400,), 3e38 if x == 3e38 else 1.0, device="cuda")
        g[399] = x
        out = B.qeft_grad_norm(B.TensorList([g]), max_norm=1.0, steps=steps)
        assert not math.isfinite(float(out[0])) and math.isnan(float(out[1]))
    assert int(steps) == 2


def test_a_list_without_values():
    for sizes in ([], [0, 0]):
        p = tensors(sizes) if sizes else dict(grads=[])
        B.qeft_adamw_step(B.TensorList(**p), 0.1, 1)


def test_clipped_steps_from_a_graph():
    """Norm, factor, count and step replayed, the learning rate changed between; a gradient that is not finite leaves a step out."""
    for bits in (32, 8):
        p, q = (tensors(SIZES, bits=bits, master=bits == 32) for _ in range(2))
        a, b = B.TensorList(decay=0.1, **p), B.TensorList(decay=0.1, **q)
        lr, steps, norm = torch.tensor([1e-3], device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda"), torch.zeros(2, device="cuda")
        ws = torch.empty(B.qeft_grad_norm_workspace(a), dtype=torch.uint8, device="cuda")
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
            B.qeft_grad_norm(a, max_norm=0.05, out=norm, steps=steps, ws=ws)
            B.qeft_adamw_step(a, lr, steps, factor=norm[1:], stochastic=True, seed=9)
        assert int(steps) == 0
        count = 0
        for i in range(5):
            lr.fill_(1e-3 / (i + 1))
            for x, y in zip(p["grads"], q["grads"]):
                x.mul_(1.5)
                y.copy_(x)
            if i == 2:
                p["grads"][3][5] = math.nan
            ws.fill_(255)
            graph.replay()
            torch.cuda.synchronize()
            if i == 2:
                p["grads"][3][5] = 1.0
                assert math.isnan(float(norm[1])) and int(steps) == count
                q["grads"][3][5] = 1.0
                continue
            count += 1
            assert int(steps) == count
            eager = B.qeft_grad_norm(b, max_norm=0.05)
            assert torch.equal(eager, norm)
            at = torch.tensor([count], dtype=torch.int32, device="cuda")
            B.qeft_adamw_step(b, lr, at, factor=eager[1:], stochastic=True, seed=9)
            for k in p:
                for x, y in zip(p[k], q[k]):
                    assert torch.equal(x, y), (bits, i, k)


def test_offsets_beyond_32_bits():
    n = (1 << 31) + 1000
    w, g = torch.zeros(n, dtype=torch.float16, device="cuda"), torch.zeros(n, dtype=torch.float16, device="cuda")
    s = B.make_adamw_states([w], 8)
    gen = torch.Generator(device="cuda").manual_seed(1)
    k = 1000
    w[-k:], g[-k:] = torch.randn(k, generator=gen, device="cuda").half(), torch.randn(k, generator=gen, device="cuda").half()
    before = dict(weights=[w[-k:].clone()], grads=[g[-k:].clone()])
    B.qeft_adamw_step(B.TensorList([g], weights=[w], **s), 0.01, 1, **KW)
    (new, ew), (m, _), _ = V.adamw(before["weights"][0], before["grads"][0], *[torch.zeros(k, dtype=torch.float64, device="cuda")] * 2, 0.01, 1, 0.0, **KW)
    V.close("weight", w[-k:], new, ew, V.HALF)
    got = V.state_values(s["m"][0][-k:], s["m_scales"][0][-8:], "m", k)
    blocks = torch.arange(k, device="cuda") // B.QEFT_STATE_BLOCK
    assert bool(((got - m).abs() <= 2.0 ** -3 * m.abs() + 2.0 ** -14 * torch.stack([m[blocks == i].abs().amax() for i in range(8)])[blocks]).all())
    assert not bool(s["m"][0][:-k].any())
    norm = B.qeft_grad_norm(B.TensorList([g]))
    want = float(before["grads"][0].double().norm())
    assert abs(float(norm[0]) - want) <= 2 * V.U * want


def test_calls_without_the_native_module(monkeypatch):
    for number, seed in ((lambda x, t: x, 5), (lambda x, t: torch.tensor([x], dtype=t, device="cuda"), 2 ** 64 - 1)):
        results = []
        for native in (True, False):
            p = tensors(SIZES, True, 8, master=False)
            plan = B.TensorList(decay=0.1, **p)
            steps = torch.zeros(1, dtype=torch.int32, device="cuda")
            with monkeypatch.context() as mp:
                if not native:
                    mp.setattr(B, "_native", V.NONE)
                norm = B.qeft_grad_norm(plan, max_norm=0.01, scale=0.5, steps=steps)
                B.qeft_adamw_step(plan, number(1e-3, torch.float32), number(4, torch.int32), 0.8, 0.99, 1e-7, factor=norm[1:], stochastic=True, seed=seed)
            results.append([norm, steps, *(t for ts in p.values() for t in ts)])
        for a, b in zip(*results):
            assert torch.equal(a, b)


def test_arguments_that_are_refused():
    p = tensors([100, 5])
    plan = B.TensorList(**p)
    one = torch.ones(1, device="cuda")
    for kw in (dict(lr=0.1, step=0), dict(lr=float("nan"), step=1), dict(lr=0.1, step=one), dict(lr=one.half(), step=1), dict(lr=0.1, step=1, factor=one.double()),
               dict(lr=0.1, step=1, factor=one.cpu()), dict(lr=0.1, step=1, factor=one[:0]), dict(lr=0.1, step=1, beta1=1.0), dict(lr=0.1, step=1, eps=0.0)):
        before = held(p)
        with pytest.raises(B.QeftError):
            B.qeft_adamw_step(plan, **kw)
        assert all(torch.equal(a, b) for k in p for a, b in zip(p[k], before[k]))
    for kw in (dict(max_norm=0.0), dict(scale=0.0), dict(out=one), dict(steps=one), dict(ws=torch.empty(0, dtype=torch.uint8, device="cuda"))):
        with pytest.raises(B.QeftError):
            B.qeft_grad_norm(plan, **kw)
    for change in (dict(weights=[w.float() for w in p["weights"]]), dict(m=[t[:3] for t in p["m"]]), dict(v=p["m"]), dict(grads=[t.repeat(2)[::2] for t in p["grads"]]),
                   dict(weights=None, masters=None), dict(m_scales=p["m"]), dict(masters=[p["masters"][0], p["masters"][0][:5]])):
        with pytest.raises(B.QeftError):
            B.TensorList(**{**p, **change})
    with pytest.raises(B.QeftError):
        B.qeft_adamw_step(B.TensorList(p["grads"]), 0.1, 1)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("half", [False, True])
def test_nothing_beside_the_tensors_is_touched(bits, half):
    """Tensors of odd sizes in larger buffers, sentinels all round."""
    sizes, gap = [1, 5, 127, 130, 8192, 8193, 2049, 4000], 128
    p = tensors(sizes, half, bits)
    buffers, views = {}, {}
    for k, ts in p.items():
        room = [-(-t.numel() // 16) * 16 + gap for t in ts]
        buffers[k] = torch.full((sum(room) + gap,), 77, dtype=ts[0].dtype, device="cuda")
        at, views[k] = gap, []
        for t, r in zip(ts, room):
            views[k].append(buffers[k][at: at + t.numel()].copy_(t))
            at += r
    held_all = {k: b.clone() for k, b in buffers.items()}
    B.qeft_adamw_step(B.TensorList(decay=0.1, **p), 1e-3, 3, seed=1)
    B.qeft_adamw_step(B.TensorList(decay=0.1, **views), 1e-3, 3, seed=1)
    for k in p:
        inside = torch.zeros_like(buffers[k], dtype=torch.bool)
        for t, v in zip(p[k], views[k]):
            assert torch.equal(t, v), k
            first = (v.data_ptr() - buffers[k].data_ptr()) // v.element_size()
            inside[first: first + v.numel()] = True
        assert torch.equal(buffers[k][~inside], held_all[k][~inside]), k
