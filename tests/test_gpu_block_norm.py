"""qeft_norm_fwd and qeft_norm_bwd against the formulas in 64 bits, and against differences of the forward."""
import pytest
import torch

import block_util as U
from paper_2410_08661_amd import binding as B

pytestmark = pytest.mark.gpu
GATES = {"none": B.QEFT_GATE_NONE, "channel": B.QEFT_GATE_CHANNEL, "token": B.QEFT_GATE_TOKEN}
EPS = 1e-5


def padded(m, n, dtype, gen, std=1.0, pad=8):
    """[m][n] with a pitch of its own."""
    ld = (n + 7) // 8 * 8 + pad
    return (torch.randn((m, ld), generator=gen, device="cuda") * std).to(dtype)[:, :n]


def inputs(m, n, f32, post, gate, seed=0):
    gen = torch.Generator(device="cuda").manual_seed(seed + 17 * n + m)
    t = torch.float32 if f32 else torch.float16
    w = [(1 + 0.2 * torch.randn(n, generator=gen, device="cuda")).half() for _ in range(2)]
    g = None
    if gate == "token":
        g = padded(m, n, torch.float16, gen)
    elif gate == "channel":
        g = torch.randn(n, generator=gen, device="cuda").half()
    return dict(y=padded(m, n, torch.float16, gen, 0.5), r=padded(m, n, t, gen, 2.0), w_pre=w[0], w_post=w[1] if post else None, gate=g,
                dx=padded(m, n, torch.float16, gen, 0.1, 0), dh=padded(m, n, t, gen, 0.2, 16))


def check_fwd(m, n, f32, post, gate, scale=0.7):
    i = inputs(m, n, f32, post, gate)
    t = i["r"].dtype
    desc = B.make_norm_desc(n, t, GATES[gate], scale, EPS)
    h, x = B.qeft_norm_fwd(desc, i["r"], i["w_pre"], y=i["y"], w_post=i["w_post"], gate=i["gate"])
    want, _ = U.norm_forward(i["r"], i["y"], i["w_pre"], i["w_post"], i["gate"], scale, EPS)
    R = U.sums_rounding(n)
    size = i["r"].double().abs() + (want - i["r"].double()).abs()
    U.close("h", h, want, 2 * R * size, U.ROUNDING[t])
    _, want = U.norm_forward(h, None, i["w_pre"], None, None, 1.0, EPS)          # x is the norm of h as stored
    U.close("x", x, want, 2 * R * want.abs(), U.HALF)
    # in place, without h, and the norm alone
    r2, y2 = i["r"].clone(), i["y"].clone()
    ld = (n + 7) // 8 * 8
    r2 = torch.empty((m, ld), dtype=t, device="cuda")[:, :n].copy_(i["r"])
    y2 = torch.empty((m, ld), dtype=torch.float16, device="cuda")[:, :n].copy_(i["y"])
    h2, x2 = B.qeft_norm_fwd(desc, r2, i["w_pre"], y=y2, w_post=i["w_post"], gate=i["gate"], h=r2, x=y2)
    assert torch.equal(h2, h) and torch.equal(x2, x) and h2 is r2 and x2 is y2
    h3, x3 = B.qeft_norm_fwd(desc, h, i["w_pre"])
    assert h3 is h and torch.equal(x3, x)


@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("post,gate", [(False, "none"), (True, "channel"), (True, "token"), (False, "token")])
@pytest.mark.parametrize("m,n", [(1, 1), (3, 7), (5, 64), (9, 100), (300, 512), (2, 520), (1, 4096), (33, 5120), (3, 8191), (4, 8200), (2, 16384), (2, 30000), (2, 33001)])
def test_forward(m, n, f32, post, gate):
    check_fwd(m, n, f32, post, gate)


def check_bwd(m, n, f32, post, gate, scale=0.7):
    i = inputs(m, n, f32, post, gate)
    t = i["r"].dtype
    desc = B.make_norm_desc(n, t, GATES[gate], scale, EPS)
    h = i["r"]
    kw = dict(dh=i["dh"], y=i["y"], w_post=i["w_post"], gate=i["gate"])
    got = dict(zip(("dr", "dy", "dw_pre", "dw_post", "dgate"), B.qeft_norm_bwd(desc, i["dx"], h, i["w_pre"], **kw)))
    want = U.norm_backward(i["dx"], i["dh"], h, i["y"], i["w_pre"], i["w_post"], i["gate"], scale, EPS, gate == "channel")
    assert {k for k, v in got.items() if v is not None} == set(want)
    for k, (w, bound) in want.items():
        U.close(k, got[k], w, bound, U.ROUNDING[got[k].dtype])
    again = dict(zip(got, B.qeft_norm_bwd(desc, i["dx"], h, i["w_pre"], **kw)))
    for k in want:
        assert torch.equal(again[k], got[k]), k                        # the order of the sums is fixed
    # the sums added to what is there, twice
    sums = {k: got[k].clone() for k in want if k in ("dw_pre", "dw_post") or (k == "dgate" and gate == "channel")}
    B.qeft_norm_bwd(desc, i["dx"], h, i["w_pre"], accumulate=True, **kw, **sums)
    for k, v in sums.items():
        assert torch.equal(v, 2 * got[k]), k
    return i, desc, got


@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("post,gate", [(False, "none"), (True, "none"), (True, "channel"), (True, "token"), (False, "channel"), (False, "token")])
@pytest.mark.parametrize("m,n", [(1, 8), (3, 7), (70, 64), (1000, 100), (300, 520), (17, 4096), (333, 5120), (3, 8191), (600, 8192), (5, 8200), (300, 16384), (70, 16400)])
def test_backward(m, n, f32, post, gate):
    check_bwd(m, n, f32, post, gate)


@pytest.mark.parametrize("n", [136, 5000, 20000])
def test_backward_in_place_and_in_parts(n):
    i, desc, got = check_bwd(40, n, True, True, "token")
    ld = (n + 7) // 8 * 8
    dh = torch.empty((40, ld), device="cuda")[:, :n].copy_(i["dh"])
    dx = torch.empty((40, ld), dtype=torch.float16, device="cuda")[:, :n].copy_(i["dx"])
    dr, dy, dw, dwp, dg = B.qeft_norm_bwd(desc, dx, i["r"], i["w_pre"], dh=dh, y=i["y"], w_post=i["w_post"], gate=i["gate"], dr=dh, dy=dx)
    assert dr is dh and dy is dx
    for k, v in zip(("dr", "dy", "dw_pre", "dw_post", "dgate"), (dr, dy, dw, dwp, dg)):
        assert torch.equal(v, got[k]), k
    # only some of them, without dh, without a block
    some = B.qeft_norm_bwd(desc, i["dx"], i["r"], i["w_pre"], dh=i["dh"], y=i["y"], w_post=i["w_post"], gate=i["gate"], dr=False, dw_pre=False, dgate=False)
    assert some[0] is None and some[2] is None and some[4] is None and torch.equal(some[1], got["dy"]) and torch.equal(some[3], got["dw_post"])
    alone = B.qeft_norm_bwd(desc, i["dx"], i["r"], i["w_pre"])
    want = U.norm_backward(i["dx"], None, i["r"], None, i["w_pre"], None, None, 1.0, EPS, False)
    assert alone[1] is None and alone[3] is None and alone[4] is None
    U.close("dr", alone[0], *want["dr"], U.U)
    U.close("dw_pre", alone[2], *want["dw_pre"], U.U)


def test_backward_against_differences():
    """Directional derivatives of the forward in 64 bits (a step each way), along a random direction of every input."""
    m, n, scale = 6, 40, 0.7
    gen = torch.Generator(device="cuda").manual_seed(3)
    for gate in ("none", "channel", "token"):
        for post in (False, True):
            i = inputs(m, n, True, post, gate)
            h64, _ = U.norm_forward(i["r"], i["y"], i["w_pre"], i["w_post"], i["gate"], scale, EPS)
            desc = B.make_norm_desc(n, torch.float32, GATES[gate], scale, EPS)
            h = torch.empty((m, n), device="cuda").copy_(h64)
            got = dict(zip(("r", "y", "w_pre", "w_post", "gate"), B.qeft_norm_bwd(desc, i["dx"], h, i["w_pre"], dh=i["dh"], y=i["y"], w_post=i["w_post"], gate=i["gate"])))
            for name, grad in got.items():
                if i[name] is None:
                    continue
                way = torch.randn(i[name].shape, generator=gen, device="cuda", dtype=torch.float64)
                ends = []
                for e in (1e-5, -1e-5):
                    moved = {k: (v.double() + e * way if k == name else v) for k, v in i.items()}
                    hh, x = U.norm_forward(moved["r"], moved["y"], moved["w_pre"], moved["w_post"], moved["gate"], scale, EPS)
                    ends.append((hh * i["dh"].double()).sum() + (x * i["dx"].double()).sum())
                slope, along = (ends[0] - ends[1]) / 2e-5, (grad.double() * way).sum()
                # fp16 gradients of unit directions: half a step of each of up to m n values, in quadrature with room
                assert abs(float(slope - along)) <= 8 * U.HALF * float((grad.double() * way).norm()) + 1e-5, (gate, post, name)


def test_no_rows():
    desc = B.make_norm_desc(64, torch.float32, B.QEFT_GATE_CHANNEL, 1.0, EPS)
    e16, e32 = torch.empty((0, 64), dtype=torch.float16, device="cuda"), torch.empty((0, 64), device="cuda")
    w, g = torch.ones(64, dtype=torch.float16, device="cuda"), torch.ones(64, dtype=torch.float16, device="cuda")
    h, x = B.qeft_norm_fwd(desc, e32, w, y=e16, gate=g)
    assert h.shape == x.shape == (0, 64)
    dw, dg = torch.full((64,), 3.0, device="cuda"), torch.full((64,), 4.0, device="cuda")
    B.qeft_norm_bwd(desc, e16, e32, w, dh=e32, y=e16, gate=g, dw_pre=dw, dgate=dg, accumulate=True)
    assert bool((dw == 3).all()) and bool((dg == 4).all())
    B.qeft_norm_bwd(desc, e16, e32, w, dh=e32, y=e16, gate=g, dw_pre=dw, dgate=dg)
    assert not bool(dw.any()) and not bool(dg.any())


def test_gradients_from_a_graph_and_without_the_native_module(monkeypatch):
    i, desc, got = check_bwd(50, 1000, False, True, "channel")
    ws = torch.empty(B.qeft_norm_workspace(desc, 50), dtype=torch.uint8, device="cuda")
    outs = [torch.empty_like(got[k]) for k in got]
    h, x = torch.empty((50, 1000), dtype=torch.float16, device="cuda"), torch.empty((50, 1000), dtype=torch.float16, device="cuda")

    def both():
        B.qeft_norm_fwd(desc, i["r"], i["w_pre"], y=i["y"], w_post=i["w_post"], gate=i["gate"], h=h, x=x)
        return B.qeft_norm_bwd(desc, i["dx"], i["r"], i["w_pre"], i["dh"], i["y"], i["w_post"], i["gate"], *outs, ws=ws)

    both()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=torch.cuda.Stream()):
        both()
    for _ in range(3):
        for o in (*outs, h, x):
            o.fill_(9)
        ws.fill_(255)
        g.replay()
        torch.cuda.synchronize()
        with monkeypatch.context() as m:
            m.setattr(B, "_native", type("None_", (), {n: staticmethod(lambda *a: None) for n in dir(B._native) if not n.startswith("__")}))
            h2, x2 = B.qeft_norm_fwd(desc, i["r"], i["w_pre"], y=i["y"], w_post=i["w_post"], gate=i["gate"])
            plain = B.qeft_norm_bwd(desc, i["dx"], i["r"], i["w_pre"], i["dh"], i["y"], i["w_post"], i["gate"])
        for a, b in zip((*outs, h, x), (*plain, h2, x2)):
            assert torch.equal(a, b)
        for a, k in zip(outs, got):
            assert torch.equal(a, got[k])


@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("post,gate", [(False, "none"), (True, "channel"), (True, "token")])
@pytest.mark.parametrize("m,n", [(1, 4096), (3, 7), (3, 512), (301, 8192), (301, 16384), (3, 16400)])
def test_backward_with_no_eps(m, n, f32, post, gate):
    """Workgroups have room for more rows than there are: a row that does not exist has no norm, and no part in the sums over rows."""
    i = inputs(m, n, f32, post, gate)
    desc = B.make_norm_desc(n, i["r"].dtype, GATES[gate], 0.7, 0.0)
    got = dict(zip(("dr", "dy", "dw_pre", "dw_post", "dgate"),
                   B.qeft_norm_bwd(desc, i["dx"], i["r"], i["w_pre"], dh=i["dh"], y=i["y"], w_post=i["w_post"], gate=i["gate"])))
    want = U.norm_backward(i["dx"], i["dh"], i["r"], i["y"], i["w_pre"], i["w_post"], i["gate"], 0.7, 0.0, gate == "channel")
    assert {k for k, v in got.items() if v is not None} == set(want)
    for k, (w, bound) in want.items():
        U.close(k, got[k], w, bound, U.ROUNDING[got[k].dtype])
    h, x = B.qeft_norm_fwd(desc, i["r"], i["w_pre"], y=i["y"], w_post=i["w_post"], gate=i["gate"])
    _, want = U.norm_forward(h, None, i["w_pre"], None, None, 1.0, 0.0)
    U.close("x", x, want, 2 * U.sums_rounding(n) * want.abs(), U.HALF)


@pytest.mark.parametrize("n", [16384, 16385])
def test_backward_without_sums_and_without_a_workspace(n):
    """Rows that fit the registers need none; longer ones are refused without it."""
    i = inputs(3, n, False, False, "none")
    desc = B.make_norm_desc(n, torch.float16, eps=EPS)
    none = torch.empty(0, dtype=torch.uint8, device="cuda")
    if n > 16384:
        with pytest.raises(B.QeftError) as e:
            B.qeft_norm_bwd(desc, i["dx"], i["r"], i["w_pre"], dw_pre=False, ws=none)
        assert e.value.status == B.QEFT_ERR_WORKSPACE
        none = torch.empty(B.qeft_norm_workspace(desc, 3), dtype=torch.uint8, device="cuda")
    got = B.qeft_norm_bwd(desc, i["dx"], i["r"], i["w_pre"], dw_pre=False, ws=none)
    want, bound = U.norm_backward(i["dx"], None, i["r"], None, i["w_pre"], None, None, 1.0, EPS, False)["dr"]
    U.close("dr", got[0], want, bound, U.HALF)
