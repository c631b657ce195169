"""References in 64 bits for the ends of a step, and their error bounds: straight from the definitions in include/qeft.h."""
import math

import torch

from block_util import HALF, ROUNDING, TINY, U, close  # noqa: F401
from paper_2410_08661_amd import binding as B

NONE = type("None_", (), {n: staticmethod(lambda *a: None) for n in dir(B._native) if not n.startswith("__")})   # in place of the native module: ctypes


def logits(m, n, f32, gen, banned=0.0, pad=8, std=3.0):
    """[m][n] with a pitch of its own; what lies behind a row's end is not a number."""
    ld = (n + 7) // 8 * 8 + pad
    t = torch.float32 if f32 else torch.float16
    z = torch.full((m, ld), float("nan"), dtype=t, device="cuda")[:, :n]
    x = torch.randn((m, n), generator=gen, device="cuda") * std
    x.masked_fill_(torch.rand((m, n), generator=gen, device="cuda") < banned, float("-inf"))
    return z.copy_(x)


def log_probabilities(z, token, scale):
    """{name: (value, bound)} of lse, logp, entropy in 64 bits, and what the gradient needs; rows that are left out have 0 everywhere."""
    m, n = z.shape
    x = z.double() * scale
    top = x.amax(1, keepdim=True)
    empty = (top == -math.inf)[:, 0]
    d = torch.where(empty[:, None], -math.inf, x - top)                     # distance from the largest
    e = d.exp()
    s = e.sum(1, keepdim=True)
    p = torch.where(empty[:, None], 0.0, e / s)
    ln_s = torch.where(empty, 0.0, s[:, 0].log())
    dist = torch.where(p > 0, d, 0.0).abs()
    D, D2 = (p * dist).sum(1), (p * dist * dist).sum(1)
    # an exponential: c and the multiply-add of its argument, 2^-23 each of the distance, and the function; the sum of n of them
    E = 4 * U * D + (n / 256 + 44) * U
    A = torch.where(empty, 0.0, top[:, 0].abs())
    lse = torch.where(empty, -math.inf, top[:, 0] + ln_s)
    out = {"lse": (lse, 5 * U * A + E + 5 * U * (1 + ln_s.abs()))}
    logs = torch.where(empty[:, None], -math.inf, d - ln_s[:, None])
    H = ln_s + D
    eH = E + 5 * U * (1 + ln_s.abs()) + 4 * U * D2 + (n / 256 + 44) * 2 * U * D + D * E
    out["entropy"] = (torch.where(empty, 0.0, H), eH)
    has = torch.ones(m, dtype=torch.bool, device=z.device) if token is None else (token >= 0) & (token < n)
    if token is not None:
        t = token.long().clamp(0, n - 1)[:, None]
        lp = logs.gather(1, t)[:, 0]
        dt = torch.where(lp > -math.inf, d.gather(1, t)[:, 0], 0.0).abs()
        out["logp"] = (lp, 5 * U * dt + E + 5 * U * (1 + ln_s.abs()))
    out = {k: (torch.where(has, v, 0.0), torch.where(has, b, 0.0)) for k, (v, b) in out.items()}
    return out, dict(x=x, p=p, logs=logs, H=H, eH=eH, E=E, lse=torch.where(empty, 0.0, lse), has=has, empty=empty)


def check_values(got, want):
    """Values of lse, logp or entropy within their bounds, infinities where they are."""
    for name, (w, b) in want.items():
        g = got[name]
        if g is None:
            continue
        assert g.dtype == torch.float32
        inf = ~w.isfinite()
        assert torch.equal(g.double()[inf], w[inf]), name
        close(name, torch.where(inf, 0.0, g.double()), torch.where(inf, 0.0, w), b, U)


def logit_gradient(z, token, scale, dlogp, dlse, dentropy):
    """(dz, bound) from the formula."""
    _, r = log_probabilities(z, token, scale)
    m, n = z.shape
    col = lambda t: torch.zeros((m, 1), dtype=torch.float64, device=z.device) if t is None else t.double()[:, None]  # noqa: E731
    dl, ds, dh = col(dlogp), col(dlse), col(dentropy)
    p, logs, H = r["p"], torch.where(r["p"] > 0, r["logs"], 0.0), r["H"][:, None]
    one = torch.zeros_like(p)
    if token is not None:
        one.scatter_(1, token.long().clamp(0, n - 1)[:, None], 1.0)
    dz = scale * (dl * (one - p) + ds * p - dh * p * (logs + H))
    u = 8 * U * (torch.where(p > 0, r["x"], 0.0).abs() + r["lse"].abs()[:, None])               # of a log probability
    rel = u + r["E"][:, None] + 6 * U
    bound = scale * (p * ((dl.abs() + ds.abs() + dh.abs() * (H.abs() + logs.abs())) * (rel + 6 * U) + dh.abs() * (u + r["eH"][:, None])) + 6 * U * (dl * one).abs()) + 1e-37
    keep = (r["has"] & ~r["empty"])[:, None]
    return torch.where(keep, dz, 0.0), torch.where(keep, bound, 0.0)


def alternatives(z, token, top):
    """Indices by value and then place; -1 where there are no more."""
    n = z.shape[1]
    key = torch.where(z.isnan(), math.inf, z.double())
    # (not-a-number above infinity: two stable sorts, the last one the first criterion)
    order = torch.sort(key, dim=1, descending=True, stable=True).indices
    nan = z.gather(1, order).isnan()
    order = order.gather(1, torch.sort(nan.int(), dim=1, descending=True, stable=True).indices)[:, :top]
    there = z.gather(1, order) != -math.inf
    if token is not None:
        there &= ((token >= 0) & (token < n))[:, None]
    return torch.where(there, order, -1).int()


# ---- heads -----------------------------------------------------------------------------------------------------------

def turn(x, rot, pos, rot_dim, sign=1):
    """Heads [m][heads][d] rotated there (1) or back (-1), and the sizes of what was added."""
    half, size = rot_dim // 2, x.abs()
    if not half:
        return x, size
    cs = rot.double()[pos.long().clamp(0, rot.shape[0] - 1)][:, None]
    c, s = cs[..., :half], cs[..., half:rot_dim] * sign
    a, b = x[..., :half], x[..., half:rot_dim]
    y, size = x.clone(), size.clone()
    y[..., :half], y[..., half:rot_dim] = a * c - b * s, b * c + a * s
    size[..., :half], size[..., half:rot_dim] = (a * c).abs() + (b * s).abs(), (b * c).abs() + (a * s).abs()
    return y, size


SUM = 48 * U       # relative, of a head's sum: at most 32 terms one after the other, 6 steps between lanes


def heads_forward(x, heads, w, eps, rot, pos, rot_dim):
    """(value, bound) of normed and rotated heads, [m][heads * d]."""
    y = x.double().view(x.shape[0], heads, -1)
    if w is not None:
        y = y / (y.square().mean(-1, keepdim=True) + eps).sqrt() * w.double()
    y, size = turn(y, rot, pos, rot_dim)
    return y.reshape(x.shape[0], -1), ((SUM if w is not None else 0) * size + 3 * U * size).reshape(x.shape[0], -1)


def heads_backward(g, x, heads, w, eps, rot, pos, rot_dim):
    """((dx, bound), (dw, bound) or None)."""
    m = g.shape[0]
    g = g.double().view(m, heads, -1)
    g, size = turn(g, rot, pos, rot_dim, -1)
    if w is None:
        return (g.reshape(m, -1), (3 * U * size).reshape(m, -1)), None
    x, w = x.double().view(m, heads, -1), w.double()
    rs = (x.square().mean(-1, keepdim=True) + eps).rsqrt()
    xh, a, am = x * rs, g * w, size * w.abs()
    dx = rs * (a - xh * (a * xh).mean(-1, keepdim=True))
    dxm = rs * (am + xh.abs() * (am * xh.abs()).mean(-1, keepdim=True))
    N = m * heads
    return (dx.reshape(m, -1), (4 * SUM * dxm).reshape(m, -1)), ((g * xh).sum((0, 1)), (2 * SUM + N * U) * (size * xh.abs()).sum((0, 1)) + 1e-40)


# ---- the optimizer ---------------------------------------------------------------------------------------------------

def stir(x):
    """32 bits stirred, on whole numbers or int64 tensors."""
    for shift, factor in ((16, 0x5C3C9CCD), (15, 0xFA1B1BF1), (16, 1)):
        x = ((x ^ (x >> shift)) * factor) % (1 << 32)
    return x


def dice(first, n, step, seed):
    """The random numbers of places first .. first + n - 1 of a list."""
    at = torch.arange(first, first + n, device="cuda")
    key = stir((step + stir((seed % (1 << 32) + stir(seed >> 32)) % (1 << 32))) % (1 << 32))
    return stir((at % (1 << 32) + stir(((at >> 32) + key) % (1 << 32))) % (1 << 32))


def on_grid(x, u, bits, least):
    """x >= 0 on the grid of `bits` mantissa bits above `least`: rounded up where what is left of it and u in [0, 1) make a whole step."""
    step = torch.exp2(torch.floor(torch.log2(x.clamp(min=least))) - bits)
    return torch.floor(x / step + u) * step


def rounded_within(got, x, error, u, cut, bits, least):
    """Whether got is x, known to `error`, rounded by u, of which a `cut` of a step is lost.  With the same u rounding is monotone: the result lies between those of the
    error's two ends.  (x / step is formed in 64 bits here: an end that is a grid point by 2^-40 of itself counts as one.)"""
    step = torch.exp2(torch.floor(torch.log2(x.clamp(min=least))) - bits)
    e = error + cut * step + 2.0 ** -40 * x
    return (got >= on_grid((x - e).clamp(min=0), u, bits, least)) & (got <= on_grid(x + e, u, bits, least))


def state_values(code, scale, name, n):
    """8-bit states as fp64 values."""
    kind = torch.float8_e4m3fn if name == "m" else torch.float8_e5m2
    s = torch.exp2(scale.double() - 127).repeat_interleave(B.QEFT_STATE_BLOCK)[:n]
    return code.reshape(-1).view(kind).double() * s


def adamw(w, grad, m, v, lr, step, decay, beta1, beta2, eps, factor=1.0):
    """(w, m, v) after a step and their bounds, in 64 bits."""
    g = grad.double() * factor
    m1, m2, v1, v2 = beta1 * m, (1 - beta1) * g, beta2 * v, (1 - beta2) * g * g
    m, v = m1 + m2, v1 + v2
    em, ev = 4 * U * (m1.abs() + m2.abs()) + 1e-44, 6 * U * (v1.abs() + v2) + 1e-44
    c1, c2 = 1 - beta1 ** step, 1 - beta2 ** step
    den = (v / c2).sqrt() + eps
    up = lr * (m / c1) / den
    # (an error of v passes through the root by half: v is a sum of terms of one sign; below 2^-100 it is an absolute one, under eps)
    eup = lr / c1 * em / den + up.abs() * (24 * U + 0.5 * ev / v.clamp(min=2.0 ** -100)) + lr / c1 * m.abs() / den ** 2 * 2.0 ** -55
    new = w.double() * (1 - lr * decay) - up
    return (new, eup + 4 * U * abs(lr * decay) * w.double().abs() + U * w.double().abs()), (m, em), (v, ev)
