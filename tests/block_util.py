"""References in 64 bits for what lies between the linear layers, and their error bounds: straight from the definitions in include/qeft.h."""
import math

import torch

HALF = 2.0 ** -11       # relative rounding of fp16
TINY = 2.0 ** -25       # and of its smallest numbers
U = 2.0 ** -24          # fp32
ROUNDING = {torch.float16: HALF, torch.float32: U}


def pool_of(pages, kv, page, d, gen, order="pages"):
    """A random pool [pages][kv][page][d]; order "tokens": lying in memory as [pages][page][kv][d], "heads": as [kv][pages][page][d]."""
    shape = {"pages": (pages, kv, page, d), "tokens": (pages, page, kv, d), "heads": (kv, pages, page, d)}[order]
    x = torch.randn(shape, generator=gen, device="cuda").half()
    return {"pages": x, "tokens": x.transpose(1, 2), "heads": x.transpose(0, 1)}[order]


def rows_of(pool, table, b, h, n):
    """The first n cached rows of one head, fp64."""
    page = pool.shape[2]
    t = torch.arange(n, device=pool.device)
    return pool[table[b].long().clamp(0, pool.shape[0] - 1)[t // page], h, t % page].double()


def attention(K, V, table, lens, q, heads, scale):
    """(out, weights, bounds of both) in 64 bits; weights [seqs][kv][longest]."""
    kv, d = K.shape[1], K.shape[3]
    seqs, g = q.shape[0], heads // kv
    longest = max(max(lens), 1)
    out = torch.zeros((seqs, heads, d), dtype=torch.float64, device=q.device)
    w = torch.zeros((seqs, kv, longest), dtype=torch.float64, device=q.device)
    eo, ew = torch.full_like(out, TINY), torch.full_like(w, 2.0 ** -120)
    for b, n in enumerate(lens):
        if n <= 0:
            continue
        for h in range(kv):
            k, v = rows_of(K, table, b, h, n), rows_of(V, table, b, h, n)
            x = q[b, h * g * d: (h + 1) * g * d].double().view(g, d)
            s = x @ k.t() * scale
            p = torch.softmax(s, 1)
            sl = slice(h * g, (h + 1) * g)
            out[b, sl] = p @ v
            w[b, h, :n] = p.sum(0)
            # of a probability: d products and sums in a score, its scaling and distance from the maximum (both of the score's size); the sum of n
            # exponentials (a lane has n / 32 of them in a row, then 16 joins); the exponential; two fp16 values of 10 cut bits each
            size = (x.abs() @ k.abs().t() * abs(scale)).amax(1, keepdim=True)
            rel = 2 * (d + 8) * U * size + (n / 32 + 32) * U + 2.0 ** -20
            eo[b, sl] += HALF * out[b, sl].abs() + rel * (p @ v.abs()) + (d + n / 32 + 32) * U * (p @ v.abs())
            ew[b, h, :n] += (rel * p).sum(0) + g * U * w[b, h, :n]
    return out.view(seqs, -1), w, eo.view(seqs, -1), ew


def rotated(x, heads, rot, pos, rot_dim):
    """Rows of heads rotated, and the bound: two products and a sum in fp32, one rounding."""
    half = rot_dim // 2
    x = x.double().view(x.shape[0], heads, -1)
    y, size = x.clone(), x.abs()
    if half:
        cs = rot.double()[pos.long().clamp(0, rot.shape[0] - 1)][:, None]
        c, s = cs[..., :half], cs[..., half: rot_dim]
        a, b = x[..., :half], x[..., half: rot_dim]
        y[..., :half], y[..., half: rot_dim] = a * c - b * s, b * c + a * s
        big = (a * c).abs() + (b * s).abs() + (b * c).abs() + (a * s).abs()
        size[..., :half], size[..., half: rot_dim] = big, big
    n = x.shape[0]
    return y.view(n, -1), (HALF * y.abs() + 2 * U * size + TINY).view(n, -1)


def evicted(score, pos, n, seen, budget, first, last):
    """What one row keeps: the token that ends up in each of its first slots."""
    left = min(n, budget)
    if n <= budget:
        return list(range(n))

    def key(i):
        if pos[i] < first or pos[i] >= seen - last:
            s = math.inf
        else:
            s = score[i] + 0.0
        return (0 if s != s else 1, 0.0 if s != s else -s, i)

    kept = sorted(range(n), key=key)[:left]
    movers = iter(sorted(i for i in kept if i >= left))
    stay = set(kept)
    return [i if i in stay else next(movers) for i in range(left)]


def unit(z, eps):
    return z / (z.square().mean(1, keepdim=True) + eps).sqrt()


def norm_forward(r, y, w_pre, w_post, gate, scale, eps):
    """h and x in 64 bits (h as it is before it is stored)."""
    r = r.double()
    h = r
    if y is not None:
        u = y.double()
        if w_post is not None:
            u = unit(u, eps) * w_post.double()
        if gate is not None:
            u = u * gate.double()
        h = r + scale * u
    return h, unit(h, eps) * w_pre.double()


def sums_rounding(n):
    """Relative rounding of a row's sum: at most 32 terms one after the other, 6 steps of a wave, 16 waves, and more terms in very long rows."""
    return (64 + n / 1024) * U


def norm_backward(dx, dh, h, y, w_pre, w_post, gate, scale, eps, channel):
    """Gradients and their bounds in 64 bits, from the formulas."""
    n = h.shape[1]
    R = sums_rounding(n)
    h, dx, wp = h.double(), dx.double(), w_pre.double()
    dh = torch.zeros_like(h) if dh is None else dh.double()
    rs = (h.square().mean(1, keepdim=True) + eps).rsqrt()
    hh, a = h * rs, dx * wp
    t = dh + rs * (a - hh * (a * hh).mean(1, keepdim=True))
    tm = dh.abs() + rs * (a.abs() + hh.abs() * (a * hh).abs().mean(1, keepdim=True))        # sizes of what t is made of
    g = {"dr": (t, 4 * R * tm), "dw_pre": ((dx * hh).sum(0), (2 * R + h.shape[0] * U) * (dx * hh).abs().sum(0) + 1e-40)}
    if y is None:
        return g
    y = y.double()
    gt = torch.ones_like(t) if gate is None else gate.double().expand_as(t)
    du, dum = scale * gt * t, abs(scale) * gt.abs() * tm
    u, um = y, y.abs()
    if w_post is not None:
        wq = w_post.double()
        ry = (y.square().mean(1, keepdim=True) + eps).rsqrt()
        yh = y * ry
        u, um = yh * wq, (yh * wq).abs()
        b, bm = du * wq, dum * wq.abs()
        g["dy"] = (ry * (b - yh * (b * yh).mean(1, keepdim=True)), 8 * R * ry * (bm + yh.abs() * (bm * yh.abs()).mean(1, keepdim=True)))
        g["dw_post"] = ((du * yh).sum(0), (8 * R + h.shape[0] * U) * (dum * yh.abs()).sum(0) + 1e-40)
    else:
        g["dy"] = (du, 8 * R * dum)
    if gate is not None:
        dg, dgm = scale * u * t, 8 * R * abs(scale) * um * tm
        g["dgate"] = (dg.sum(0), dgm.sum(0) + h.shape[0] * U * (scale * um * tm).abs().sum(0) + 1e-40) if channel else (dg, dgm)
    return g


def close(name, got, want, bound, rounding=0.0):
    """Every value within its bound and a rounding to the output's type."""
    got = got.double()
    assert got.shape == want.shape, name
    tol = bound + rounding * want.abs() + (TINY if rounding == HALF else 0.0)
    bad = ~((got - want).abs() <= tol)
    if bool(bad.any()):
        i = tuple(bad.nonzero()[0].tolist())
        raise AssertionError(f"{name}: {int(bad.sum())} of {bad.numel()} off, first at {i}: {got[i].item()} for {want[i].item()}, bound {tol[i].item() if tol.dim() else tol}")
