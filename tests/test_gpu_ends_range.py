"""Log probabilities and the logits' gradient where scaled logits are large: offsets, low temperatures, the largest numbers, masks of the type's lowest value.

The bounds are those of arithmetic by differences from the row's largest logit M, so that nothing but lse, and what is made of a stored lse, depends on how large the logits are.
With d = scale (M - z), U = 2^-24:  an exponential exp(-d) is off by 4 U d (the difference, the factor scale log2 e of two roundings, the product) and 2 U (the function); parts and
waves of a row are brought to one M by one factor more, of the same kind for the rest of the distance, and 3 U.  The sum of a row: chains of 64 terms, then 1 + 6 + 4 + 8 steps
between accumulators, lanes, waves and parts."""
import math
import zlib

import pytest
import torch

import ends_util as V
from paper_2410_08661_amd import binding as B

pytestmark = pytest.mark.gpu
U = V.U
SIZES = [(3, 40), (3, 4099), (3, 32000), (3, 70003), (2, 140001), (200, 70003)]
# fp32, offset, deviation, scale, share at the type's lowest value
RANGES = [
    (False, 0.0, 4.0, 1e3, 0.0), (False, 0.0, 4.0, 1e5, 0.0), (False, 0.0, 4.0, 2.0 ** 20, 0.3), (False, 3e4, 300.0, 1 / 64, 0.0), (False, 6e4, 900.0, 1.0, 0.0), (False, -6e4, 900.0, 1 / 16, 0.2),
    (False, 3e4, 300.0, 0.7, 0.0), (False, 6e4, 900.0, 2.0 ** 100, 0.0), (True, 1e3, 3.0, 1.0, 0.0), (True, 3e4, 3.0, 1.0, 0.3), (True, 3e4, 3.0, 0.7, 0.0), (True, -1e6, 3.0, 1.3, 0.3), (True, 1e9, 200.0, 1.0, 0.0),
    (True, 3.5e9, 600.0, 0.1, 0.2), (True, 0.0, 3e9, 1.0, 0.0), (True, 0.0, 1e12, 1.0, 0.0), (True, 0.0, 1e20, 1e5, 0.0), (True, 1e38, 3e37, 1.0, 0.0), (True, 1e38, 3e37, 2e-38, 0.0), (True, 3.0, 3.0, 1e30, 0.5),
    (True, 5.8145e6, 300.0, 1.0, 0.0), (True, -5.8145e6, 300.0, 1.0, 0.3)]


def exact32(x):
    return float(torch.tensor(x, dtype=torch.float32))


def rows(m, n, f32, offset, std, lowest, gen):
    z = V.logits(m, n, f32, gen, pad=0)
    x = offset + std * torch.randn((m, n), generator=gen, device="cuda", dtype=torch.float64)
    z.copy_(x.clamp(-65504, 65504) if not f32 else x)
    low = torch.finfo(z.dtype).min
    z.masked_fill_(torch.rand((m, n), generator=gen, device="cuda") < lowest, low)
    z[0, n // 3] = z[0, n // 2] = z[0].max()       # two largest
    z[1, n // 5] = -math.inf
    return z


def reference(z, token, scale):
    """lse, logp, entropy and probabilities in 64 bits with their bounds."""
    x = z.double()
    top = x.amax(1, keepdim=True)
    d = (top - x) * scale
    e = (-d).exp()
    s = e.sum(1)
    p = e / s[:, None]
    dist = torch.where(p > 0, d, 0.0)
    D, D2 = (p * dist).sum(1), (p * dist * dist).sum(1)
    ln_s = s.log()
    E = 4 * U * D + 88 * U                         # of s: 83 steps and 5 of the terms
    eln = E + 4 * U * ln_s                         # (the logarithm)
    lse, logp, H = top[:, 0] * scale + ln_s, -d - ln_s[:, None], ln_s + D
    eH = eln + 4 * U * D2 + 200 * U * D + D * E + 4 * U * H
    lp = logp.gather(1, token.long()[:, None])[:, 0]
    dt = torch.where(lp > -math.inf, lp + ln_s, 0.0).abs()
    want = {"lse": (lse, eln + 2 * U * lse.abs()), "logp": (lp, eln + 4 * U * dt + 2 * U * (dt + ln_s)), "entropy": (H, eH)}
    return want, dict(d=dist, p=p, logp=torch.where(p > 0, logp, 0.0), all_logp=logp, H=H, eH=eH, E=E, eln=eln, lse=lse, ln_s=ln_s, top=top * scale)


def gradient(r, token, scale, dl, ds, dh, kept=0.0):
    """(dz, bound); kept: what a probability made of a stored lse has besides, relative."""
    p, d = r["p"], r["d"]
    one = torch.zeros_like(p).scatter_(1, token.long()[:, None], 1.0)
    dl, ds, dh = (g.double()[:, None] for g in (dl, ds, dh))
    H, eH = r["H"][:, None], r["eH"][:, None]
    dz = scale * (dl * (one - p) + ds * p - dh * p * (r["logp"] + H))
    rel = 4 * U * d + 5 * U + r["E"][:, None] + kept
    size = dl.abs() + ds.abs() + dh.abs() * (H + r["logp"].abs())
    bound = scale * p * (size * (rel + 8 * U) + dh.abs() * (4 * U * d + r["eln"][:, None] + eH + kept)) + 8 * U * scale * (dl * one).abs()
    # (an exponential below the smallest normal number may be 0)
    return dz, bound + scale * size * 2.0 ** -125


def finite(t):
    return torch.where(t.abs() <= torch.finfo(torch.float32).max, t, torch.where(t > 0, math.inf, -math.inf))


@pytest.mark.parametrize("m,n", SIZES)
@pytest.mark.parametrize("f32,offset,std,scale,lowest", RANGES)
def test_large_scaled_logits_forward(f32, offset, std, scale, lowest, m, n):
    gen = torch.Generator(device="cuda").manual_seed(zlib.crc32(repr((f32, offset, scale, m, n)).encode()))
    scale = exact32(scale)
    z = rows(m, n, f32, offset, std, lowest, gen)
    token = torch.randint(0, n, (m,), generator=gen, device="cuda").int()
    token[0] = n // 2                              # one of the two largest
    desc = B.make_logprob_desc(n, z.dtype, scale)
    logp, lse, entropy, top_logp, top_index = B.qeft_logprob_fwd(desc, z, token, top=3)
    want, r = reference(z, token, scale)
    for name, got in (("lse", lse), ("logp", logp), ("entropy", entropy)):
        w, b = want[name]
        w = finite(w)
        assert not bool(got.isnan().any()), name
        assert torch.equal(got.double()[w.isinf()], w[w.isinf()]), name
        V.close(name, torch.where(w.isinf(), 0.0, got.double()), torch.where(w.isinf(), 0.0, w), b, U)
    index = V.alternatives(z, None, 3)
    assert torch.equal(top_index, index)
    lp = r["all_logp"].gather(1, index.long())
    b = r["eln"][:, None] + 6 * U * (lp.abs() + 2 * r["ln_s"][:, None])
    there = finite(lp).isfinite()
    assert torch.equal(top_logp.double()[~there], finite(lp)[~there])
    V.close("top_logp", top_logp[there], lp[there], b[there], U)


@pytest.mark.parametrize("n", [8, 100, 4099, 140001])
def test_rows_of_the_lowest_value_and_of_nothing(n):
    """Every entry the type's lowest value: all equally likely, unlike a row of -infinity."""
    for t in (torch.float16, torch.float32):
        z = torch.full((3, (n + 7) // 8 * 8), torch.finfo(t).min, dtype=t, device="cuda")[:, :n]
        z[1] = -math.inf
        z[2] = torch.finfo(t).max
        token = torch.full((3,), n - 1, dtype=torch.int32, device="cuda")
        logp, lse, entropy, lp, ix = B.qeft_logprob_fwd(B.make_logprob_desc(n, t, 0.5), z, token, top=2)
        for i, x in ((0, torch.finfo(t).min), (2, torch.finfo(t).max)):
            assert abs(float(logp[i]) + math.log(n)) <= 200 * U and abs(float(entropy[i]) - math.log(n)) <= 200 * U
            assert abs(float(lse[i]) - (0.5 * x + math.log(n))) <= 2 * U * abs(0.5 * x) and ix[i].tolist() == [0, 1]
            assert torch.equal(lp[i], logp[i].expand(2))
        assert lse[1] == logp[1] == -math.inf and entropy[1] == 0 and ix[1].tolist() == [-1, -1]


def some_gradients(m, scale, gen):
    return [torch.randn(m, generator=gen, device="cuda") * min(1 / scale, 1e30) for _ in range(3)]


def check_one_call(f32, offset, std, scale, lowest, m, n):
    gen = torch.Generator(device="cuda").manual_seed(zlib.crc32(repr((f32, offset, scale, m, n, "g")).encode()))
    scale = exact32(scale)
    z = rows(m, n, f32, offset, std, lowest, gen)
    token = torch.randint(0, n, (m,), generator=gen, device="cuda").int()
    token[0] = n // 2
    desc = B.make_logprob_desc(n, z.dtype, scale)
    _, r = reference(z, token, scale)
    g = some_gradients(m, scale, gen)
    want, bound = gradient(r, token, scale, *g)
    V.close("dz", B.qeft_logprob_fwd_bwd(desc, z, token, *g)[0], want, bound, V.ROUNDING[z.dtype])
    # a loss moves no row's sum: probabilities and the token's one, however large the logits
    none = torch.zeros(m, device="cuda")
    want, bound = gradient(r, token, scale, g[0], none, none)
    dz = B.qeft_logprob_fwd_bwd(desc, z, token, g[0])[0]
    V.close("dz of a loss", dz, want, bound, V.ROUNDING[z.dtype])
    room = bound + V.ROUNDING[z.dtype] * want.abs() + (V.TINY if not f32 else 0.0)
    assert bool((dz.double().sum(1).abs() <= room.sum(1)).all())


@pytest.mark.parametrize("m,n", [(3, 40), (3, 4099), (3, 32000), (200, 65536)])
@pytest.mark.parametrize("f32,offset,std,scale,lowest", RANGES)
def test_gradient_in_one_call_of_large_scaled_logits(f32, offset, std, scale, lowest, m, n):
    check_one_call(f32, offset, std, scale, lowest, m, n)


@pytest.mark.parametrize("m,n", [(2, 140001), (300, 132001)])
@pytest.mark.parametrize("f32,offset,std,scale,lowest", RANGES)
def test_gradient_in_one_call_of_large_scaled_logits_in_parts(f32, offset, std, scale, lowest, m, n):
    check_one_call(f32, offset, std, scale, lowest, m, n)


@pytest.mark.parametrize("m,n", [(3, 40), (3, 4099), (3, 32000), (2, 140001)])
@pytest.mark.parametrize("f32,offset,std,scale,lowest", [r for r in RANGES if max(abs(r[1]), 4 * r[2]) * r[3] <= 1e5])
def test_gradient_of_large_scaled_logits_by_a_stored_lse(f32, offset, std, scale, lowest, m, n):
    """As exact as lse is as fp32, which is U of its size."""
    gen = torch.Generator(device="cuda").manual_seed(zlib.crc32(repr((f32, offset, scale, m, n, "s")).encode()))
    scale = exact32(scale)
    z = rows(m, n, f32, offset, std, lowest, gen)
    token = torch.randint(0, n, (m,), generator=gen, device="cuda").int()
    desc = B.make_logprob_desc(n, z.dtype, scale)
    _, lse, entropy, _, _ = B.qeft_logprob_fwd(desc, z, token)
    _, r = reference(z, token, scale)
    g = some_gradients(m, scale, gen)
    kept = torch.expm1((U * r["lse"].abs() + r["eln"])[:, None] + 4 * U * r["logp"].abs())
    want, bound = gradient(r, token, scale, *g, kept=kept)
    V.close("dz", B.qeft_logprob_bwd(desc, z, lse, token=token, dlogp=g[0], dlse=g[1], entropy=entropy, dentropy=g[2]), want, bound, V.ROUNDING[z.dtype])


@pytest.mark.parametrize("n", [40, 4099, 32000])
@pytest.mark.parametrize("offset,std,scale", [(0.0, 3.0, 1.0), (1e3, 3.0, 1.0), (1e3, 3.0, 0.7), (3e4, 3.0, 1.3), (-1e6, 3.0, 1.7), (5.8145e6, 20.0, 1.0), (5.8145e6, 20.0, 1 / 3), (1e9, 200.0, 0.9), (0.0, 4.0, 1e5), (1e20, 1e16, 1e-19),
                                              (0.0, 1e4, 1e25)])
def test_gradient_of_logits_by_a_given_lse(offset, std, scale, n):
    """dlse p with p = exp(scale z - lse) of the lse that is given: what the forward's is off by does not grow on the way.  The argument: the factor's two roundings and the multiply-add's (or
    difference, log2 e and product), 4 U of its distance; the exponential 2 U, its share's 2 U and those of the argument's known error, below 4 U; three products."""
    gen = torch.Generator(device="cuda").manual_seed(zlib.crc32(repr((offset, scale, n)).encode()))
    scale = exact32(scale)
    z = rows(3, n, True, offset, std, 0.0, gen)
    desc = B.make_logprob_desc(n, torch.float32, scale)
    lse = (z.double().amax(1) * scale + math.log(n)).float()        # (near the forward's)
    g = some_gradients(3, scale, gen)[0]
    x = z.double() * scale - lse.double()[:, None]
    p = x.exp()
    want = scale * g.double()[:, None] * p
    bound = want.abs() * (4 * U * torch.where(p > 0, x, 0.0).abs() + 12 * U) + scale * g.double().abs()[:, None] * 2.0 ** -125
    dz, want = B.qeft_logprob_bwd(desc, z, lse, dlse=g), finite(want)      # (an lse rounded far below the largest: infinity)
    inf = want.isinf()
    assert torch.equal(dz.double()[inf], want[inf])
    V.close("dz", dz[~inf], want[~inf], bound[~inf], U)
