"""The weights' gradients of normed heads where every term counts: heads of plus and minus one have the norm one, gradients are whole numbers and rotations quarter turns, so that every product
is whole and every sum below 2^24 and exact in fp32 in any order.  A term that is missing or counted twice shows, however many there are."""
import pytest
import torch

from paper_2410_08661_amd import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d,rot_dim", [(128, 128), (128, 0), (64, 32), (40, 20), (80, 80), (256, 128), (40, 6), (8, 2)])
@pytest.mark.parametrize("m,heads,kv", [(1, 1, 1), (7, 3, 2), (333, 32, 1), (1348, 8, 40), (4001, 16, 4), (20001, 3, 3)])
def test_every_term_of_the_sums(m, heads, kv, d, rot_dim):
    gen = torch.Generator(device="cuda").manual_seed(m * 1000 + d + rot_dim)
    whole = lambda n, most: torch.randint(-most, most + 1, (m, n), generator=gen, device="cuda").half()  # noqa: E731
    sign = lambda n: (torch.randint(0, 2, (m, n), generator=gen, device="cuda") * 2 - 1).half()  # noqa: E731
    q, k, gq, gk = sign(heads * d), sign(kv * d), whole(heads * d, 8), whole(kv * d, 8)
    w = [(1 + torch.rand(d, generator=gen, device="cuda")).half() for _ in range(2)]
    rot = pos = None
    half = rot_dim // 2
    if half:
        turns = torch.randint(0, 4, (50, half), generator=gen, device="cuda")
        c, s = torch.tensor([1.0, 0, -1, 0], device="cuda")[turns], torch.tensor([0, 1.0, 0, -1], device="cuda")[turns]
        rot, pos = torch.cat((c, s), 1).contiguous(), torch.randint(0, 50, (m,), generator=gen, device="cuda").int()

    def sums(g, x, n):
        g, x = g.double().view(m, n, d), x.double().view(m, n, d)
        if half:
            c, s = (t[pos.long()][:, None].double() for t in (rot[:, :half], rot[:, half:]))
            a, b = g[..., :half], g[..., half:rot_dim]
            g = torch.cat((a * c + b * s, b * c - a * s, g[..., rot_dim:]), 2)
        return (g * x).sum((0, 1))

    desc = B.make_qk_desc(d, heads, kv, rot_dim, eps=0.0)
    want = sums(gq, q, heads), sums(gk, k, kv)
    assert max(float(t.abs().max()) for t in want) < 2 ** 24 and m * max(heads, kv) * 16 < 2 ** 24
    _, _, dw_q, dw_k = B.qeft_qk_norm_bwd(desc, gq, gk, q=q, k=k, w_q=w[0], w_k=w[1], rot=rot, pos=pos)
    assert torch.equal(dw_q.double(), want[0]) and torch.equal(dw_k.double(), want[1])
    # added to what is there, and for one side alone
    have = torch.arange(d, dtype=torch.float32, device="cuda")
    out = B.qeft_qk_norm_bwd(desc, gq, gk, q=q, k=k, w_q=w[0], w_k=w[1], rot=rot, pos=pos, dq=False, dk=False, dw_q=have.clone(), dw_k=have.clone(), accumulate=True)
    assert torch.equal(out[2].double(), want[0] + have) and torch.equal(out[3].double(), want[1] + have)
    assert torch.equal(B.qeft_qk_norm_bwd(desc, None, gk, k=k, w_k=w[1], rot=rot, pos=pos, dk=False)[3], dw_k)
