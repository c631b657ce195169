"""qeft_cache_append and qeft_cache_evict against their definitions: rotation in 64 bits, kept sets and slots exactly."""
import pytest
import torch

import block_util as U
from paper_2410_08661_amd import binding as B

pytestmark = pytest.mark.gpu


def rotation(positions, rot):
    f = 10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64, device="cuda") / rot)
    a = torch.arange(positions, dtype=torch.float64, device="cuda")[:, None] * f
    return torch.cat([a.cos(), a.sin()], 1).float()


@pytest.mark.parametrize("heads,kv,d,rot", [(8, 8, 128, 128), (12, 2, 96, 48), (4, 4, 80, 80), (4, 2, 80, 40), (5, 5, 64, 36), (3, 1, 24, 6), (2, 2, 8, 2), (8, 1, 256, 256),
                                            (6, 6, 64, 0), (0, 3, 128, 64)])
@pytest.mark.parametrize("tokens,seqs,page", [(1, 1, 16), (9, 3, 5), (2300, 2, 64)])
def test_append(heads, kv, d, rot, tokens, seqs, page):
    gen = torch.Generator(device="cuda").manual_seed(7 * d + tokens)
    each = -(-tokens // seqs)
    cols = -(-(each + 40) // page)
    pages = seqs * cols + 2
    K, V = (U.pool_of(pages, kv, page, d, gen) for _ in range(2))
    cache = B.Cache(B.make_cache_desc(pages, page, kv, d), k=K.clone(), v=V.clone())
    table = torch.randperm(pages, generator=gen, device="cuda")[: seqs * cols].int().view(seqs, cols)
    t = torch.arange(tokens, device="cuda")
    seq, index = (t // each).int(), (t % each + 40 - (t // each)).int()
    pos = (index * 3 + 1).int()
    k, v = (torch.randn((tokens, kv * d + 16), generator=gen, device="cuda").half()[:, 8: 8 + kv * d] for _ in range(2))
    q = torch.randn((tokens, heads * d), generator=gen, device="cuda").half() if heads else None
    table_rot = rotation(int(pos.max()) + 1, rot) if rot else None
    got = B.qeft_cache_append(cache, table, k, v, index, seq=seq, q=q, rot=table_rot, pos=pos)
    if heads:
        want, bound = U.rotated(q, heads, table_rot, pos, rot)
        U.close("q", got, want, bound)
        again = q.clone()
        B.qeft_cache_append(cache, table, k, v, index, seq=seq, q=again, q_out=again, rot=table_rot, pos=pos)
        assert torch.equal(again, got)
    else:
        assert got is None
    page_of, slot = table.long()[seq.long(), index.long() // page], index.long() % page
    want, bound = U.rotated(k, kv, table_rot, pos, rot)
    U.close("k", cache.k[page_of, :, slot].reshape(tokens, -1), want, bound)
    assert torch.equal(cache.v[page_of, :, slot].reshape(tokens, -1), v)
    K[page_of, :, slot], V[page_of, :, slot] = cache.k[page_of, :, slot], cache.v[page_of, :, slot]
    assert torch.equal(K, cache.k) and torch.equal(V, cache.v)          # nothing else was written
    if not rot:
        assert torch.equal(cache.k[page_of, :, slot].reshape(tokens, -1), k)


def test_append_without_sequences_and_positions():
    """One token of every sequence; its position is its index, clamped to the table."""
    kv, d, page = 2, 64, 8
    K = torch.zeros((6, page, kv, d), dtype=torch.float16, device="cuda").transpose(1, 2)
    V = torch.zeros_like(K)
    s = K.stride()
    cache = B.Cache(B.make_cache_desc(6, page, kv, d, s[0], s[1], s[2]), k=K, v=V)
    table = torch.tensor([[5, 0], [1, 2], [3, 4]], dtype=torch.int32, device="cuda")
    index = torch.tensor([3, 15, 9], dtype=torch.int32, device="cuda")
    k, v = torch.randn((3, kv * d), device="cuda").half(), torch.randn((3, kv * d), device="cuda").half()
    rot = rotation(10, d)
    B.qeft_cache_append(cache, table, k, v, index, rot=rot)
    want, bound = U.rotated(k, kv, rot, index, d)
    for b, (p, s) in enumerate([(5, 3), (2, 7), (4, 1)]):
        U.close("k", K[p, :, s].reshape(-1), want[b], bound[b])
        assert torch.equal(V[p, :, s].reshape(-1), v[b])


def test_append_skips_what_has_no_slot():
    kv, d, page = 1, 32, 4
    cache = B.Cache(B.make_cache_desc(3, page, kv, d))
    table = torch.tensor([[0, 7], [-1, 2]], dtype=torch.int32, device="cuda")
    seq = torch.tensor([0, 0, 1, 1, -1, 2, 0, 1, 0], dtype=torch.int32, device="cuda")
    index = torch.tensor([1, 4, 0, 5, 0, 0, 8, -1, 2 ** 31 - 1], dtype=torch.int32, device="cuda")   # only the first and the fourth have one
    k = torch.arange(1, 10, device="cuda").half()[:, None].expand(9, d).contiguous()
    q = B.qeft_cache_append(cache, table, k, -k, index, seq=seq, q=k)
    assert torch.equal(q, k)
    want = torch.zeros((3, kv, page, d), dtype=torch.float16, device="cuda")
    want[0, 0, 1], want[2, 0, 1] = 1, 4
    assert torch.equal(cache.k, want) and torch.equal(cache.v, -want)


def check_evict(kv, d, page, lens, budget, first=0, last=0, seed=0, inplace=False, make=None, order="pages", seen=None):
    gen = torch.Generator(device="cuda").manual_seed(seed + 31 * kv + d)
    seqs, longest = len(lens), max(max(lens), 1)
    cols = -(-longest // page)
    pages = seqs * cols + 1
    K, V = (U.pool_of(pages, kv, page, d, gen, order) for _ in range(2))
    table = torch.randperm(pages, generator=gen, device="cuda")[: seqs * cols].int().view(seqs, cols)
    score = torch.rand((seqs, kv, longest + 2), generator=gen, device="cuda").mul(40).round().div(16)
    if make:
        make(score)
    pos = torch.rand((seqs, kv, longest + 2), generator=gen, device="cuda").argsort(-1).int()
    seen = torch.tensor([n + 5 for n in lens] if seen is None else seen, dtype=torch.int32, device="cuda")
    s = K.stride()
    cache = B.Cache(B.make_cache_desc(pages, page, kv, d, s[0], s[1], s[2]), k=K.clone(memory_format=torch.preserve_format), v=V.clone(memory_format=torch.preserve_format))
    dev_lens = torch.tensor(lens, dtype=torch.int32, device="cuda")
    so, po = (score.clone(), pos.clone()) if inplace else (torch.full_like(score, -7), torch.full_like(pos, -7))
    keep_s, keep_p = so.clone(), po.clone()
    a, b = (so, po) if inplace else (score, pos)
    _, _, lens_out = B.qeft_cache_evict(cache, table, dev_lens, longest, budget, a, b, seen, keep_first=first, keep_last=last, score_out=so, pos_out=po)
    assert lens_out.tolist() == [min(n, budget) for n in lens] and dev_lens.tolist() == lens
    rows = table.long()
    moved = 0
    for i, n in enumerate(lens):
        for h in range(kv):
            to = U.evicted(score[i, h].tolist(), pos[i, h].tolist(), n, int(seen[i]), budget, first, last)
            at = torch.tensor(to, dtype=torch.long, device="cuda")
            dst = torch.arange(len(to), device="cuda")
            keep_s[i, h, : len(to)], keep_p[i, h, : len(to)] = score[i, h, at], pos[i, h, at]
            if n > budget:
                ch = at != dst
                moved += int(ch.sum())
                for pool in (K, V):
                    pool[rows[i, dst[ch] // page], h, dst[ch] % page] = pool[rows[i, at[ch] // page], h, at[ch] % page]
    assert torch.equal(so.view(torch.int32), keep_s.view(torch.int32)) and torch.equal(po, keep_p)
    assert torch.equal(cache.k, K) and torch.equal(cache.v, V)
    return moved


@pytest.mark.parametrize("inplace", [False, True])
@pytest.mark.parametrize("kv,d,page,lens,budget,first,last", [
    (4, 128, 16, [65, 64, 63, 1], 64, 4, 16),         # one token over, at, below the budget
    (2, 64, 8, [300, 299, 298, 297], 296, 0, 0),      # one to four to go
    (3, 80, 5, [301, 0, 120], 296, 2, 100),           # five to go: the selection by digits
    (2, 96, 16, [1000, 700], 100, 4, 30),             # lists and a second launch
    (1, 256, 64, [3000], 2999, 0, 50),
    (2, 8, 1, [50, 33], 20, 0, 0),
    (2, 64, 16, [200], 50, 30, 60),                   # more that must stay than the budget holds
    (2, 64, 16, [200, 3], 0, 0, 0),                   # nothing stays
    (2, 64, 32, [9000], 4500, 1, 1),
])
def test_evict(kv, d, page, lens, budget, first, last, inplace):
    check_evict(kv, d, page, lens, budget, first, last, inplace=inplace)


@pytest.mark.parametrize("budget", [299, 200, 10])
@pytest.mark.parametrize("kind", ["equal", "zeros", "nan", "inf", "negative", "close"])
def test_evict_ties_and_special_weights(budget, kind):
    def make(s):
        if kind == "equal":
            s.fill_(0.25)
        elif kind == "zeros":       # -0 and +0 are equal
            s.zero_()
            s[..., ::3] = -0.0
            s[..., ::50] = 1.0
        elif kind == "nan":
            s[..., 7::9] = float("nan")
            s[..., 3::11] = -float("nan")
        elif kind == "inf":
            s[..., 7::9] = float("inf")
            s[..., 4::9] = float("-inf")
        elif kind == "negative":
            s.sub_(1.2)
        else:                        # neighbours in the last bits only
            s.copy_((torch.arange(s.shape[-1], device="cuda", dtype=torch.int32).mul(7).remainder(251) + 0x3f000000).view(torch.float32).expand_as(s))
    check_evict(2, 64, 16, [300, 280], budget, 3, 9, make=make)


@pytest.mark.parametrize("n,budget", [(40000, 39999), (40000, 20000), (35841, 35000)])
def test_evict_rows_longer_than_shared_memory(n, budget):
    check_evict(1, 8, 64, [n], budget, 4, 100)


@pytest.mark.parametrize("inplace", [False, True])
def test_evict_short_rows_beside_one_longer_than_shared_memory(inplace):
    """More rows than several workgroups a row are for, most of them too short to give every wave a token."""
    def make(s):
        s.copy_((torch.arange(s.shape[-1], device="cuda") % 3).float().expand_as(s))
    check_evict(1, 8, 32, [33000] + [10, 60, 64, 1100] * 51 + [32769], 55, 4, 50, inplace=inplace, make=make)


@pytest.mark.parametrize("inplace", [False, True])
@pytest.mark.parametrize("kv,lens,budget,kind", [
    (2, [70001, 50000, 20000, 40000], 40000, "equal"),     # many parts a row; rows at, below and above the budget
    (1, [33000, 8192, 8193, 0], 8192, "few"),              # the border in few different weights, parts that end at the budget
    (3, [40961], 5, "distinct"),
    (1, [32769], 32768, "nan"),
    (1, [36000, 70], 0, "equal"),                          # nothing stays
    (1, [33000] + [10, 60, 64] * 68 + [32769], 55, "few"),   # more rows than several workgroups a row are for
])
def test_evict_rows_of_many_parts(kv, lens, budget, kind, inplace):
    def make(s):
        t = torch.arange(s.shape[-1], device="cuda")
        if kind == "equal":
            s.fill_(0.5)
        elif kind == "few":
            s.copy_((t % 3).float().expand_as(s))
        elif kind == "distinct":
            s.copy_(((t * 7919) % s.shape[-1]).float().expand_as(s))
        else:
            s.copy_(torch.where(t % 1000 == 3, float("nan"), -(t % 7).float()).expand_as(s))
    check_evict(kv, 8, 32, lens, budget, 4, 50, inplace=inplace, make=make)


@pytest.mark.parametrize("budget", [60, 300])
@pytest.mark.parametrize("longest", [190, 430, 2000, 4097, 9000, 20001, 32768, 33001])
def test_evict_rows_of_all_lengths_in_one_call(longest, budget):
    """Threads, waves and whole words of a workgroup without tokens; rows at, just above and far above the budget."""
    lens = [longest] + [n for n in (0, 1, 10, 60, 61, 63, 64, 65, 130, 257, 299, 300, 301, 304, 305, 511, 1100, 4095, 8200) if n <= longest]
    def make(s):
        s.copy_(((torch.arange(s.shape[-1], device="cuda") * 31) % 17).float().expand_as(s))
    check_evict(2, 8, 16, lens, budget, 4, 20, inplace=longest % 2 == 0, make=make)


def test_evict_pools_of_other_strides_and_a_count_that_is_far_ahead():
    assert check_evict(3, 72, 7, [100, 90], 40, 0, 20, order="tokens") > 0
    check_evict(2, 64, 16, [100], 60, 0, 2 ** 31 - 1, seen=[2 ** 31 - 1])


def test_evict_clamps_lengths():
    cache = B.Cache(B.make_cache_desc(4, 8, 1, 64))
    table = torch.arange(4, dtype=torch.int32, device="cuda").view(2, 2)
    lens = torch.tensor([1000, -5], dtype=torch.int32, device="cuda")
    score, pos = torch.rand((2, 1, 16), device="cuda"), torch.arange(16, device="cuda").int().expand(2, 1, 16).contiguous()
    want = U.evicted(score[0, 0].tolist(), pos[0, 0].tolist(), 16, 16, 10, 0, 0)
    s2 = score.clone()
    _, _, out = B.qeft_cache_evict(cache, table, lens, 1 << 20, 10, s2, pos, torch.tensor([16, 16], dtype=torch.int32, device="cuda"))
    assert out.tolist() == [10, 0] and pos[0, 0, :10].tolist() == want and torch.equal(s2[1], score[1])


def test_calls_without_the_native_module_give_the_same(monkeypatch):
    kv, d, page = 2, 64, 16
    lens = torch.tensor([100, 61], dtype=torch.int32, device="cuda")
    table = torch.randperm(14, device="cuda").int().view(2, 7)
    K, V, q = torch.randn((14, kv, page, d), device="cuda").half(), torch.randn((14, kv, page, d), device="cuda").half(), torch.randn((2, 4 * d), device="cuda").half()
    score0, pos0 = torch.rand((2, kv, 112), device="cuda"), torch.arange(112, device="cuda").int().expand(2, kv, 112).contiguous()
    rot = rotation(128, d)

    def all_of_it():
        cache = B.Cache(B.make_cache_desc(14, page, kv, d), k=K.clone(), v=V.clone())
        score, pos = score0.clone(), pos0.clone()
        q2 = B.qeft_cache_append(cache, table, q[:, : kv * d], q[:, kv * d:], lens, q=q, rot=rot)
        out = B.qeft_attn_decode(cache, table, lens + 1, 112, q2, score=score, accumulate=True)
        s, p, n = B.qeft_cache_evict(cache, table, lens + 1, 112, 50, score, pos, lens + 1, keep_first=4, keep_last=8)
        return [q2, out, s, p, n, cache.k, cache.v]

    native = all_of_it()
    with monkeypatch.context() as m:
        m.setattr(B, "_native", type("None_", (), {n: staticmethod(lambda *a: None) for n in dir(B._native) if not n.startswith("__")}))
        plain = all_of_it()
    for a, b in zip(native, plain):
        assert torch.equal(a, b)


@pytest.mark.parametrize("seqs,n,budget", [(3, 70, 67), (3, 150, 60), (3, 900, 500), (2, 33000, 20000), (700, 33000, 40)])
def test_evict_stores_nothing_in_pages_that_are_out_of_range(seqs, n, budget):
    """Few to go, moves by the workgroup itself, by a second launch, of rows by many workgroups and of long rows by one: slots freed in pages that are not the pool's."""
    kv, d, page = 1, 8, 10
    cols = -(-n // page)
    own, lens = min(seqs, 3), [n] * 3 + [5] * seqs
    lens, pages = lens[:seqs], own * cols + 2                     # (the first page and the last are no sequence's; short sequences, within the budget, name any)
    gen = torch.Generator(device="cuda").manual_seed(n)
    K, V = (torch.randn((pages, kv, page, d), generator=gen, device="cuda").half() for _ in range(2))
    table = torch.ones((seqs, cols), dtype=torch.int32, device="cuda")
    table[:own] = (1 + torch.randperm(own * cols, generator=gen, device="cuda")).int().view(own, cols)
    bad = torch.tensor([-1, pages, 2 ** 31 - 1, -2 ** 31], dtype=torch.int32, device="cuda")
    table[0, 0], table[1, 1:5] = bad[0], bad
    table[0, -1] = bad[0] if own > 1 else table[0, -1]            # and a source, which is read from the first page
    score = torch.rand((seqs, kv, n), generator=gen, device="cuda")
    score[:, :, : budget // 2] *= 0.1                             # most that go are in the first slots
    pos = torch.arange(n, device="cuda").int().expand(seqs, kv, n).contiguous()
    cache = B.Cache(B.make_cache_desc(pages, page, kv, d), k=K.clone(), v=V.clone())
    dev_lens = torch.tensor(lens, dtype=torch.int32, device="cuda")
    so, po = score.clone(), pos.clone()
    _, _, left = B.qeft_cache_evict(cache, table, dev_lens, n, budget, so, po, dev_lens)
    skipped = 0
    for b in range(own):
        at = torch.tensor(U.evicted(score[b, 0].tolist(), pos[b, 0].tolist(), n, n, budget, 0, 0), device="cuda")
        dst = torch.arange(budget, device="cuda")
        assert torch.equal(so[b, 0, :budget], score[b, 0, at]) and torch.equal(po[b, 0, :budget], pos[b, 0, at])
        to, src = table[b].long()[dst // page], table[b].long().clamp(0, pages - 1)[at // page]
        stored = (at != dst) & (to >= 0) & (to < pages)
        skipped += int(((at != dst) & ~stored).sum())
        for pool in (K, V):
            pool[to[stored], 0, dst[stored] % page] = pool[src[stored], 0, at[stored] % page]
    assert skipped > 0 and left.tolist() == [min(x, budget) for x in lens]
    assert torch.equal(cache.k, K) and torch.equal(cache.v, V)
