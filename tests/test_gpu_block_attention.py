"""qeft_attn_decode against the definition in 64 bits: head layouts, head and page sizes, lengths from none to many chunks, pools of other strides, slots
that were never written."""
import math

import pytest
import torch

import block_util as U
from paper_2410_08661_amd import binding as B

pytestmark = pytest.mark.gpu


def setup(heads, kv, d, page, lens, seed=0, order="pages", spare=3):
    gen = torch.Generator(device="cuda").manual_seed(seed + 1000 * heads + d)
    cols = max(1, -(-max(lens) // page)) + 1
    pages = len(lens) * cols + spare
    K, V = (U.pool_of(pages, kv, page, d, gen, order) for _ in range(2))
    table = torch.randperm(pages, generator=gen, device="cuda")[: len(lens) * cols].int().view(len(lens), cols)
    # slots at and behind a length hold not-a-number, and table entries of pages that no token uses anything
    t = torch.arange(cols * page, device="cuda").view(cols, page)
    for b, n in enumerate(lens):
        for i in range(cols):
            for pool in (K, V):
                pool[int(table[b, i])] = pool[int(table[b, i])].masked_fill((t[i] >= n)[None, :, None], float("nan"))
        used = -(-n // page)
        table[b, used:] = torch.tensor([-1, 2 ** 31 - 1, -2 ** 31, pages], device="cuda", dtype=torch.int32).repeat(cols)[: cols - used]
    s = K.stride()
    cache = B.Cache(B.make_cache_desc(pages, page, kv, d, s[0], s[1], s[2]), k=K, v=V)
    q = (torch.randn((len(lens), heads * d), generator=gen, device="cuda") * 1.5).half()
    return cache, table, torch.tensor(lens, dtype=torch.int32, device="cuda"), q


CASES = [
    (4, 4, 128, 16, [1, 31, 32, 33]),
    (8, 8, 64, 8, [0, 5, 257, 64]),
    (1, 1, 128, 16, [203]),
    (16, 4, 80, 16, [100, 513, 700]),
    (12, 2, 96, 32, [1000, 3]),
    (32, 1, 128, 64, [1500]),
    (20, 1, 256, 128, [300, 900]),
    (6, 6, 256, 16, [70, 600]),
    (10, 2, 248, 8, [530]),
    (8, 2, 128, 5, [44, 600]),
    (4, 4, 40, 1, [77]),
    (2, 2, 8, 3, [19, 1]),
    (64, 8, 128, 64, [4001]),
    (8, 1, 128, 256, [20011]),
    (51, 3, 64, 16, [900, 17]),
]


@pytest.mark.parametrize("heads,kv,d,page,lens", CASES)
def test_attention(heads, kv, d, page, lens):
    cache, table, dev_lens, q = setup(heads, kv, d, page, lens)
    want, weights, eo, ew = U.attention(cache.k, cache.v, table, lens, q, heads, d ** -0.5)
    longest = max(max(lens), 1)
    got = B.qeft_attn_decode(cache, table, dev_lens, longest, q)
    U.close("out", got, want, eo)
    score = torch.full((len(lens), kv, longest + 3), 7.0, device="cuda")
    got2 = B.qeft_attn_decode(cache, table, dev_lens, longest, q, score=score)
    U.close("out with weights", got2, want, eo)
    for b, n in enumerate(lens):
        U.close("weights", score[b, :, :n], weights[b, :, :n], ew[b, :, :n])
        assert bool((score[b, :, n:] == 7.0).all())
    before = score.clone()
    B.qeft_attn_decode(cache, table, dev_lens, longest, q, score=score, accumulate=True)
    for b, n in enumerate(lens):
        U.close("weights added", score[b, :, :n], 2 * weights[b, :, :n], 2 * ew[b, :, :n] + 2 * U.U * weights[b, :, :n])
        assert torch.equal(score[b, :, n:], before[b, :, n:])
    assert torch.equal(got, B.qeft_attn_decode(cache, table, dev_lens, longest, q))


@pytest.mark.parametrize("order", ["tokens", "heads"])
@pytest.mark.parametrize("page", [16, 7])
def test_pools_of_other_strides_and_pitches(order, page):
    lens = [130, 0, 45]
    cache, table, dev_lens, q = setup(8, 4, 72, page, lens, order=order)
    wide = torch.full((3, 8 * 72 + 24), float("nan"), dtype=torch.float16, device="cuda")
    wide[:, 8: 8 + 8 * 72] = q
    out = torch.full((3, 8 * 72 + 40), 9.0, dtype=torch.float16, device="cuda")
    want, _, eo, _ = U.attention(cache.k, cache.v, table, lens, q, 8, 0.3)
    B.qeft_attn_decode(cache, table, dev_lens, 130, wide[:, 8: 8 + 8 * 72], out=out[:, 16: 16 + 8 * 72], scale=0.3)
    U.close("out", out[:, 16: 16 + 8 * 72], want, eo)
    assert bool((out[:, :16] == 9).all()) and bool((out[:, 16 + 8 * 72:] == 9).all())


def test_lengths_are_cut_at_the_bound_and_at_the_table():
    cache, table, _, q = setup(4, 2, 64, 16, [100, 90])
    long = torch.tensor([5000, 90], dtype=torch.int32, device="cuda")
    want, _, eo, _ = U.attention(cache.k, cache.v, table, [64, 64], q, 4, 0.125)
    U.close("cut at the bound", B.qeft_attn_decode(cache, table, long, 64, q), want, eo)
    want, _, eo, _ = U.attention(cache.k, cache.v, table, [96, 90], q, 4, 0.125)
    U.close("cut at the table", B.qeft_attn_decode(cache, table[:, :6], long, 100000, q), want, eo)
    negative = torch.tensor([-3, 90], dtype=torch.int32, device="cuda")
    want, _, eo, _ = U.attention(cache.k, cache.v, table, [0, 90], q, 4, 0.125)
    U.close("below zero", B.qeft_attn_decode(cache, table, negative, 100, q), want, eo)
    assert not bool(B.qeft_attn_decode(cache, table, negative, 0, q).any())


def test_pages_out_of_range_are_clamped():
    cache, table, lens, q = setup(4, 2, 64, 16, [100, 90])
    cache.k.nan_to_num_(), cache.v.nan_to_num_()
    bad = table.clone()
    bad[0, 1], bad[1, 2], bad[1, 0] = -7, 2 ** 31 - 1, cache.desc.pages
    want, _, eo, _ = U.attention(cache.k, cache.v, bad, [100, 90], q, 4, 0.125)
    U.close("out", B.qeft_attn_decode(cache, bad, lens, 100, q), want, eo)


@pytest.mark.parametrize("scale", [100.0, -3.0, 0.0])
def test_steep_flat_and_negative_scales(scale):
    lens = [700, 1000]
    cache, table, dev_lens, q = setup(4, 4, 64, 16, lens)
    want, weights, eo, ew = U.attention(cache.k, cache.v, table, lens, q, 4, scale)
    score = torch.zeros((2, 4, 1000), device="cuda")
    U.close("out", B.qeft_attn_decode(cache, table, dev_lens, 1000, q, scale=scale, score=score), want, eo)
    U.close("weights", score[:, :, :700], weights[:, :, :700], ew[:, :, :700])


def test_scores_of_the_lowest_value():
    """A row of infinite negative scores beside finite ones has no weight, and the waves that meet only such rows nothing to add."""
    lens = [600]
    cache, table, dev_lens, q = setup(2, 2, 64, 16, lens)
    q.fill_(1.0)
    low = cache.k.clone()
    rows = table[0].long()
    t = torch.arange(600, device="cuda")
    dead = (t % 37 != 5)
    low[rows[t[dead] // 16], :, t[dead] % 16] = float("-inf")
    cache.k.copy_(low)
    score = torch.full((1, 2, 600), 3.0, device="cuda")
    out = B.qeft_attn_decode(cache, table, dev_lens, 600, q, score=score)
    alive = (~dead).nonzero()[:, 0]
    for h in range(2):
        k, v = (U.rows_of(p, table, 0, h, 600)[alive] for p in (cache.k, cache.v))
        p = torch.softmax(k.sum(1) / 8, 0)
        assert float((out[0, h * 64: (h + 1) * 64].double() - p @ v).abs().max()) <= 2e-3
        assert float((score[0, h, alive].double() - p).abs().max()) <= 1e-5
        assert not bool(score[0, h, dead].any())


def test_offsets_beyond_32_bits():
    """A pool of more than 2^32 bytes and 2^31 elements, its last pages in use."""
    kv, page, d = 8, 64, 128
    pages = (1 << 31) // (kv * page * d) + 40
    K, V = (torch.empty((pages, kv, page, d), dtype=torch.float16, device="cuda") for _ in range(2))
    gen = torch.Generator(device="cuda").manual_seed(5)
    table = torch.stack([torch.arange(pages - 16, pages, device="cuda"), torch.arange(16, device="cuda")]).int()
    for p in table.view(-1).tolist():
        for pool in (K, V):
            pool[p] = torch.randn((kv, page, d), generator=gen, device="cuda").half()
    cache = B.Cache(B.make_cache_desc(pages, page, kv, d), k=K, v=V)
    q = torch.randn((2, 16 * d), generator=gen, device="cuda").half()
    lens = [1000, 1024]
    want, _, eo, _ = U.attention(K, V, table, lens, q, 16, d ** -0.5)
    U.close("out", B.qeft_attn_decode(cache, table, torch.tensor(lens, dtype=torch.int32, device="cuda"), 1024, q), want, eo)


def test_replayed_from_a_graph_on_another_stream():
    lens = [900, 40]
    cache, table, dev_lens, q = setup(8, 2, 128, 16, lens)
    score, out = torch.zeros((2, 2, 1000), device="cuda"), torch.empty_like(q)
    ws = torch.empty(B.qeft_attn_workspace(cache.desc, 2, 8, 1000, True), dtype=torch.uint8, device="cuda")
    B.qeft_attn_decode(cache, table, dev_lens, 1000, q, out=out, score=score, ws=ws)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=torch.cuda.Stream()):
        B.qeft_attn_decode(cache, table, dev_lens, 1000, q, out=out, score=score, ws=ws)
    for i in range(4):
        q.normal_()
        dev_lens.copy_(torch.tensor([900 - 100 * i, 40 + i], dtype=torch.int32))
        cache.k.nan_to_num_(), cache.v.nan_to_num_()
        score.zero_()
        ws.fill_(255)                       # whatever a workspace holds
        g.replay()
        torch.cuda.synchronize()
        s2 = torch.zeros_like(score)
        want = B.qeft_attn_decode(cache, table, dev_lens, 1000, q, score=s2)
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(score, s2)


@pytest.mark.parametrize("kv,seqs", [(1, 1), (2, 1), (2, 2)])
def test_rows_of_weights_narrower_than_the_tokens_are_refused(kv, seqs):
    d, page, n = 64, 8, 32
    gen = torch.Generator(device="cuda").manual_seed(kv + 10 * seqs)
    K, V = (U.pool_of(4 * seqs, kv, page, d, gen) for _ in range(2))
    cache = B.Cache(B.make_cache_desc(4 * seqs, page, kv, d), k=K, v=V)
    table = torch.arange(4 * seqs, dtype=torch.int32, device="cuda").view(seqs, 4)
    lens = torch.full((seqs,), n, dtype=torch.int32, device="cuda")
    q = torch.randn((seqs, kv * d), generator=gen, device="cuda").half()
    base = torch.full((seqs, kv, 64), 7.0, device="cuda")
    pos = torch.arange(64, dtype=torch.int32, device="cuda").expand(seqs, kv, 64).contiguous()
    for width in (29, 31):
        with pytest.raises(B.QeftError) as e:
            B.qeft_attn_decode(cache, table, lens, n, q, score=base[:, :, :width])
        assert e.value.status == B.QEFT_ERR_SHAPE
        with pytest.raises(B.QeftError) as e:
            B.qeft_cache_evict(cache, table, lens, n, 16, base[:, :, :width], pos[:, :, :width], lens)
        assert e.value.status == B.QEFT_ERR_SHAPE
        with pytest.raises(B.QeftError) as e:
            B.qeft_cache_evict(cache, table, lens, n, 30, base, pos, lens, score_out=base.clone()[:, :, :29], pos_out=pos.clone()[:, :, :29])
        assert e.value.status == B.QEFT_ERR_SHAPE
    assert (base == 7.0).all()
    B.qeft_attn_decode(cache, table, lens, n, q, score=base[:, :, :n])
    torch.testing.assert_close(base[:, :, :n].sum(2), torch.ones((seqs, kv), device="cuda"), rtol=0, atol=n * 2.0 ** -20)
    assert (base[:, :, n:] == 7.0).all()


@pytest.mark.parametrize("heads,kv,d,page,lens", [
    (4, 4, 128, 16, [1, 31, 32, 0, 17]),
    (40, 2, 72, 5, [32, 9]),            # two tiles of heads
    (32, 1, 64, 8, [6, 32, 1]),
    (12, 2, 256, 8, [20, 0, 32, 3]),
    (5, 1, 200, 7, [30, 11]),
    (64, 64, 64, 16, [64, 33, 32, 63] * 4),
    (32, 32, 256, 32, [50, 1, 64, 40] * 8),
    (96, 32, 80, 24, [64, 60, 0, 33] * 8),
])
def test_short_rows(heads, kv, d, page, lens):
    test_attention(heads, kv, d, page, lens)


@pytest.mark.parametrize("heads,kv,d,page,lens", [
    (64, 8, 128, 16, [1400, 0, 33, 700, 1, 1399, 640, 128] * 2),       # one chunk of eight waves a row
    (32, 32, 64, 16, [800, 30, 799]),
    (96, 32, 96, 8, [1100, 257, 600, 4]),
    (64, 8, 128, 16, [2900, 100, 513, 1664] + [70] * 9),                # four chunks, three, ...
    (16, 16, 256, 32, [600, 280, 31, 599, 1, 64, 65, 0]),
])
def test_rows_that_half_fill_the_gpu(heads, kv, d, page, lens):
    test_attention(heads, kv, d, page, lens)


@pytest.mark.parametrize("kv,lens", [(64, [2048] * 7 + [1500]), (1, [20001])])
@pytest.mark.parametrize("below", [31.01, 30.2, 25.3, 20.5])
def test_many_tokens_of_little_weight_beside_one_of_much(below, kv, lens):
    """The first token has nearly all the weight and nothing in half of its value's channels; the others, 2^-below of its weight each, are what those channels hold."""
    d, page = 8, 16
    cache, table, dev_lens, q = setup(kv, kv, d, page, lens)
    q.fill_(1.0)
    gen = torch.Generator(device="cuda").manual_seed(11)
    cache.k.masked_fill_(cache.k == cache.k, 0.0)                                    # (slots that were never written stay not-a-number)
    cache.v.copy_(torch.where(cache.v == cache.v, (torch.rand(cache.v.shape, generator=gen, device="cuda") * 4096 + 4096).half(), cache.v))
    for b in range(len(lens)):
        cache.k[int(table[b, 0]), :, 0] = 1.0
        cache.v[int(table[b, 0]), :, 0] = torch.tensor([0.0] * 4 + [1.0] * 4, device="cuda").half()
    scale = below * math.log(2.0) / d
    want, weights, eo, ew = U.attention(cache.k, cache.v, table, lens, q, kv, scale)
    score = torch.zeros((len(lens), kv, max(lens)), device="cuda")
    got = B.qeft_attn_decode(cache, table, dev_lens, max(lens), q, scale=scale, score=score)
    # beside the bound of ordinary rows: half a step of fp16's smallest numbers for each token, against a largest of 2^14 or more
    U.close("out", got, want, eo + max(lens) * 2.0 ** -39 * 8192)
    for b, n in enumerate(lens):
        U.close("weights", score[b, :, :n], weights[b, :, :n], ew[b, :, :n])


@pytest.mark.parametrize("heads,kv,lens", [(4, 4, [300, 33]), (16, 2, [5000, 64])])
@pytest.mark.parametrize("power", [24, 25, 26, 27, 28, 30])
def test_scores_far_beyond_the_exponents_reach(power, heads, kv, lens):
    """Scores of 2^power in log2, where fp32 has steps of 2 to 128: equal ones share the weight, of distant ones the largest has it all."""
    d = 64
    cache, table, dev_lens, q = setup(heads, kv, d, 16, lens)
    longest = max(lens)
    for odd in (1.0, 1.25, 1.75):
        q.fill_(odd)
        scale = math.log(2.0) * 2.0 ** power / d
        score = torch.zeros((len(lens), kv, longest), device="cuda")
        cache.k.copy_(torch.where(cache.k == cache.k, 1.0, cache.k))
        got = B.qeft_attn_decode(cache, table, dev_lens, longest, q, scale=scale, score=score)
        for b, n in enumerate(lens):
            for h in range(heads):
                v = U.rows_of(cache.v, table, b, h * kv // heads, n)
                bound = U.HALF * v.mean(0).abs() + U.TINY + (n / 32 + 64 + d) * U.U * v.abs().mean(0) + 2.0 ** -20 * v.abs().mean(0)
                U.close("mean", got[b, h * d: (h + 1) * d], v.mean(0), bound)
            U.close("weights", score[b, :, :n], torch.full((kv, n), heads / kv / n, dtype=torch.float64, device="cuda"), (n / 32 + 64) * U.U * heads / kv / n)
        # every 7th token's keys half as large again as its neighbours', the last of all twice
        cache.k.copy_(torch.where(cache.k == cache.k, 1.0 + 0.5 * (torch.arange(16, device="cuda")[:, None] % 7 == 3), cache.k))
        for b, n in enumerate(lens):
            cache.k[int(table[b, (n - 1) // 16]), :, (n - 1) % 16] = 2.0
        got = B.qeft_attn_decode(cache, table, dev_lens, longest, q, scale=scale, score=score)
        for b, n in enumerate(lens):
            last = torch.stack([cache.v[int(table[b, (n - 1) // 16]), h * kv // heads, (n - 1) % 16] for h in range(heads)])
            assert torch.equal(got[b].view(heads, d), last)
            assert bool((score[b, :, n - 1] == heads / kv).all()) and not bool(score[b, :, : n - 1].any())
