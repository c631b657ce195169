"""What the calls between the linear layers refuse, and their workspaces: host checks only, no GPU needed."""
import ctypes as C

import pytest
import torch

from paper_2410_08661_amd import binding as B

P = 0x100000     # an address that nothing reads: every call below ends before a launch


def cache_args(seqs=2, cols=4, **over):
    d = B.make_cache_desc(8, 16, 4, 64)
    for k, v in over.items():
        setattr(d, k, v)
    return d, B.qeft_cache_t(P, P), B.qeft_table_t(P, cols, cols, seqs)


def call(fn, d, pools, table, a):
    ref = lambda x: None if x is None else C.byref(x)  # noqa: E731
    return fn(ref(d), ref(pools), ref(table), ref(a), None)


def attn(**over):
    f = dict(lens=P, longest=64, q=P, out=P, ldq=512, ldo=512, heads=8, scale=1.0, score=0, ld_score=0, accumulate=0, ws=0, ws_bytes=0)
    return B.qeft_attn_t(**{**f, **over})


def append(**over):
    f = dict(q=P, k=P, v=P, q_out=P, ldq=512, ldq_out=512, ldk=256, ldv=256, seq=P, index=P, pos=P, rot=P, ld_rot=64, positions=9, rot_dim=64, heads=8, tokens=3)
    return B.qeft_append_t(**{**f, **over})


def evict(**over):
    f = dict(lens=P, seen=P, longest=64, budget=63, score=P, pos=2 * P, ld=64, keep_first=0, keep_last=0, score_out=3 * P, pos_out=4 * P, ld_out=64, lens_out=5 * P, ws=0, ws_bytes=0)
    return B.qeft_evict_t(**{**f, **over})


@pytest.mark.parametrize("over,status", [
    (dict(pages=0), B.QEFT_ERR_SHAPE), (dict(page_size=0), B.QEFT_ERR_SHAPE), (dict(kv_heads=-1), B.QEFT_ERR_SHAPE), (dict(head_dim=0), B.QEFT_ERR_SHAPE),
    (dict(head_dim=264), B.QEFT_ERR_SHAPE), (dict(head_dim=60), B.QEFT_ERR_UNSUPPORTED), (dict(token_stride=56), B.QEFT_ERR_SHAPE),
    (dict(head_stride=-8), B.QEFT_ERR_SHAPE), (dict(page_stride=4100), B.QEFT_ERR_ALIGN)])
def test_caches_that_are_refused(over, status):
    d, pools, table = cache_args(**over)
    assert call(B.raw.qeft_attn_decode, d, pools, table, attn()) == status
    assert call(B.raw.qeft_cache_append, d, pools, table, append()) == status
    assert call(B.raw.qeft_cache_evict, d, pools, table, evict()) == status
    assert B.qeft_attn_workspace(d, 2, 8, 4096, True) == 0 and B.qeft_evict_workspace(d, 2, 4096, 100) == 0


@pytest.mark.parametrize("fn,make", [(B.raw.qeft_attn_decode, attn), (B.raw.qeft_cache_append, append), (B.raw.qeft_cache_evict, evict)])
def test_missing_and_misaligned_structs(fn, make):
    d, pools, table = cache_args()
    for args in ((None, pools, table, make()), (d, None, table, make()), (d, pools, None, make()), (d, pools, table, None),
                 (d, B.qeft_cache_t(0, P), table, make()), (d, B.qeft_cache_t(P, 0), table, make()), (d, pools, B.qeft_table_t(0, 4, 4, 2), make())):
        assert call(fn, *args) == B.QEFT_ERR_NULL
    assert call(fn, d, B.qeft_cache_t(P + 8, P), table, make()) == B.QEFT_ERR_ALIGN
    assert call(fn, d, pools, B.qeft_table_t(P + 2, 4, 4, 2), make()) == B.QEFT_ERR_ALIGN
    for table in (B.qeft_table_t(P, 3, 4, 2), B.qeft_table_t(P, 4, -1, 2), B.qeft_table_t(P, 4, 4, -1)):
        assert call(fn, d, pools, table, make()) == B.QEFT_ERR_SHAPE


@pytest.mark.parametrize("over,status", [
    (dict(heads=6), B.QEFT_ERR_SHAPE), (dict(heads=0), B.QEFT_ERR_SHAPE), (dict(longest=-1), B.QEFT_ERR_SHAPE), (dict(longest=1 << 25), B.QEFT_ERR_SHAPE),
    (dict(ldq=504), B.QEFT_ERR_SHAPE), (dict(ldo=516), B.QEFT_ERR_ALIGN), (dict(q=0), B.QEFT_ERR_NULL), (dict(out=0), B.QEFT_ERR_NULL), (dict(q=P + 8), B.QEFT_ERR_ALIGN),
    (dict(lens=0), B.QEFT_ERR_NULL), (dict(lens=P + 2), B.QEFT_ERR_ALIGN), (dict(score=P, ld_score=63), B.QEFT_ERR_SHAPE), (dict(score=P + 1, ld_score=64), B.QEFT_ERR_ALIGN),
    (dict(score=P, ld_score=64), B.QEFT_ERR_WORKSPACE), (dict(score=P, ld_score=64, ws=P, ws_bytes=100), B.QEFT_ERR_WORKSPACE),
    (dict(score=P, ld_score=64, ws=P + 8, ws_bytes=1 << 30), B.QEFT_ERR_ALIGN)])
def test_attention_refuses(over, status):
    d, pools, table = cache_args()
    assert call(B.raw.qeft_attn_decode, d, pools, table, attn(**over)) == status


def test_attention_workspace():
    d, pools, table = cache_args(cols=1000)
    assert B.qeft_attn_workspace(d, 2, 8, 200) == 0                      # one chunk, one launch
    need = B.qeft_attn_workspace(d, 2, 8, 16000)
    assert need > 0
    assert call(B.raw.qeft_attn_decode, d, pools, table, attn(longest=16000)) == B.QEFT_ERR_WORKSPACE
    assert call(B.raw.qeft_attn_decode, d, pools, table, attn(longest=16000, ws=P, ws_bytes=need - 1)) == B.QEFT_ERR_WORKSPACE
    assert B.qeft_attn_workspace(d, 2, 8, 16000, True) >= need + 2 * 8 * 16000 * 4
    # the bound counts, also where the table holds less
    assert call(B.raw.qeft_attn_decode, d, pools, B.qeft_table_t(P, 1000, 2, 2), attn(longest=16000, ws=P, ws_bytes=need - 1)) == B.QEFT_ERR_WORKSPACE
    assert B.qeft_attn_workspace(d, 1 << 23, 8, 100) == 0 and B.qeft_attn_workspace(d, 1, 8, -1) == 0 and B.qeft_attn_workspace(d, 0, 8, 100000) == 0


@pytest.mark.parametrize("over,status", [
    (dict(tokens=-1), B.QEFT_ERR_SHAPE), (dict(rot_dim=66), B.QEFT_ERR_SHAPE), (dict(rot_dim=31), B.QEFT_ERR_UNSUPPORTED), (dict(rot_dim=-2), B.QEFT_ERR_SHAPE),
    (dict(ldk=248), B.QEFT_ERR_SHAPE), (dict(ldv=260), B.QEFT_ERR_ALIGN), (dict(k=0), B.QEFT_ERR_NULL), (dict(v=0), B.QEFT_ERR_NULL), (dict(q_out=0), B.QEFT_ERR_NULL),
    (dict(heads=0), B.QEFT_ERR_SHAPE), (dict(ldq_out=8), B.QEFT_ERR_SHAPE), (dict(index=0), B.QEFT_ERR_NULL), (dict(index=P + 1), B.QEFT_ERR_ALIGN), (dict(seq=0), B.QEFT_ERR_SHAPE),
    (dict(rot=0), B.QEFT_ERR_NULL), (dict(positions=0), B.QEFT_ERR_SHAPE), (dict(ld_rot=60), B.QEFT_ERR_SHAPE), (dict(rot=P + 2), B.QEFT_ERR_ALIGN)])
def test_append_refuses(over, status):
    d, pools, table = cache_args()
    assert call(B.raw.qeft_cache_append, d, pools, table, append(**over)) == status
    assert call(B.raw.qeft_cache_append, d, pools, table, append(tokens=0, k=0, v=0, q=0, index=0)) == B.QEFT_OK


@pytest.mark.parametrize("over,status", [
    (dict(longest=-1), B.QEFT_ERR_SHAPE), (dict(budget=-1), B.QEFT_ERR_SHAPE), (dict(ld=63), B.QEFT_ERR_SHAPE), (dict(ld_out=62), B.QEFT_ERR_SHAPE), (dict(keep_first=-1), B.QEFT_ERR_SHAPE),
    (dict(keep_last=-1), B.QEFT_ERR_SHAPE), (dict(lens=0), B.QEFT_ERR_NULL), (dict(seen=0), B.QEFT_ERR_NULL), (dict(lens_out=0), B.QEFT_ERR_NULL), (dict(score=0), B.QEFT_ERR_NULL),
    (dict(pos_out=0), B.QEFT_ERR_NULL), (dict(pos=P + 2), B.QEFT_ERR_ALIGN), (dict(lens_out=P), B.QEFT_ERR_UNSUPPORTED), (dict(lens_out=P + 4), B.QEFT_ERR_UNSUPPORTED),
    (dict(seen=5 * P), B.QEFT_ERR_UNSUPPORTED), (dict(score_out=P + 64), B.QEFT_ERR_UNSUPPORTED), (dict(pos_out=3 * P + 4), B.QEFT_ERR_UNSUPPORTED),
    (dict(score_out=2 * P), B.QEFT_ERR_UNSUPPORTED), (dict(score_out=P, ld_out=72), B.QEFT_ERR_SHAPE), (None, B.QEFT_ERR_WORKSPACE)])
def test_evict_refuses(over, status):
    d, pools, table = cache_args()
    if over is None:        # more moves than the first launch makes: the lists need a workspace
        d, pools, table = cache_args(cols=100)
        need = B.qeft_evict_workspace(d, 2, 1000, 500)
        assert need >= 2 * 4 * 1000 / 8 and B.qeft_evict_workspace(d, 2, 1000, 999) == 0 == B.qeft_evict_workspace(d, 2, 1000, 1000)
        a = evict(longest=1000, budget=500, ld=1000, ld_out=1000, ws=P, ws_bytes=need - 1)
        assert call(B.raw.qeft_cache_evict, d, pools, table, a) == status
        return
    assert call(B.raw.qeft_cache_evict, d, pools, table, evict(**over)) == status


def norm_desc(**over):
    d = B.make_norm_desc(64, torch.float32, B.QEFT_GATE_CHANNEL)
    for k, v in over.items():
        setattr(d, k, v)
    return d


def nfwd(**over):
    f = dict(r=P, y=P, gate=P, w_pre=P, w_post=P, h=P, x=P, ldr=64, ldy=64, ldg=64, ldh=64, ldx=64, m=5)
    return B.qeft_norm_fwd_t(**{**f, **over})


def nbwd(**over):
    f = dict(dx=P, dh=P, h=P, y=P, gate=P, w_pre=P, w_post=P, dr=P, dy=P, dgate=P, dw_pre=P, dw_post=P, lddx=64, lddh=64, ldh=64, ldy=64, ldg=64, lddr=64, lddy=64, lddg=64, m=5, accumulate=0,
             ws=0, ws_bytes=0)
    return B.qeft_norm_bwd_t(**{**f, **over})


@pytest.mark.parametrize("desc,over,status", [
    (dict(n=0), {}, B.QEFT_ERR_SHAPE), (dict(n=1 << 25), {}, B.QEFT_ERR_SHAPE), (dict(residual_dtype=5), {}, B.QEFT_ERR_UNSUPPORTED), (dict(gate=3), {}, B.QEFT_ERR_UNSUPPORTED),
    (dict(eps=-1.0), {}, B.QEFT_ERR_SHAPE), (dict(eps=float("nan")), {}, B.QEFT_ERR_SHAPE),
    ({}, dict(m=-1), B.QEFT_ERR_SHAPE), ({}, dict(ldy=56), B.QEFT_ERR_SHAPE), ({}, dict(ldh=68), B.QEFT_ERR_ALIGN), ({}, dict(y=P + 2), B.QEFT_ERR_ALIGN), ({}, dict(w_pre=0), B.QEFT_ERR_NULL),
    ({}, dict(w_post=P + 2), B.QEFT_ERR_ALIGN), ({}, dict(gate=0), B.QEFT_ERR_NULL), (dict(gate=0), {}, B.QEFT_ERR_UNSUPPORTED), (dict(gate=2), dict(ldg=8), B.QEFT_ERR_SHAPE)])
def test_norms_refuse(desc, over, status):
    d = norm_desc(**desc)
    assert B.raw.qeft_norm_fwd(C.byref(d), C.byref(nfwd(**over)), None) == status
    assert B.raw.qeft_norm_bwd(C.byref(d), C.byref(nbwd(**over)), None) == status
    if desc and "gate" not in desc:
        assert B.qeft_norm_workspace(d, 5) == 0


def test_norms_refuse_more():
    d = norm_desc()
    assert B.raw.qeft_norm_fwd(C.byref(d), C.byref(nfwd(y=0, gate=0, w_post=0)), None) == B.QEFT_ERR_UNSUPPORTED      # h without anything added
    assert B.raw.qeft_norm_fwd(C.byref(d), C.byref(nfwd(y=0, h=0, gate=0)), None) == B.QEFT_ERR_NULL                  # a norm of nothing
    assert B.raw.qeft_norm_fwd(C.byref(d), C.byref(nfwd(x=0)), None) == B.QEFT_ERR_NULL
    assert B.raw.qeft_norm_fwd(C.byref(d), C.byref(nfwd(m=0, r=0, x=0)), None) == B.QEFT_OK
    assert B.raw.qeft_norm_fwd(None, C.byref(nfwd()), None) == B.raw.qeft_norm_bwd(C.byref(d), None, None) == B.QEFT_ERR_NULL
    need = B.qeft_norm_workspace(d, 5)
    assert need > 0
    assert B.raw.qeft_norm_bwd(C.byref(d), C.byref(nbwd()), None) == B.QEFT_ERR_WORKSPACE
    assert B.raw.qeft_norm_bwd(C.byref(d), C.byref(nbwd(ws=P, ws_bytes=need - 1)), None) == B.QEFT_ERR_WORKSPACE
    assert B.raw.qeft_norm_bwd(C.byref(d), C.byref(nbwd(ws=P + 4, ws_bytes=need)), None) == B.QEFT_ERR_ALIGN
    for over in (dict(w_post=0), dict(y=0, w_post=0, gate=0, dgate=0)):     # gradients of what is not there
        assert B.raw.qeft_norm_bwd(C.byref(d), C.byref(nbwd(ws=P, ws_bytes=need, **over)), None) == B.QEFT_ERR_NULL
    long = norm_desc(n=20000)
    wide = {k: 20000 for k in ("lddx", "lddh", "ldh", "ldy", "ldg", "lddr", "lddy", "lddg")}
    assert B.raw.qeft_norm_bwd(C.byref(long), C.byref(nbwd(dw_pre=0, dw_post=0, dgate=0, **wide)), None) == B.QEFT_ERR_WORKSPACE


def test_the_binding_refuses_tensors_that_do_not_fit():
    d = B.make_cache_desc(4, 8, 2, 64)
    cache = B.Cache(d, device="cpu")
    table, lens, q = torch.zeros((1, 4), dtype=torch.int32), torch.zeros(1, dtype=torch.int32), torch.zeros((1, 128), dtype=torch.float16)
    with pytest.raises(B.QeftError) as e:      # host memory
        B.qeft_attn_decode(cache, table, lens, 8, q)
    assert e.value.status == B.QEFT_ERR_UNSUPPORTED
    for bad in (torch.zeros((4, 2, 8, 72), dtype=torch.float16), torch.zeros((4, 2, 8, 64)), torch.zeros((4, 8, 2, 64), dtype=torch.float16).transpose(1, 2)):
        with pytest.raises(B.QeftError) as e:
            B.Cache(d, k=bad, v=cache.v)
        assert e.value.status == B.QEFT_ERR_SHAPE
    n = B.make_norm_desc(64, torch.float16)
    r, w = torch.zeros((2, 64), dtype=torch.float16), torch.ones(64, dtype=torch.float16)
    for args, status in (((r.float(), w), B.QEFT_ERR_UNSUPPORTED), ((r[:, :32], w), B.QEFT_ERR_SHAPE), ((r, w), B.QEFT_ERR_UNSUPPORTED)):
        with pytest.raises(B.QeftError) as e:
            B.qeft_norm_fwd(n, *args, x=r)
        assert e.value.status == status
    with pytest.raises(B.QeftError) as e:
        B.qeft_norm_bwd(n, r, r, None, ws=torch.zeros(4096, dtype=torch.uint8))
    assert e.value.status in (B.QEFT_ERR_NULL, B.QEFT_ERR_UNSUPPORTED)


def test_rows_of_weights_hold_the_tokens_whatever_their_pitch():
    for t in (torch.zeros((1, 1, 5)), torch.zeros((2, 2, 16))[:, :, :5], torch.zeros((2, 2, 0))):   # (a single row's pitch counts in eights; a view's is its base's)
        with pytest.raises(B.QeftError) as e:
            B._take("f", "score", t, torch.float32, (t.shape[0], t.shape[1], None), True, 6)
        assert e.value.status == B.QEFT_ERR_SHAPE


def test_the_workspace_of_an_eviction_does_not_shrink_with_the_bound():
    for rows in (1, 2, 64, 204, 205, 3000):
        d = B.make_cache_desc(4, 8, rows, 8)
        bounds = (0, 100, 128, 229, 1000, 32768, 32769, 40960, 40961, 131072, 1 << 18, 1 << 19)
        sizes = [B.qeft_evict_workspace(d, 1, n, 100) for n in bounds if rows * (n // 128 + 1) <= 4 << 21]   # (more are refused)
        assert sizes == sorted(sizes) and sizes[2] == 0 < sizes[4]
        assert B.qeft_evict_workspace(d, 0, 40000, 100) == 0
