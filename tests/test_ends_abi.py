"""What the calls at the ends of a step refuse, their workspaces and plans: host checks only, no GPU needed."""
import ctypes as C
import math
import struct

import pytest
import torch

from paper_2410_08661_amd import binding as B

P = 0x100000     # an address that nothing reads: every call below ends before a launch
NULL, SHAPE, ALIGN, WORKSPACE, UNSUPPORTED = B.QEFT_ERR_NULL, B.QEFT_ERR_SHAPE, B.QEFT_ERR_ALIGN, B.QEFT_ERR_WORKSPACE, B.QEFT_ERR_UNSUPPORTED
MUCH = 1 << 40


def ref(x):
    return None if x is None else C.byref(x)


def struct_of(kind, base, over):
    return kind(**{**base, **over})


def lfwd(**over):
    return struct_of(B.qeft_logprob_fwd_t, dict(z=P, token=P, logp=P, lse=P, entropy=P, top_logp=P, top_index=P, ldz=104, ld_top=5, m=3, top=5, ws=P, ws_bytes=MUCH), over)


def lbwd(**over):
    return struct_of(B.qeft_logprob_bwd_t, dict(z=P, token=P, lse=P, entropy=P, dlogp=P, dlse=P, dentropy=P, dz=2 * P, ldz=104, lddz=104, m=3), over)


LDESC = B.make_logprob_desc(100)


def fwd(desc=LDESC, **over):
    return B.raw.qeft_logprob_fwd(ref(desc), ref(lfwd(**over)), None)


def bwd(desc=LDESC, **over):
    return B.raw.qeft_logprob_bwd(ref(desc), ref(lbwd(**over)), None)


def both(desc=LDESC, f={}, **over):
    return B.raw.qeft_logprob_fwd_bwd(ref(desc), ref(lfwd(**{**dict(top=0, top_logp=0, top_index=0), **f})), ref(lbwd(**over)), None)


@pytest.mark.parametrize("desc,status", [
    (None, NULL), (B.qeft_logprob_desc_t(0, 0, 1.0), SHAPE), (B.qeft_logprob_desc_t(1 << 25, 0, 1.0), SHAPE), (B.qeft_logprob_desc_t(100, 2, 1.0), UNSUPPORTED),
    (B.qeft_logprob_desc_t(100, 0, 0.0), SHAPE), (B.qeft_logprob_desc_t(100, 0, -1.0), SHAPE), (B.qeft_logprob_desc_t(100, 0, math.nan), SHAPE), (B.qeft_logprob_desc_t(100, 0, math.inf), SHAPE)])
def test_descriptions_of_logits(desc, status):
    assert fwd(desc) == bwd(desc) == both(desc) == status
    assert B.raw.qeft_logprob_workspace(ref(desc), 3, 5) == 0


@pytest.mark.parametrize("over,status", [
    (dict(m=-1), SHAPE), (dict(m=(1 << 21) + 1), SHAPE), (dict(top=-1), SHAPE), (dict(top=65, ld_top=65), SHAPE), (dict(z=0), NULL), (dict(ldz=96), SHAPE), (dict(ldz=108), ALIGN),
    (dict(z=P + 8), ALIGN), (dict(token=0), NULL), (dict(token=P + 2), ALIGN), (dict(logp=P + 1), ALIGN), (dict(lse=P + 2), ALIGN), (dict(entropy=P + 2), ALIGN), (dict(top_logp=0), NULL),
    (dict(top_index=0), NULL), (dict(top_index=P + 2), ALIGN), (dict(ld_top=4), SHAPE), (dict(top=0), SHAPE), (dict(top=0, top_logp=0), SHAPE)])
def test_log_probabilities_refuse(over, status):
    assert fwd(**over) == status


def test_more_alternatives_than_entries():
    assert fwd(B.make_logprob_desc(4), ldz=8) == SHAPE
    assert fwd(m=0, z=0, token=0) == 0 == bwd(m=0, z=0, dz=0, lse=0) and B.raw.qeft_logprob_fwd(ref(LDESC), None, None) == NULL


@pytest.mark.parametrize("over,status", [
    (dict(m=-1), SHAPE), (dict(z=0), NULL), (dict(dz=0), NULL), (dict(lse=0), NULL), (dict(entropy=0), NULL), (dict(token=0), NULL), (dict(lddz=96), SHAPE), (dict(lddz=100), ALIGN),
    (dict(dz=P + 4), ALIGN), (dict(dlogp=P + 2), ALIGN), (dict(dlse=P + 2), ALIGN), (dict(dentropy=P + 2), ALIGN), (dict(lse=P + 2), ALIGN), (dict(dz=P, lddz=112), SHAPE)])
def test_gradients_of_logits_refuse(over, status):
    assert bwd(**over) == status
    if "lse" not in over and "entropy" not in over and "z" not in over:
        f = {k: v for k, v in over.items() if k == "token"}
        assert both(f={**f, **(dict(logp=0) if f else {})}, **over) == status


def test_one_call_refuses():
    assert both(f=dict(top=5, top_logp=P, top_index=P)) == UNSUPPORTED
    assert both(m=4) == SHAPE and B.raw.qeft_logprob_fwd_bwd(ref(LDESC), None, ref(lbwd()), None) == NULL
    assert B.raw.qeft_logprob_fwd_bwd(ref(LDESC), ref(lfwd(top=0, top_logp=0, top_index=0)), None, None) == NULL


def test_workspaces_of_log_probabilities():
    for n in (1, 100, 32000, 131072, 1 << 24):
        for f32 in (torch.float16, torch.float32):
            d = B.make_logprob_desc(n, f32)
            for m in (1, 2, 64, 1000, 1 << 21):
                for top in (0, 1, 64):
                    if top > n:
                        continue
                    need = B.qeft_logprob_workspace(d, m, top)
                    assert 0 <= need < 1 << 30
                    if need:
                        a = lfwd(ldz=n + 7 & ~7, m=m, top=top, ld_top=64, ws_bytes=need - 1, **({} if top else dict(top_logp=0, top_index=0)))
                        assert B.raw.qeft_logprob_fwd(ref(d), ref(a), None) == WORKSPACE
                        a.ws, a.ws_bytes = P + 8, need
                        assert B.raw.qeft_logprob_fwd(ref(d), ref(a), None) == ALIGN
                        a.ws = 0
                        assert B.raw.qeft_logprob_fwd(ref(d), ref(a), None) == WORKSPACE
    assert B.qeft_logprob_workspace(LDESC, -1) == B.qeft_logprob_workspace(LDESC, 3, 65) == 0


def test_a_workspace_for_more_does_for_less():
    for n in (100, 65537, 98305, 130001, 140001, 262144, 1 << 20, 1 << 24):
        for kind in (torch.float16, torch.float32):
            d = B.make_logprob_desc(n, kind)
            for top in (0, 1, 20, 64):
                sizes = [B.qeft_logprob_workspace(d, m, top) for m in (*range(1, 300), 1000, 5000, 30000, 60000, 64000, 64100, 100000, 1 << 21)]
                assert sizes == sorted(sizes), (n, kind, top)
            for m in (1, 57, 300, 64100, 1 << 21):
                sizes = [B.qeft_logprob_workspace(d, m, top) for top in range(65)]
                assert sizes == sorted(sizes), (n, kind, m)
    for d in (qdesc(), qdesc(head_dim=128, rot_dim=128), qdesc(head_dim=256, rot_dim=2)):
        sizes = [B.qeft_qk_norm_workspace(d, m) for m in (*range(1, 300), 4096, 1 << 21)]
        assert sizes == sorted(sizes)


def qdesc(**over):
    return struct_of(B.qeft_qk_desc_t, dict(head_dim=64, heads=4, kv_heads=2, rot_dim=32, eps=1e-6), over)


def qfwd(**over):
    return struct_of(B.qeft_qk_fwd_t, dict(q=P, k=P, w_q=P, w_k=P, q_out=2 * P, k_out=2 * P, pos=P, rot=P, ldq=256, ldk=128, ldq_out=256, ldk_out=128, ld_rot=32, m=3, positions=9), over)


def qbwd(**over):
    f = dict(gq=P, gk=P, q=P, k=P, w_q=P, w_k=P, dq=2 * P, dk=2 * P, dw_q=P, dw_k=2 * P, pos=P, rot=P, ldgq=256, ldgk=128, ldq=256, ldk=128, lddq=256, lddk=128, ld_rot=32, m=3, positions=9,
             accumulate=0, ws=P, ws_bytes=MUCH)
    return struct_of(B.qeft_qk_bwd_t, f, over)


@pytest.mark.parametrize("desc,over,status", [
    (dict(head_dim=0), {}, SHAPE), (dict(head_dim=264), {}, SHAPE), (dict(head_dim=60), {}, UNSUPPORTED), (dict(rot_dim=31), {}, UNSUPPORTED), (dict(rot_dim=66), {}, SHAPE), (dict(rot_dim=-2), {}, SHAPE),
    (dict(heads=0), {}, SHAPE), (dict(kv_heads=0), {}, SHAPE), (dict(heads=-1), {}, SHAPE), (dict(eps=-1.0), {}, SHAPE), (dict(eps=math.nan), {}, SHAPE), ({}, dict(m=-1), SHAPE), ({}, dict(m=1 << 22), SHAPE),
    ({}, dict(ldq=248), SHAPE), ({}, dict(ldk=132), ALIGN), ({}, dict(q=P + 8), ALIGN), ({}, dict(w_q=P + 8), ALIGN), ({}, dict(w_k=P + 2), ALIGN), ({}, dict(rot=0), NULL), ({}, dict(rot=P + 2), ALIGN),
    ({}, dict(pos=P + 2), ALIGN), ({}, dict(positions=0), SHAPE), ({}, dict(ld_rot=30), SHAPE)])
def test_heads_refuse(desc, over, status):
    d = qdesc(**desc)
    assert B.raw.qeft_qk_norm_fwd(ref(d), ref(qfwd(**over)), None) == status
    assert B.raw.qeft_qk_norm_bwd(ref(d), ref(qbwd(**over)), None) == status
    if desc and not {"heads", "kv_heads"} & set(desc):
        assert B.qeft_qk_norm_workspace(d, 3) == 0


def test_heads_refuse_more():
    d = qdesc()
    for over, status in ((dict(q_out=0), NULL), (dict(k_out=0), NULL), (dict(q_out=P, ldq_out=264), SHAPE), (dict(k_out=P, ldk_out=136), SHAPE), (dict(ldk_out=120), SHAPE)):
        assert B.raw.qeft_qk_norm_fwd(ref(d), ref(qfwd(**over)), None) == status
    assert B.raw.qeft_qk_norm_fwd(None, ref(qfwd()), None) == B.raw.qeft_qk_norm_fwd(ref(d), None, None) == NULL == B.raw.qeft_qk_norm_bwd(ref(d), None, None)
    assert B.raw.qeft_qk_norm_fwd(ref(d), ref(qfwd(m=0, q_out=0)), None) == 0 == B.raw.qeft_qk_norm_fwd(ref(d), ref(qfwd(q=0, k=0)), None)
    need = B.qeft_qk_norm_workspace(d, 3)
    assert need > 0 and B.qeft_qk_norm_workspace(d, 0) == 0
    for over, status in ((dict(q=0), NULL), (dict(k=0), NULL), (dict(w_q=0), NULL), (dict(w_k=0), NULL), (dict(gq=0), NULL), (dict(gk=0, dk=0), NULL), (dict(dq=P, lddq=264), SHAPE),
                         (dict(dk=P, lddk=136), SHAPE), (dict(dw_q=P + 8), ALIGN), (dict(dw_q=2 * P), UNSUPPORTED), (dict(ws=0), WORKSPACE), (dict(ws_bytes=need - 1), WORKSPACE),
                         (dict(ws=P + 4), ALIGN)):
        assert B.raw.qeft_qk_norm_bwd(ref(d), ref(qbwd(**over)), None) == status, over
    assert B.raw.qeft_qk_norm_bwd(ref(d), ref(qbwd(dq=0, dk=0, dw_q=0, dw_k=0, ws=0)), None) == 0


def test_append_with_norms_refuses():
    d, pools, table = B.make_cache_desc(8, 16, 4, 64), B.qeft_cache_t(P, P), B.qeft_table_t(P, 4, 4, 2)
    f = dict(q=P, k=P, v=P, q_out=P, ldq=512, ldq_out=512, ldk=256, ldv=256, seq=P, index=P, pos=P, rot=P, ld_rot=64, positions=9, rot_dim=64, heads=8, tokens=3)

    def call(norm, **over):
        return B.raw.qeft_cache_append_norm(ref(d), ref(pools), ref(table), ref(B.qeft_append_t(**{**f, **over})), ref(norm), None)

    ok = B.qeft_append_norm_t(P, P, 1e-6)
    assert call(None) == NULL
    for norm, status in ((B.qeft_append_norm_t(P + 8, P, 1e-6), ALIGN), (B.qeft_append_norm_t(P, P + 2, 1e-6), ALIGN), (B.qeft_append_norm_t(P, P, -1.0), SHAPE), (B.qeft_append_norm_t(P, P, math.nan), SHAPE)):
        assert call(norm) == status
    for over, status in ((dict(k=0), NULL), (dict(ldk=248), SHAPE), (dict(rot_dim=31), UNSUPPORTED), (dict(index=P + 1), ALIGN), (dict(tokens=-1), SHAPE)):
        assert call(ok, **over) == status
    assert call(ok, tokens=0) == 0


# ---- lists of tensors ------------------------------------------------------------------------------------------------

def rows(*over, n=1000, bits=32, weight=True, master=True):
    """Tensors side by side in an address space that nothing reads."""
    out = (B.qeft_tensor_t * max(1, len(over)))()
    at = 1 << 20
    for i, o in enumerate(over):
        r = dict(n=n, decay=0.1)
        for name in ("weight", "master", "grad", "m", "v", "m_scale", "v_scale"):
            r[name] = at
            at += 1 << 24
        if not weight:
            r["weight"] = 0
        if not master:
            r["master"] = 0
        if bits == 32:
            r["m_scale"] = r["v_scale"] = 0
        for k, v in {**r, **o}.items():
            setattr(out[i], k, v)
    return out


def plan(tensors, count=None, grad=1, bits=32, bytes_=None, where=None):
    count = len(tensors) if count is None else count
    size = B.raw.qeft_tensors_plan_bytes(tensors, count)
    buf = C.create_string_buffer(max(size, 1) + 16)
    at = C.addressof(buf) + 15 & ~15
    out = B.qeft_tensors_t()
    st = B.raw.qeft_tensors_plan(tensors, count, grad, bits, at if where is None else where, size if bytes_ is None else bytes_, ref(out))
    return st, out, C.string_at(at, size), buf


@pytest.mark.parametrize("over,status", [
    (dict(n=-1), SHAPE), (dict(n=(1 << 40) + 1), SHAPE), (dict(grad=0), NULL), (dict(m=0), NULL), (dict(v=0), NULL), (dict(m_scale=P), NULL), (dict(weight=0, master=0), NULL),
    (dict(weight=0), UNSUPPORTED), (dict(master=0), UNSUPPORTED), (dict(grad=(1 << 20) + 8), ALIGN), (dict(m=(1 << 30) + 4), ALIGN), (dict(decay=math.inf), SHAPE), (dict(decay=math.nan), SHAPE)])
def test_plans_refuse(over, status):
    assert plan(rows({}, over))[0] == status
    assert plan(rows({}, {}))[0] == 0


def test_plans_refuse_what_overlaps():
    t = rows({}, {}, n=1000)
    names = ("weight", "master", "grad", "m", "v")
    for a in names:
        for b in names:
            x = rows({}, {}, n=1000)
            setattr(x[1], a, getattr(x[0], b))
            assert plan(x)[0] == (0 if a == b == "grad" else UNSUPPORTED), (a, b)       # (gradients are only read: two tensors may have one)
    for shift, status in ((16, UNSUPPORTED), (4000 - 16 + 15 & ~15, UNSUPPORTED), (4000, 0), (4016, 0)):
        x = rows({}, n=1000)
        x[0].v = x[0].m + shift
        assert plan(x, 1)[0] == status, shift
    x = rows({}, n=1000, bits=8)
    assert plan(x, 1, bits=8)[0] == 0
    x[0].v_scale = x[0].m_scale + 7
    assert plan(x, 1, bits=8)[0] == UNSUPPORTED
    x[0].v_scale = x[0].m_scale + 8             # (eight blocks: scales need no alignment)
    assert plan(x, 1, bits=8)[0] == 0
    x[0].m_scale = 0
    assert plan(x, 1, bits=8)[0] == NULL
    assert plan(t, 2, grad=3)[0] == plan(t, 2, bits=16)[0] == UNSUPPORTED


def test_plans_say_what_is_where():
    t = rows({}, dict(n=0, grad=0, m=0), dict(n=5000, decay=0.5), dict(n=1), n=2048)
    st, out, data, _ = plan(t)
    assert st == 0 and (out.work, out.count, out.grad_dtype, out.state_bits, out.has_weight, out.has_master) == (5, 4, 1, 32, 1, 1) and out.plan is None
    records = [struct.unpack_from("<7QqqfI", data, 80 * i) for i in range(4)]
    assert [r[7] for r in records] == [2048, 0, 5000, 1] and [r[8] for r in records] == [0, 16, 16, 56] and [r[10] for r in records] == [0, 1, 1, 4]
    assert [r[9] for r in records[2:]] == [0.5, pytest.approx(0.1)] and records[2][2] == t[2].grad
    assert list(struct.unpack_from("<5i", data, 320)) == [0, 2, 2, 2, 3]
    assert plan(t, bytes_=len(data) - 1)[0] == WORKSPACE and plan(t, where=0)[0] == WORKSPACE and plan(t, where=P + 4)[0] == ALIGN
    assert B.raw.qeft_tensors_plan(None, 1, 1, 32, P, 0, ref(out)) == NULL == B.raw.qeft_tensors_plan(t, 4, 1, 32, P, 0, None)
    assert B.raw.qeft_tensors_plan(t, -1, 1, 32, P, 0, ref(out)) == SHAPE and B.raw.qeft_tensors_plan_bytes(t, -1) == 0
    big = rows({}, dict(n=2), n=1 << 23)
    big[0].master, big[0].m, big[0].v, big[0].grad = (i << 40 for i in (1, 2, 3, 4))
    big[0].weight = 5 << 40
    st, out, _, _ = plan(big)
    assert st == 0 and out.work == 4097
    st, out, data, _ = plan(rows({}), 0)
    assert st == 0 and out.work == 0 and data == b""


def slist(**over):
    return struct_of(B.qeft_tensors_t, dict(plan=P, work=3, count=2, grad_dtype=1, state_bits=32, has_weight=1, has_master=1), over)


def adamw(**over):
    return struct_of(B.qeft_adamw_t, dict(lr=0.1, beta1=0.9, beta2=0.99, eps=1e-8, step=1, seed=0, lr_at=0, step_at=0, factor=0, stochastic=0), over)


@pytest.mark.parametrize("over,status", [
    (dict(work=-1), SHAPE), (dict(work=(1 << 30) + 1), SHAPE), (dict(count=-1), SHAPE), (dict(count=(1 << 20) + 1), SHAPE), (dict(plan=0), NULL), (dict(plan=P + 8), ALIGN),
    (dict(grad_dtype=2), UNSUPPORTED), (dict(state_bits=4), UNSUPPORTED)])
def test_lists_that_are_refused(over, status):
    norm = B.qeft_grad_norm_t(1.0, 1.0, P, 0, P, MUCH)
    assert B.raw.qeft_adamw_step(ref(slist(**over)), ref(adamw()), None) == status == B.raw.qeft_grad_norm(ref(slist(**over)), ref(norm), None)
    assert B.raw.qeft_grad_norm_workspace(ref(slist(**over))) == 0


@pytest.mark.parametrize("over,status", [
    (dict(beta1=1.0), SHAPE), (dict(beta1=-0.1), SHAPE), (dict(beta2=1.0), SHAPE), (dict(beta2=math.nan), SHAPE), (dict(eps=0.0), SHAPE), (dict(eps=1e-50), SHAPE), (dict(eps=math.inf), SHAPE),
    (dict(lr=math.nan), SHAPE), (dict(lr=math.inf), SHAPE), (dict(step=0), SHAPE), (dict(step=(1 << 30) + 1), SHAPE), (dict(lr_at=P + 2), ALIGN), (dict(step_at=P + 1), ALIGN), (dict(factor=P + 2), ALIGN)])
def test_steps_refuse(over, status):
    assert B.raw.qeft_adamw_step(ref(slist()), ref(adamw(**over)), None) == status


def test_steps_and_norms_refuse_more():
    assert B.raw.qeft_adamw_step(None, ref(adamw()), None) == NULL == B.raw.qeft_adamw_step(ref(slist()), None, None)
    assert B.raw.qeft_adamw_step(ref(slist(has_weight=0, has_master=0)), ref(adamw()), None) == NULL
    assert B.raw.qeft_adamw_step(ref(slist(work=0, plan=0)), ref(adamw()), None) == 0
    need = B.raw.qeft_grad_norm_workspace(ref(slist()))
    assert 0 < need <= B.raw.qeft_grad_norm_workspace(ref(slist(work=1 << 30))) < 1 << 20
    base = dict(scale=1.0, max_norm=1.0, out=P, steps=0, ws=P, ws_bytes=need)
    for over, status in ((dict(scale=0.0), SHAPE), (dict(scale=math.inf), SHAPE), (dict(max_norm=0.0), SHAPE), (dict(max_norm=math.nan), SHAPE), (dict(out=0), NULL), (dict(out=P + 2), ALIGN),
                         (dict(steps=P + 2), ALIGN), (dict(ws=0), WORKSPACE), (dict(ws_bytes=need - 1), WORKSPACE), (dict(ws=P + 8), ALIGN)):
        assert B.raw.qeft_grad_norm(ref(slist()), ref(B.qeft_grad_norm_t(**{**base, **over})), None) == status, over
    assert B.raw.qeft_grad_norm(ref(slist()), None, None) == NULL


def test_the_binding_refuses_tensors_that_do_not_fit():
    z, t = torch.zeros((2, 64), dtype=torch.float16), torch.zeros(2, dtype=torch.int32)
    d = B.make_logprob_desc(64)
    for args, status in (((z, t), UNSUPPORTED), ((z.float(), t), UNSUPPORTED), ((z[:, :32], t), SHAPE), ((z[0], t), UNSUPPORTED)):
        with pytest.raises(B.QeftError) as e:
            B.qeft_logprob_fwd(d, *args, ws=torch.zeros(1 << 16, dtype=torch.uint8))
        assert e.value.status == status
    with pytest.raises(B.QeftError) as e:
        B.qeft_qk_norm_fwd(B.make_qk_desc(64, 1, 1), z, z)
    assert e.value.status == UNSUPPORTED
    with pytest.raises(B.QeftError) as e:
        B.qeft_qk_norm_fwd(B.make_qk_desc(64, 2, 1), z, z)
    assert e.value.status == SHAPE
    g = [torch.zeros(8)]
    for kw, status in ((dict(), UNSUPPORTED), (dict(masters=[]), SHAPE), (dict(decay=[1.0, 2.0]), SHAPE), (dict(m=[torch.zeros(8, dtype=torch.int8)]), UNSUPPORTED)):
        with pytest.raises(B.QeftError) as e:
            B.TensorList(g, **kw)
        assert e.value.status == status
    with pytest.raises(B.QeftError) as e:
        B.make_adamw_states(g, 16)
    assert e.value.status == UNSUPPORTED
    s = B.make_adamw_states([torch.zeros(300)], 8)
    assert {k: (v[0].dtype, v[0].numel()) for k, v in s.items()} == dict(m=(torch.uint8, 300), v=(torch.uint8, 300), m_scales=(torch.uint8, 3), v_scales=(torch.uint8, 3))
    assert B._native.logprob_fwd(d, z, t, None, None, None, 0, None, None, None) is None and B._native.qk_norm_fwd(B.make_qk_desc(64, 1, 1), z, z, None, None, None, None, z, z) is None


def test_random_numbers_are_spread():
    """The numbers that round states: every bit of neighbouring places set half the time, and independent of its neighbours' bits."""
    import ends_util as V
    n = 1 << 16
    x = torch.arange(n)
    h = V.stir((x + V.stir(12345)) % (1 << 32))
    bits = (h[:, None] >> torch.arange(32)) & 1
    s = 0.5 / math.sqrt(n)                                   # the deviation of a mean of n coins
    assert float((bits.double().mean(0) - 0.5).abs().max()) < 5 * s
    same = (bits[1:] == bits[:-1]).double().mean(0)
    assert float((same - 0.5).abs().max()) < 5 * s
    flipped = ((h ^ V.stir((x ^ 1) + V.stir(12345) & 0xFFFFFFFF))[:, None] >> torch.arange(32)) & 1
    assert float((flipped.double().mean(0) - 0.5).abs().max()) < 8 * s


def test_scales_of_logits():
    """scale log2 e has to be a finite number."""
    for scale, status in ((2.0 ** 127, 0), (2.3586e38, 0), (1e-38, 0), (2.3587e38, SHAPE), (3.4e38, SHAPE)):
        d = B.qeft_logprob_desc_t(100, 0, scale)
        assert fwd(d, m=0) == bwd(d, m=0) == both(d, f=dict(m=0), m=0) == status
