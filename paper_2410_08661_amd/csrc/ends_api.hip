// The C ABI of a step's ends (include/qeft.h): argument checks before anything is launched.
#include <math.h>
#include <algorithm>
#include <new>
#include "qeft_internal.h"

using namespace qeft;

namespace {

inline bool aligned(const void* p, uintptr_t to) { return ((uintptr_t)p & (to - 1)) == 0; }
inline int hip_status(hipError_t e) { return e == hipSuccess ? QEFT_OK : QEFT_ERR_HIP; }

#define CHECK(x)                         \
    do {                                 \
        const int st_ = (x);             \
        if (st_ != QEFT_OK) return st_;  \
    } while (0)

int check_rows(const void* p, int64_t ld, int64_t width) {
    if (!p) return QEFT_ERR_NULL;
    if (ld < width) return QEFT_ERR_SHAPE;
    return aligned(p, 16) && (ld & 7) == 0 ? QEFT_OK : QEFT_ERR_ALIGN;
}
int check_workspace(const void* ws, size_t have, size_t need) {
    if (need == 0) return QEFT_OK;
    if (!ws || have < need) return QEFT_ERR_WORKSPACE;
    return aligned(ws, 16) ? QEFT_OK : QEFT_ERR_ALIGN;
}

// ---- log probabilities ----
int check_logprob_desc(const qeft_logprob_desc_t* d) {
    if (!d) return QEFT_ERR_NULL;
    if (d->n <= 0 || d->n > QEFT_MAX_DIM || !(d->scale > 0.f) || !(d->scale * 1.44269504f < INFINITY)) return QEFT_ERR_SHAPE;
    return d->dtype == QEFT_DTYPE_F16 || d->dtype == QEFT_DTYPE_F32 ? QEFT_OK : QEFT_ERR_UNSUPPORTED;
}
int check_top(const qeft_logprob_desc_t* d, int64_t m, int32_t top) {
    return m < 0 || m > QEFT_MAX_ROWS || top < 0 || top > QEFT_MAX_TOP || top > d->n ? QEFT_ERR_SHAPE : QEFT_OK;
}
Logprob logprob_of(const qeft_logprob_desc_t* d, const qeft_logprob_fwd_t* f, const qeft_logprob_bwd_t* b) {
    Logprob p{};
    p.n = d->n;
    p.f32 = d->dtype == QEFT_DTYPE_F32;
    p.scale = d->scale;
    if (f) {
        p.z = f->z;
        p.token = f->token;
        p.logp = f->logp;
        p.lse = f->lse;
        p.entropy = f->entropy;
        p.top_logp = f->top_logp;
        p.top_index = f->top_index;
        p.ldz = f->ldz;
        p.ld_top = f->ld_top;
        p.m = f->m;
        p.top = f->top;
        p.ws = (unsigned char*)f->ws;
    } else {
        p.z = b->z;
        p.token = b->token;
        p.ldz = b->ldz;
        p.m = b->m;
        p.lse_in = b->lse;
        p.entropy_in = b->entropy;
    }
    if (b) {
        p.dlogp = b->dlogp;
        p.dlse = b->dlse;
        p.dentropy = b->dentropy;
        p.dz = b->dz;
        p.lddz = b->lddz;
    }
    return p;
}
int check_logprob_fwd(const qeft_logprob_desc_t* d, const qeft_logprob_fwd_t* a) {
    if (!a) return QEFT_ERR_NULL;
    CHECK(check_top(d, a->m, a->top));
    if (a->m == 0) return QEFT_OK;
    CHECK(check_rows(a->z, a->ldz, d->n));
    if (a->logp && !a->token) return QEFT_ERR_NULL;
    if (a->top > 0 && (!a->top_logp || !a->top_index)) return QEFT_ERR_NULL;
    if (a->top == 0 && (a->top_logp || a->top_index)) return QEFT_ERR_SHAPE;
    if (a->top > 0 && a->ld_top < a->top) return QEFT_ERR_SHAPE;
    for (const void* p : {(const void*)a->token, (const void*)a->logp, (const void*)a->lse, (const void*)a->entropy, (const void*)a->top_logp, (const void*)a->top_index})
        if (!aligned(p, 4)) return QEFT_ERR_ALIGN;
    return check_workspace(a->ws, a->ws_bytes, logprob_workspace(d->n, d->dtype == QEFT_DTYPE_F32, a->m, a->top));
}
int check_logprob_grad(const qeft_logprob_desc_t* d, const qeft_logprob_bwd_t* b, const int32_t* token, int64_t m) {
    if (m == 0) return QEFT_OK;
    CHECK(check_rows(b->dz, b->lddz, d->n));
    if (b->dlogp && !token) return QEFT_ERR_NULL;
    for (const void* p : {(const void*)token, (const void*)b->lse, (const void*)b->entropy, (const void*)b->dlogp, (const void*)b->dlse, (const void*)b->dentropy})
        if (!aligned(p, 4)) return QEFT_ERR_ALIGN;
    return QEFT_OK;
}

// ---- heads ----
int check_qk_desc(const qeft_qk_desc_t* d) {
    if (!d) return QEFT_ERR_NULL;
    if (d->head_dim <= 0 || d->head_dim > QEFT_MAX_HEAD_DIM || d->heads < 0 || d->heads > QEFT_MAX_DIM || d->kv_heads < 0 || d->kv_heads > QEFT_MAX_DIM ||
        d->rot_dim < 0 || d->rot_dim > d->head_dim || !(d->eps >= 0.f))
        return QEFT_ERR_SHAPE;
    return d->head_dim % 8 != 0 || d->rot_dim % 2 != 0 ? QEFT_ERR_UNSUPPORTED : QEFT_OK;
}
int check_turn(const qeft_qk_desc_t* d, const int32_t* pos, const float* rot, int64_t ld_rot, int32_t positions) {
    if (!aligned(pos, 4) || !aligned(rot, 4)) return QEFT_ERR_ALIGN;
    if (d->rot_dim == 0) return QEFT_OK;
    if (!rot) return QEFT_ERR_NULL;
    return positions <= 0 || ld_rot < d->rot_dim ? QEFT_ERR_SHAPE : QEFT_OK;
}

// ---- tensors ----
struct Span {
    uintptr_t begin, end;
    bool written;
};
int count_tensors(const qeft_tensor_t* t, int32_t count, int64_t* pieces) {
    *pieces = 0;
    if (count < 0 || count > QEFT_MAX_TENSORS) return QEFT_ERR_SHAPE;
    if (count > 0 && !t) return QEFT_ERR_NULL;
    for (int32_t i = 0; i < count; ++i) {
        if (t[i].n < 0 || t[i].n > ((int64_t)1 << 40)) return QEFT_ERR_SHAPE;
        *pieces += (t[i].n + PIECE - 1) / PIECE;
    }
    return *pieces > ((int64_t)1 << 30) ? QEFT_ERR_SHAPE : QEFT_OK;
}
size_t plan_bytes(int32_t count, int64_t pieces) { return tensors_map_at(count) + (size_t)pieces * sizeof(int); }

int check_list(const qeft_tensors_t* l, Tensors* t) {
    if (!l) return QEFT_ERR_NULL;
    if (l->count < 0 || l->count > QEFT_MAX_TENSORS || l->work < 0 || l->work > ((int64_t)1 << 30)) return QEFT_ERR_SHAPE;
    if ((l->grad_dtype != QEFT_DTYPE_F16 && l->grad_dtype != QEFT_DTYPE_F32) || (l->state_bits != 8 && l->state_bits != 32)) return QEFT_ERR_UNSUPPORTED;
    if (l->work > 0 && !l->plan) return QEFT_ERR_NULL;
    if (!aligned(l->plan, 16)) return QEFT_ERR_ALIGN;
    t->records = (const TensorRecord*)l->plan;
    t->piece_of = (const int*)((const char*)l->plan + tensors_map_at(l->count));
    t->work = (int)l->work;
    t->grad_f32 = l->grad_dtype == QEFT_DTYPE_F32;
    t->bits = l->state_bits;
    t->has_weight = l->has_weight != 0;
    t->has_master = l->has_master != 0;
    return QEFT_OK;
}

}  // namespace

extern "C" {

size_t qeft_logprob_workspace(const qeft_logprob_desc_t* desc, int64_t m, int32_t top) {
    if (check_logprob_desc(desc) != QEFT_OK || check_top(desc, m, top) != QEFT_OK || m == 0) return 0;
    return logprob_workspace(desc->n, desc->dtype == QEFT_DTYPE_F32, m, top);
}
int qeft_logprob_fwd(const qeft_logprob_desc_t* desc, const qeft_logprob_fwd_t* a, void* stream) {
    CHECK(check_logprob_desc(desc));
    CHECK(check_logprob_fwd(desc, a));
    if (a->m == 0) return QEFT_OK;
    return hip_status(logprob_fwd(logprob_of(desc, a, nullptr), (hipStream_t)stream));
}
int qeft_logprob_bwd(const qeft_logprob_desc_t* desc, const qeft_logprob_bwd_t* a, void* stream) {
    CHECK(check_logprob_desc(desc));
    if (!a) return QEFT_ERR_NULL;
    CHECK(check_top(desc, a->m, 0));
    if (a->m == 0) return QEFT_OK;
    CHECK(check_rows(a->z, a->ldz, desc->n));
    if (!a->lse || (a->dentropy && !a->entropy)) return QEFT_ERR_NULL;
    CHECK(check_logprob_grad(desc, a, a->token, a->m));
    if (a->dz == a->z && a->lddz != a->ldz) return QEFT_ERR_SHAPE;
    return hip_status(logprob_bwd(logprob_of(desc, nullptr, a), (hipStream_t)stream));
}
int qeft_logprob_fwd_bwd(const qeft_logprob_desc_t* desc, const qeft_logprob_fwd_t* a, const qeft_logprob_bwd_t* b, void* stream) {
    CHECK(check_logprob_desc(desc));
    CHECK(check_logprob_fwd(desc, a));
    if (!b) return QEFT_ERR_NULL;
    if (a->top != 0) return QEFT_ERR_UNSUPPORTED;
    if (b->m != a->m) return QEFT_ERR_SHAPE;
    CHECK(check_logprob_grad(desc, b, a->token, a->m));
    if (a->m == 0) return QEFT_OK;
    if (b->dz == a->z && b->lddz != a->ldz) return QEFT_ERR_SHAPE;
    return hip_status(logprob_fwd(logprob_of(desc, a, b), (hipStream_t)stream));
}

int qeft_qk_norm_fwd(const qeft_qk_desc_t* desc, const qeft_qk_fwd_t* a, void* stream) {
    CHECK(check_qk_desc(desc));
    if (!a) return QEFT_ERR_NULL;
    if (a->m < 0 || a->m > QEFT_MAX_ROWS) return QEFT_ERR_SHAPE;
    if (a->m == 0 || (!a->q && !a->k)) return QEFT_OK;
    CHECK(check_turn(desc, a->pos, a->rot, a->ld_rot, a->positions));
    Heads p{};
    const int64_t d = desc->head_dim;
    if (a->q) {
        if (desc->heads == 0) return QEFT_ERR_SHAPE;
        CHECK(check_rows(a->q, a->ldq, desc->heads * d));
        CHECK(check_rows(a->q_out, a->ldq_out, desc->heads * d));
        if (a->q_out == a->q && a->ldq_out != a->ldq) return QEFT_ERR_SHAPE;
        p.q.heads = desc->heads;
    }
    if (a->k) {
        if (desc->kv_heads == 0) return QEFT_ERR_SHAPE;
        CHECK(check_rows(a->k, a->ldk, desc->kv_heads * d));
        CHECK(check_rows(a->k_out, a->ldk_out, desc->kv_heads * d));
        if (a->k_out == a->k && a->ldk_out != a->ldk) return QEFT_ERR_SHAPE;
        p.k.heads = desc->kv_heads;
    }
    if (!aligned(a->w_q, 16) || !aligned(a->w_k, 16)) return QEFT_ERR_ALIGN;
    p.q.x = (const __half*)a->q;
    p.q.w = (const __half*)a->w_q;
    p.q.out = (__half*)a->q_out;
    p.q.ldx = a->ldq;
    p.q.ldout = a->ldq_out;
    p.k.x = (const __half*)a->k;
    p.k.w = (const __half*)a->w_k;
    p.k.out = (__half*)a->k_out;
    p.k.ldx = a->ldk;
    p.k.ldout = a->ldk_out;
    p.pos = a->pos;
    p.rot = a->rot;
    p.ld_rot = a->ld_rot;
    p.m = a->m;
    p.d = desc->head_dim;
    p.rot_dim = desc->rot_dim;
    p.positions = a->positions;
    p.eps = desc->eps;
    return hip_status(heads_fwd(p, (hipStream_t)stream));
}
size_t qeft_qk_norm_workspace(const qeft_qk_desc_t* desc, int64_t m) {
    if (check_qk_desc(desc) != QEFT_OK || m <= 0 || m > QEFT_MAX_ROWS) return 0;
    return heads_workspace(desc->head_dim, desc->heads, desc->kv_heads, desc->rot_dim, m);
}
int qeft_qk_norm_bwd(const qeft_qk_desc_t* desc, const qeft_qk_bwd_t* a, void* stream) {
    CHECK(check_qk_desc(desc));
    if (!a) return QEFT_ERR_NULL;
    if (a->m < 0 || a->m > QEFT_MAX_ROWS) return QEFT_ERR_SHAPE;
    if (!aligned(a->w_q, 16) || !aligned(a->w_k, 16) || !aligned(a->dw_q, 16) || !aligned(a->dw_k, 16)) return QEFT_ERR_ALIGN;
    if (a->dw_q && a->dw_q == a->dw_k) return QEFT_ERR_UNSUPPORTED;
    Heads p{};
    const int64_t d = desc->head_dim;
    if (a->m > 0) {
        CHECK(check_turn(desc, a->pos, a->rot, a->ld_rot, a->positions));
        if (a->gq) {
            if (desc->heads == 0) return QEFT_ERR_SHAPE;
            CHECK(check_rows(a->gq, a->ldgq, desc->heads * d));
            if (a->w_q) CHECK(check_rows(a->q, a->ldq, desc->heads * d));
            if (a->dq) CHECK(check_rows(a->dq, a->lddq, desc->heads * d));
            if (a->dq == a->gq && a->lddq != a->ldgq) return QEFT_ERR_SHAPE;
            p.q.heads = desc->heads;
        } else if (a->dq || a->dw_q) return QEFT_ERR_NULL;
        if (a->gk) {
            if (desc->kv_heads == 0) return QEFT_ERR_SHAPE;
            CHECK(check_rows(a->gk, a->ldgk, desc->kv_heads * d));
            if (a->w_k) CHECK(check_rows(a->k, a->ldk, desc->kv_heads * d));
            if (a->dk) CHECK(check_rows(a->dk, a->lddk, desc->kv_heads * d));
            if (a->dk == a->gk && a->lddk != a->ldgk) return QEFT_ERR_SHAPE;
            p.k.heads = desc->kv_heads;
        } else if (a->dk || a->dw_k) return QEFT_ERR_NULL;
        if ((a->dw_q && !a->w_q) || (a->dw_k && !a->w_k)) return QEFT_ERR_NULL;
        if (a->dw_q || a->dw_k)
            CHECK(check_workspace(a->ws, a->ws_bytes, heads_workspace(desc->head_dim, desc->heads, desc->kv_heads, desc->rot_dim, a->m)));
    }
    if (!a->dq && !a->dk && !a->dw_q && !a->dw_k) return QEFT_OK;
    p.q.x = (const __half*)a->q;
    p.q.w = (const __half*)a->w_q;
    p.q.g = (const __half*)a->gq;
    p.q.dx = (__half*)a->dq;
    p.q.dw = a->dw_q;
    p.q.ldx = a->ldq;
    p.q.ldg = a->ldgq;
    p.q.lddx = a->lddq;
    p.k.x = (const __half*)a->k;
    p.k.w = (const __half*)a->w_k;
    p.k.g = (const __half*)a->gk;
    p.k.dx = (__half*)a->dk;
    p.k.dw = a->dw_k;
    p.k.ldx = a->ldk;
    p.k.ldg = a->ldgk;
    p.k.lddx = a->lddk;
    p.pos = a->pos;
    p.rot = a->rot;
    p.ld_rot = a->ld_rot;
    p.m = a->m;
    p.d = desc->head_dim;
    p.rot_dim = desc->rot_dim;
    p.positions = a->positions;
    p.accumulate = a->accumulate != 0;
    p.eps = desc->eps;
    p.ws = (unsigned char*)a->ws;
    return hip_status(heads_bwd(p, (hipStream_t)stream));
}

size_t qeft_tensors_plan_bytes(const qeft_tensor_t* tensors, int32_t count) {
    int64_t pieces;
    return count_tensors(tensors, count, &pieces) == QEFT_OK ? plan_bytes(count, pieces) : 0;
}
int qeft_tensors_plan(const qeft_tensor_t* tensors, int32_t count, int32_t grad_dtype, int32_t state_bits, void* plan, size_t bytes, qeft_tensors_t* list) {
    if (!list) return QEFT_ERR_NULL;
    int64_t pieces;
    CHECK(count_tensors(tensors, count, &pieces));
    if ((grad_dtype != QEFT_DTYPE_F16 && grad_dtype != QEFT_DTYPE_F32) || (state_bits != 8 && state_bits != 32)) return QEFT_ERR_UNSUPPORTED;
    if (plan_bytes(count, pieces) > bytes || (bytes > 0 && !plan)) return QEFT_ERR_WORKSPACE;
    if (!aligned(plan, 8)) return QEFT_ERR_ALIGN;
    // the same arrays for every tensor that has values
    const qeft_tensor_t* one = nullptr;
    int64_t spans = 0;
    for (int32_t i = 0; i < count; ++i) {
        const qeft_tensor_t& t = tensors[i];
        if (t.n == 0) continue;
        if (!one) one = &t;
        const bool states = t.weight || t.master;
        if (!t.grad || !t.m != !states || !t.v != !states || !t.m_scale != !(states && state_bits == 8) || !t.v_scale != !(states && state_bits == 8)) return QEFT_ERR_NULL;
        if (!t.weight != !one->weight || !t.master != !one->master) return QEFT_ERR_UNSUPPORTED;
        for (const void* p : {(const void*)t.weight, (const void*)t.master, t.grad, (const void*)t.m, (const void*)t.v})
            if (!aligned(p, 16)) return QEFT_ERR_ALIGN;
        if (!(fabsf(t.decay) < INFINITY)) return QEFT_ERR_SHAPE;
        spans += 7;
    }
    // nothing that is written may overlap anything else of the list
    Span* span = spans ? new (std::nothrow) Span[spans] : nullptr;
    if (spans && !span) return QEFT_ERR_WORKSPACE;
    int64_t used = 0;
    for (int32_t i = 0; i < count; ++i) {
        const qeft_tensor_t& t = tensors[i];
        const int64_t blocks = (t.n + QEFT_STATE_BLOCK - 1) / QEFT_STATE_BLOCK, state = state_bits == 8 ? 1 : 4;
        const struct { const void* p; int64_t bytes; bool written; } parts[] = {
            {t.weight, 2 * t.n, true}, {t.master, 4 * t.n, true}, {t.grad, (grad_dtype == QEFT_DTYPE_F32 ? 4 : 2) * t.n, false}, {t.m, state * t.n, true},
            {t.v, state * t.n, true}, {t.m_scale, blocks, true}, {t.v_scale, blocks, true}};
        for (const auto& p : parts)
            if (p.p && t.n > 0) span[used++] = Span{(uintptr_t)p.p, (uintptr_t)p.p + (uintptr_t)p.bytes, p.written};
    }
    std::sort(span, span + used, [](const Span& a, const Span& b) { return a.begin < b.begin; });
    bool overlap = false;
    uintptr_t any = 0, written = 0;      // where what began before ends
    for (int64_t i = 0; i < used; ++i) {
        overlap |= span[i].begin < (span[i].written ? any : written) || span[i].end < span[i].begin;
        any = std::max(any, span[i].end);
        if (span[i].written) written = std::max(written, span[i].end);
    }
    delete[] span;
    if (overlap) return QEFT_ERR_UNSUPPORTED;
    TensorRecord* rec = (TensorRecord*)plan;
    int* map = (int*)((char*)plan + tensors_map_at(count));
    int64_t piece = 0, block = 0;
    for (int32_t i = 0; i < count; ++i) {
        const qeft_tensor_t& t = tensors[i];
        rec[i] = TensorRecord{t.weight, t.master, t.grad, t.m, t.v, t.m_scale, t.v_scale, t.n, block, t.decay, (int32_t)piece};
        for (const int64_t last = piece + (t.n + PIECE - 1) / PIECE; piece < last; ++piece) map[piece] = i;
        block += (t.n + QEFT_STATE_BLOCK - 1) / QEFT_STATE_BLOCK;
    }
    *list = qeft_tensors_t{nullptr, piece, count, grad_dtype, state_bits, one && one->weight, one && one->master};
    return QEFT_OK;
}
int qeft_adamw_step(const qeft_tensors_t* list, const qeft_adamw_t* a, void* stream) {
    Tensors t;
    CHECK(check_list(list, &t));
    if (!a) return QEFT_ERR_NULL;
    if (!(a->beta1 >= 0. && a->beta1 < 1.) || !(a->beta2 >= 0. && a->beta2 < 1.) || !((float)a->eps > 0.f) || !((float)a->eps < INFINITY) || !(fabs(a->lr) < INFINITY)) return QEFT_ERR_SHAPE;
    if (!a->step_at && (a->step < 1 || a->step > (1 << 30))) return QEFT_ERR_SHAPE;
    if (!aligned(a->lr_at, 4) || !aligned(a->step_at, 4) || !aligned(a->factor, 4)) return QEFT_ERR_ALIGN;
    if (t.work == 0) return QEFT_OK;
    if (!t.has_weight && !t.has_master) return QEFT_ERR_NULL;
    Adamw p{};
    p.lr = (float)a->lr;
    p.beta1 = (float)a->beta1;
    p.beta2 = (float)a->beta2;
    p.one_minus_beta1 = (float)(1. - a->beta1);
    p.one_minus_beta2 = (float)(1. - a->beta2);
    p.eps = (float)a->eps;
    p.log_beta1 = (float)log(a->beta1);
    p.log_beta2 = (float)log(a->beta2);
    p.step = a->step_at ? 1 : (int)a->step;
    p.c1 = (float)(1. - pow(a->beta1, p.step));
    p.c2 = (float)(1. - pow(a->beta2, p.step));
    p.stochastic = a->stochastic != 0;
    p.seed_low = (uint32_t)a->seed;
    p.seed_high = (uint32_t)(a->seed >> 32);
    p.lr_at = a->lr_at;
    p.factor = a->factor;
    p.step_at = a->step_at;
    return hip_status(adamw_step(t, p, (hipStream_t)stream));
}
size_t qeft_grad_norm_workspace(const qeft_tensors_t* list) {
    Tensors t;
    return check_list(list, &t) == QEFT_OK ? grad_norm_workspace(t.work) : 0;
}
int qeft_grad_norm(const qeft_tensors_t* list, const qeft_grad_norm_t* a, void* stream) {
    Tensors t;
    CHECK(check_list(list, &t));
    if (!a || !a->out) return QEFT_ERR_NULL;
    if (!(a->scale > 0.f) || !(a->scale < INFINITY) || !(a->max_norm > 0.f)) return QEFT_ERR_SHAPE;
    if (!aligned(a->out, 4) || !aligned(a->steps, 4)) return QEFT_ERR_ALIGN;
    CHECK(check_workspace(a->ws, a->ws_bytes, grad_norm_workspace(t.work)));
    return hip_status(grad_norm(t, a->scale, a->max_norm, a->out, a->steps, (unsigned char*)a->ws, (hipStream_t)stream));
}

}  // extern "C"
