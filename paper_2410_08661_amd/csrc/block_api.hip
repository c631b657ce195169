// The C ABI of what lies between a decoder block's linear layers (include/qeft.h): argument checks before anything is launched.
#include "qeft_internal.h"

using namespace qeft;

namespace {

inline bool aligned16(const void* p) { return ((uintptr_t)p & 15u) == 0; }
inline bool aligned4(const void* p) { return ((uintptr_t)p & 3u) == 0; }
inline int hip_status(hipError_t e) { return e == hipSuccess ? QEFT_OK : QEFT_ERR_HIP; }
inline bool overlap(const void* a, size_t an, const void* b, size_t bn) {
    const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
    return a && b && x < y + bn && y < x + an;
}

// A matrix that the call reads or writes: `width` values of a row, 16-byte rows
int check_rows(const void* p, int64_t rows, int64_t ld, int64_t width) {
    if (rows == 0) return QEFT_OK;
    if (!p) return QEFT_ERR_NULL;
    if (ld < width) return QEFT_ERR_SHAPE;
    if (!aligned16(p) || (ld & 7) != 0) return QEFT_ERR_ALIGN;
    return QEFT_OK;
}
// The same where the matrix may be left out
int check_optional(const void* p, int64_t rows, int64_t ld, int64_t width) { return p ? check_rows(p, rows, ld, width) : QEFT_OK; }

int check_cache_desc(const qeft_cache_desc_t* d) {
    if (!d) return QEFT_ERR_NULL;
    if (d->pages <= 0 || d->page_size <= 0 || d->page_size > QEFT_MAX_DIM || d->kv_heads <= 0 || d->kv_heads > QEFT_MAX_DIM || d->head_dim <= 0 ||
        d->head_dim > QEFT_MAX_HEAD_DIM)
        return QEFT_ERR_SHAPE;
    if (d->head_dim % 8 != 0) return QEFT_ERR_UNSUPPORTED;
    if (d->page_stride < 0 || d->head_stride < 0 || d->token_stride < 0) return QEFT_ERR_SHAPE;
    // a head's row is contiguous; axes of one entry have no pitch to speak of
    if ((d->page_size > 1 && d->token_stride < d->head_dim) || (d->kv_heads > 1 && d->head_stride < d->head_dim) ||
        (d->pages > 1 && d->page_stride < d->head_dim))
        return QEFT_ERR_SHAPE;
    if ((d->page_stride | d->head_stride | d->token_stride) & 7) return QEFT_ERR_ALIGN;
    return QEFT_OK;
}

int make_cache(const qeft_cache_desc_t* d, const qeft_cache_t* p, const qeft_table_t* t, Cache* c) {
    int st = check_cache_desc(d);
    if (st != QEFT_OK) return st;
    if (!p || !p->k || !p->v || !t) return QEFT_ERR_NULL;
    if (!aligned16(p->k) || !aligned16(p->v)) return QEFT_ERR_ALIGN;
    if (t->seqs < 0 || t->seqs > QEFT_MAX_DIM || t->table_pages < 0 || t->ld_table < t->table_pages) return QEFT_ERR_SHAPE;
    if (t->seqs > 0 && t->table_pages > 0 && !t->table) return QEFT_ERR_NULL;
    if (!aligned4(t->table)) return QEFT_ERR_ALIGN;
    c->k = (__half*)p->k;
    c->v = (__half*)p->v;
    c->page_stride = d->page_stride;
    c->head_stride = d->head_stride;
    c->token_stride = d->token_stride;
    c->table = t->table;
    c->ld_table = t->ld_table;
    c->table_pages = t->table_pages;
    c->pages = d->pages;
    c->page_size = d->page_size;
    c->kv = d->kv_heads;
    c->d = d->head_dim;
    c->seqs = t->seqs;
    c->by_page = divider(d->page_size);
    return QEFT_OK;
}

int check_attn(const qeft_cache_desc_t* d, int64_t seqs, int32_t heads, int64_t longest) {
    if (seqs < 0 || seqs > QEFT_MAX_DIM || heads <= 0 || heads > QEFT_MAX_DIM || heads % d->kv_heads != 0 || longest < 0 || longest > QEFT_MAX_DIM)
        return QEFT_ERR_SHAPE;
    if (seqs * heads > QEFT_MAX_ROWS / 8) return QEFT_ERR_SHAPE;
    return QEFT_OK;
}
int check_evict(const qeft_cache_desc_t* d, int64_t seqs, int64_t longest, int64_t budget) {
    if (seqs < 0 || seqs > QEFT_MAX_DIM || longest < 0 || longest > QEFT_MAX_DIM || budget < 0 || budget > QEFT_MAX_DIM) return QEFT_ERR_SHAPE;
    const int64_t tiles = longest / 128 + 1;   // (workgroups of the second launch for a row)
    if (seqs * d->kv_heads > QEFT_MAX_ROWS || seqs * d->kv_heads * tiles > 4 * (int64_t)QEFT_MAX_ROWS) return QEFT_ERR_SHAPE;
    return QEFT_OK;
}
int check_workspace(const void* ws, size_t have, size_t need) {
    if (need == 0) return QEFT_OK;
    if (!ws || have < need) return QEFT_ERR_WORKSPACE;
    return aligned16(ws) ? QEFT_OK : QEFT_ERR_ALIGN;
}

int check_norm_desc(const qeft_norm_desc_t* d) {
    if (!d) return QEFT_ERR_NULL;
    if (d->n <= 0 || d->n > QEFT_MAX_DIM) return QEFT_ERR_SHAPE;
    if (!(d->eps >= 0.f)) return QEFT_ERR_SHAPE;
    if (d->residual_dtype != QEFT_DTYPE_F16 && d->residual_dtype != QEFT_DTYPE_F32) return QEFT_ERR_UNSUPPORTED;
    if (d->gate != QEFT_GATE_NONE && d->gate != QEFT_GATE_CHANNEL && d->gate != QEFT_GATE_TOKEN) return QEFT_ERR_UNSUPPORTED;
    return QEFT_OK;
}
// weights of n values, and a gate as its kind has it
int check_norm_weights(const qeft_norm_desc_t* d, const void* w_pre, const void* w_post, const void* gate, const void* y, int64_t ldg, int64_t m) {
    if (!w_pre) return QEFT_ERR_NULL;
    if ((d->gate != QEFT_GATE_NONE && y && !gate) || (w_post && !y)) return QEFT_ERR_NULL;
    if (gate && (d->gate == QEFT_GATE_NONE || !y)) return QEFT_ERR_UNSUPPORTED;
    if (!aligned16(w_pre) || !aligned16(w_post) || !aligned16(gate)) return QEFT_ERR_ALIGN;
    return d->gate == QEFT_GATE_TOKEN ? check_optional(gate, m, ldg, d->n) : QEFT_OK;
}

#define CHECK(x)                         \
    do {                                 \
        const int st_ = (x);             \
        if (st_ != QEFT_OK) return st_;  \
    } while (0)

int make_append(const qeft_cache_desc_t* desc, const qeft_cache_t* cache, const qeft_table_t* table, const qeft_append_t* a, Cache* cp, Append* ap) {
    CHECK(make_cache(desc, cache, table, cp));
    const Cache& c = *cp;
    if (!a) return QEFT_ERR_NULL;
    if (a->tokens < 0 || a->tokens > QEFT_MAX_ROWS || a->rot_dim < 0 || a->rot_dim > c.d) return QEFT_ERR_SHAPE;
    if (a->rot_dim % 2 != 0) return QEFT_ERR_UNSUPPORTED;
    if (a->q && (a->heads <= 0 || a->heads > QEFT_MAX_DIM)) return QEFT_ERR_SHAPE;
    Append& p = *ap;
    p.tokens = (int)a->tokens;
    if (a->tokens == 0) return QEFT_OK;
    CHECK(check_rows(a->k, a->tokens, a->ldk, (int64_t)c.kv * c.d));
    CHECK(check_rows(a->v, a->tokens, a->ldv, (int64_t)c.kv * c.d));
    if (a->q) {
        CHECK(check_rows(a->q, a->tokens, a->ldq, (int64_t)a->heads * c.d));
        CHECK(check_rows(a->q_out, a->tokens, a->ldq_out, (int64_t)a->heads * c.d));
    }
    if (!a->index) return QEFT_ERR_NULL;
    if (!a->seq && a->tokens > c.seqs) return QEFT_ERR_SHAPE;
    if (!aligned4(a->index) || !aligned4(a->seq) || !aligned4(a->pos) || !aligned4(a->rot)) return QEFT_ERR_ALIGN;
    if (a->rot_dim > 0) {
        if (!a->rot) return QEFT_ERR_NULL;
        if (a->positions <= 0 || a->ld_rot < a->rot_dim) return QEFT_ERR_SHAPE;
    }
    p.q = (const __half*)a->q;
    p.k = (const __half*)a->k;
    p.v = (const __half*)a->v;
    p.q_out = (__half*)a->q_out;
    p.ldq = a->ldq;
    p.ldq_out = a->ldq_out;
    p.ldk = a->ldk;
    p.ldv = a->ldv;
    p.seq = a->seq;
    p.index = a->index;
    p.pos = a->pos;
    p.rot = a->rot;
    p.ld_rot = a->ld_rot;
    p.positions = a->positions;
    p.rot_dim = a->rot_dim;
    p.heads = a->q ? a->heads : 0;
    return QEFT_OK;
}

}  // namespace

extern "C" {

int qeft_cache_append(const qeft_cache_desc_t* desc, const qeft_cache_t* cache, const qeft_table_t* table, const qeft_append_t* a, void* stream) {
    Cache c;
    Append p;
    CHECK(make_append(desc, cache, table, a, &c, &p));
    return p.tokens == 0 ? QEFT_OK : hip_status(cache_append(c, p, (hipStream_t)stream));
}

int qeft_cache_append_norm(const qeft_cache_desc_t* desc, const qeft_cache_t* cache, const qeft_table_t* table, const qeft_append_t* a,
                           const qeft_append_norm_t* norm, void* stream) {
    Cache c;
    Append p;
    CHECK(make_append(desc, cache, table, a, &c, &p));
    if (!norm) return QEFT_ERR_NULL;
    if (!(norm->eps >= 0.f)) return QEFT_ERR_SHAPE;
    if (!aligned16(norm->w_q) || !aligned16(norm->w_k)) return QEFT_ERR_ALIGN;
    if (p.tokens > 0 && !norm->w_q && !norm->w_k) return hip_status(cache_append(c, p, (hipStream_t)stream));
    return p.tokens == 0 ? QEFT_OK : hip_status(heads_append(c, p, (const __half*)norm->w_q, (const __half*)norm->w_k, norm->eps, (hipStream_t)stream));
}

size_t qeft_attn_workspace(const qeft_cache_desc_t* desc, int64_t seqs, int32_t heads, int64_t longest, int weights) {
    if (check_cache_desc(desc) != QEFT_OK || check_attn(desc, seqs, heads, longest) != QEFT_OK || seqs == 0) return 0;
    return attn_workspace(desc->kv_heads, desc->head_dim, seqs, heads, (int)longest, weights != 0);
}

int qeft_attn_decode(const qeft_cache_desc_t* desc, const qeft_cache_t* cache, const qeft_table_t* table, const qeft_attn_t* a, void* stream) {
    Cache c;
    CHECK(make_cache(desc, cache, table, &c));
    if (!a) return QEFT_ERR_NULL;
    CHECK(check_attn(desc, c.seqs, a->heads, a->longest));
    if (c.seqs == 0) return QEFT_OK;
    CHECK(check_rows(a->q, c.seqs, a->ldq, (int64_t)a->heads * c.d));
    CHECK(check_rows(a->out, c.seqs, a->ldo, (int64_t)a->heads * c.d));
    if (!a->lens) return QEFT_ERR_NULL;
    if (!aligned4(a->lens) || !aligned4(a->score)) return QEFT_ERR_ALIGN;
    const int longest = a->longest < c.tokens() ? (int)a->longest : c.tokens();
    if (a->score && a->ld_score < longest) return QEFT_ERR_SHAPE;
    const size_t need = attn_workspace(c.kv, c.d, c.seqs, a->heads, (int)a->longest, a->score != nullptr);   // (the caller's bound, as in qeft_attn_workspace)
    CHECK(check_workspace(a->ws, a->ws_bytes, need));
    Attention p;
    p.lens = a->lens;
    p.bound = (int)a->longest;
    p.longest = longest;
    p.q = (const __half*)a->q;
    p.out = (__half*)a->out;
    p.ldq = a->ldq;
    p.ldo = a->ldo;
    p.heads = a->heads;
    p.scale = a->scale;
    p.score = a->score;
    p.ld_score = a->ld_score;
    p.accumulate = a->accumulate != 0;
    p.ws = (unsigned char*)a->ws;
    return hip_status(attn_decode(c, p, (hipStream_t)stream));
}

size_t qeft_evict_workspace(const qeft_cache_desc_t* desc, int64_t seqs, int64_t longest, int64_t budget) {
    if (check_cache_desc(desc) != QEFT_OK || check_evict(desc, seqs, longest, budget) != QEFT_OK) return 0;
    return evict_workspace(desc->kv_heads, seqs, (int)longest, (int)(budget < longest ? budget : longest));
}

int qeft_cache_evict(const qeft_cache_desc_t* desc, const qeft_cache_t* cache, const qeft_table_t* table, const qeft_evict_t* a, void* stream) {
    Cache c;
    CHECK(make_cache(desc, cache, table, &c));
    if (!a) return QEFT_ERR_NULL;
    CHECK(check_evict(desc, c.seqs, a->longest, a->budget));
    if (a->keep_first < 0 || a->keep_last < 0) return QEFT_ERR_SHAPE;
    if (c.seqs == 0) return QEFT_OK;
    if (!a->lens || !a->seen || !a->lens_out) return QEFT_ERR_NULL;
    const int longest = a->longest < c.tokens() ? (int)a->longest : c.tokens();
    const int budget = a->budget < longest ? (int)a->budget : longest;
    if (longest > 0 && (!a->score || !a->pos)) return QEFT_ERR_NULL;
    if (budget > 0 && (!a->score_out || !a->pos_out)) return QEFT_ERR_NULL;
    if (a->ld < longest || a->ld_out < budget) return QEFT_ERR_SHAPE;
    if (!aligned4(a->lens) || !aligned4(a->seen) || !aligned4(a->lens_out) || !aligned4(a->score) || !aligned4(a->pos) || !aligned4(a->score_out) ||
        !aligned4(a->pos_out))
        return QEFT_ERR_ALIGN;
    // every head of a sequence reads its length and count: the new length cannot go where they are; an output that is not the input itself lies elsewhere
    const int64_t rows = (int64_t)c.seqs * c.kv;
    const size_t in = ((size_t)(rows - 1) * a->ld + longest) * 4, out = ((size_t)(rows - 1) * a->ld_out + budget) * 4, lens = (size_t)c.seqs * 4;
    if (overlap(a->lens_out, lens, a->lens, lens) || overlap(a->lens_out, lens, a->seen, lens)) return QEFT_ERR_UNSUPPORTED;
    const bool same_score = (const void*)a->score_out == (const void*)a->score, same_pos = (const void*)a->pos_out == (const void*)a->pos;
    if ((same_score || same_pos) && a->ld_out != a->ld) return QEFT_ERR_SHAPE;
    if ((!same_score && overlap(a->score_out, out, a->score, in)) || (!same_pos && overlap(a->pos_out, out, a->pos, in)) ||
        overlap(a->score_out, out, a->pos, in) || overlap(a->pos_out, out, a->score, in) || overlap(a->score_out, out, a->pos_out, out))
        return QEFT_ERR_UNSUPPORTED;
    CHECK(check_workspace(a->ws, a->ws_bytes, evict_workspace(c.kv, c.seqs, longest, budget)));
    Evict p;
    p.lens = a->lens;
    p.seen = a->seen;
    p.longest = longest;
    p.budget = budget;
    p.score = a->score;
    p.pos = a->pos;
    p.ld = a->ld;
    p.keep_first = a->keep_first;
    p.keep_last = a->keep_last;
    p.score_out = a->score_out;
    p.pos_out = a->pos_out;
    p.ld_out = a->ld_out;
    p.lens_out = a->lens_out;
    p.ws = (unsigned char*)a->ws;
    return hip_status(cache_evict(c, p, (hipStream_t)stream));
}

int qeft_norm_fwd(const qeft_norm_desc_t* desc, const qeft_norm_fwd_t* a, void* stream) {
    CHECK(check_norm_desc(desc));
    if (!a) return QEFT_ERR_NULL;
    if (a->m < 0 || a->m > QEFT_MAX_ROWS) return QEFT_ERR_SHAPE;
    if (a->m == 0) return QEFT_OK;
    CHECK(check_rows(a->r, a->m, a->ldr, desc->n));
    CHECK(check_rows(a->x, a->m, a->ldx, desc->n));
    CHECK(check_optional(a->y, a->m, a->ldy, desc->n));
    CHECK(check_optional(a->h, a->m, a->ldh, desc->n));
    if (a->h && !a->y) return QEFT_ERR_UNSUPPORTED;   // nothing is added: h would be r
    CHECK(check_norm_weights(desc, a->w_pre, a->w_post, a->gate, a->y, a->ldg, a->m));
    Norm p{};
    p.n = desc->n;
    p.f32 = desc->residual_dtype == QEFT_DTYPE_F32;
    p.gate_kind = a->y ? desc->gate : QEFT_GATE_NONE;
    p.scale = desc->scale;
    p.eps = desc->eps;
    p.m = a->m;
    p.r = a->r;
    p.y = (const __half*)a->y;
    p.gate = (const __half*)a->gate;
    p.w_pre = (const __half*)a->w_pre;
    p.w_post = (const __half*)a->w_post;
    p.h = a->h;
    p.x = (__half*)a->x;
    p.ldr = a->ldr;
    p.ldy = a->ldy;
    p.ldg = a->ldg;
    p.ldh = a->ldh;
    p.ldx = a->ldx;
    return hip_status(norm_fwd(p, (hipStream_t)stream));
}

size_t qeft_norm_workspace(const qeft_norm_desc_t* desc, int64_t m) {
    if (check_norm_desc(desc) != QEFT_OK || m <= 0 || m > QEFT_MAX_ROWS) return 0;
    return norm_workspace(desc->n, m);
}

int qeft_norm_bwd(const qeft_norm_desc_t* desc, const qeft_norm_bwd_t* a, void* stream) {
    CHECK(check_norm_desc(desc));
    if (!a) return QEFT_ERR_NULL;
    if (a->m < 0 || a->m > QEFT_MAX_ROWS) return QEFT_ERR_SHAPE;
    const bool sums = a->dw_pre || a->dw_post || (a->dgate && desc->gate == QEFT_GATE_CHANNEL);
    if (a->m > 0) {
        CHECK(check_rows(a->dx, a->m, a->lddx, desc->n));
        CHECK(check_rows(a->h, a->m, a->ldh, desc->n));
        CHECK(check_optional(a->dh, a->m, a->lddh, desc->n));
        CHECK(check_optional(a->y, a->m, a->ldy, desc->n));
        CHECK(check_optional(a->dr, a->m, a->lddr, desc->n));
        CHECK(check_optional(a->dy, a->m, a->lddy, desc->n));
        CHECK(check_norm_weights(desc, a->w_pre, a->w_post, a->gate, a->y, a->ldg, a->m));
        if ((a->dy && !a->y) || (a->dw_post && !a->w_post) || (a->dgate && !a->gate)) return QEFT_ERR_NULL;
        if (desc->gate == QEFT_GATE_TOKEN) CHECK(check_optional(a->dgate, a->m, a->lddg, desc->n));
        CHECK(check_workspace(a->ws, a->ws_bytes, norm_bwd_workspace(desc->n, a->m, sums)));
    }
    if (!aligned16(a->dw_pre) || !aligned16(a->dw_post) || !aligned16(a->dgate)) return QEFT_ERR_ALIGN;
    Norm p{};
    p.n = desc->n;
    p.f32 = desc->residual_dtype == QEFT_DTYPE_F32;
    p.gate_kind = a->y || a->m == 0 ? desc->gate : QEFT_GATE_NONE;   // (an empty y may have no address)
    p.scale = desc->scale;
    p.eps = desc->eps;
    p.m = a->m;
    p.dx = (const __half*)a->dx;
    p.dh = a->dh;
    p.r = a->h;
    p.y = (const __half*)a->y;
    p.gate = (const __half*)a->gate;
    p.w_pre = (const __half*)a->w_pre;
    p.w_post = (const __half*)a->w_post;
    p.dr = a->dr;
    p.dy = (__half*)a->dy;
    p.dgate = a->dgate;
    p.dw_pre = a->dw_pre;
    p.dw_post = a->dw_post;
    p.lddx = a->lddx;
    p.lddh = a->lddh;
    p.ldr = a->ldh;
    p.ldy = a->ldy;
    p.ldg = a->ldg;
    p.lddr = a->lddr;
    p.lddy = a->lddy;
    p.lddg = a->lddg;
    p.accumulate = a->accumulate != 0;
    p.ws = (unsigned char*)a->ws;
    return hip_status(norm_bwd(p, (hipStream_t)stream));
}

}  // extern "C"
