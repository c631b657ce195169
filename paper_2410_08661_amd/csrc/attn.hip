// Attention of one new token per sequence over its paged cache (qeft_attn_decode).
//
//   out[b][h] = sum_t p_t V_t,  p = softmax_t(scale q[b][h] . K_t),  t < lens[b]
//
// What bounds it: every cached byte is read once and used for 2 flops per query head of its kv head, so HBM for up to about a hundred heads per kv
// head.  One pass: a wave takes 32 tokens at a time, keeps the running maximum m and sum l of its softmax and the unnormalised output, and rescales
// those when a maximum grows by more than 1 in log2 (between, p = 2^(x - m) is taken against the older maximum: it then is at most twice too large, in numerator and
// denominator alike).
//
// Both products run on the matrix units for any number of heads (a single head uses one of 16 columns, which costs nothing a bandwidth-bound
// kernel misses), on fragments that come straight from global memory:
//   S^T = K q^T     K's rows are tokens.  The two 16-row tiles of a step take their rows so that lane (c, grp) = (lane & 15, lane >> 4) ends up with
//                   the scores of head column c for the 8 consecutive tokens t0 + 8 grp ..: tile u's row r is token t0 + 8 (r >> 2) + 4 u + (r & 3).
//   O = P V         those 8 probabilities are then the lane's piece of the left operand as they stand, without a shuffle.  V is read by rows (4 rows
//                   of 256 bytes per load at head_dim 128) so that a lane holds 8 tokens x NV dimensions; one v_perm per register makes the columns.
// P enters as hi + lo, two fp16 values rounded to nearest (22 bits): rounding it once would add half of the output's own rounding error again.  The pair is
// of 2^14 p, as large as fp16 holds beside the maximum's growth: it has its 22 bits down to p = 2^-16 of the largest, and is off by 2^-39 of the largest
// at most below that (many tokens of little weight beside one of much must not vanish from O while l counts them).  O's factor is taken out with l's.  (By a product, not in the
// exponent: beside a maximum of 2^25 a difference of 14 is rounded, up to 16, which fp16 does not hold.)
//
// Work: a workgroup of 4 or 8 waves (one wave for a great many short rows) takes a chunk of one sequence's tokens for one kv head (16 query heads at a time; more heads read the chunk again, from
// L2), joins its waves through LDS and writes out, or, where the sequence is cut in several chunks, m, l and O to the workspace for a second launch.
//
// Measured, head_dim 128: 131001 tokens, 64 / 8 heads: 95 us, 5.6 TB/s (a device copy moves 5.2); 8 x 2048 tokens, 32 heads: 47.8 us, 5.6 TB/s;
// 203 tokens, 32 heads: 5.3 us, a chain of latencies.
#include "qeft_internal.h"
#include "wave.h"

namespace qeft {
namespace {

typedef uint32_t u4 __attribute__((ext_vector_type(4)));
typedef uint32_t u2 __attribute__((ext_vector_type(2)));
typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef _Float16 h2 __attribute__((ext_vector_type(2)));
typedef float f2 __attribute__((ext_vector_type(2)));
typedef float f4 __attribute__((ext_vector_type(4)));

constexpr int STEP = 32;                // tokens of a wave's step
constexpr float FACTOR = 16384.f;       // of O, and of p in the product that makes it
constexpr float SLACK = 1.f;            // log2: growth of a maximum that is let pass without rescaling (FACTOR 2^SLACK is below fp16's largest)
constexpr float NEG_INF = -__builtin_inff();

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// Partial results of one (sequence, query head, chunk): m, l, and O[d], in arrays of their own.
struct Partials {
    float* m;      // [seqs][heads][chunks]
    float* l;
    float* o;      // [seqs][heads][chunks][d], FACTOR times what it stands for
    float* raw;    // scores in log2 units, [seqs][heads][pitch] (only where weights are asked for)
    int64_t pitch;
    int chunks, chunk;
};

// NV dimensions of a lane's V rows; 16 lanes cover DP
template <int DP> struct VReg;
template <> struct VReg<64> { typedef u2 type; static constexpr int n = 1; };
template <> struct VReg<128> { typedef u4 type; static constexpr int n = 1; };
template <> struct VReg<256> { typedef u4 type; static constexpr int n = 2; };

// DP: head_dim padded to 64, 128 or 256; FULL: head_dim is DP, and a page's rows lie one behind the other; OCT: page_size is a multiple of 8, one table entry serves an octet of tokens
template <int DP, bool FULL, bool OCT, int WAVES>
__global__ __launch_bounds__(64 * WAVES, 2) void attn_chunk_kernel(Cache c, Attention a, Partials ps, int g, int tiles) {
    constexpr int KS = DP / 32, NV = DP / 16, ROUND = WAVES * STEP;   // (tokens of a round of the waves)
    typedef typename VReg<DP>::type vreg;
    constexpr int VN = VReg<DP>::n, VW = sizeof(vreg) / 4;
    // Queries of 256 dimensions lie in LDS, as the fragments that every wave's lanes need: beside them K's and V's rows and the output would spill
    // (8 x 2000 tokens, 32 heads: 90 us against 125).
    constexpr bool Q_IN_LDS = DP == 256;
    __shared__ u4 sq[Q_IN_LDS ? KS : 1][64];
    __shared__ float sm[WAVES][16], sl[WAVES][16], sL[16], sM[16];
    __shared__ __align__(16) float so[WAVES][4][DP];

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = lane & 15, grp = lane >> 4;
    // Neighbours in the grid, which run at the same time, take the same tokens of neighbouring heads: what they read lies together in a page.
    int id = blockIdx.x;
    const int kvh = id % c.kv;
    id /= c.kv;
    const int tile = id % tiles;
    id /= tiles;
    const int chunk = id % ps.chunks, b = id / ps.chunks;
    const int head0 = kvh * g + 16 * tile, nh = min(16, g - 16 * tile);   // this workgroup's query heads
    const int begin = chunk * ps.chunk;

    // head slot of a column or row r of the products: r = 4 (h % 4) + h / 4, so that up to 4 heads lie in one register of O
    const int my_head = (col >> 2) + 4 * (col & 3);
    h8 q[KS];
    {
        const __half* qp = a.q + (size_t)b * a.ldq + (size_t)(head0 + my_head) * c.d;
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            u4 v = {0, 0, 0, 0};
            const int dim = 32 * s + 8 * grp;
            if (my_head < nh && (FULL || dim < c.d) && (!Q_IN_LDS || s % WAVES == wave)) v = *reinterpret_cast<const u4*>(qp + dim);
            if (!Q_IN_LDS) q[s] = __builtin_bit_cast(h8, v);
            else if (s % WAVES == wave) sq[s][lane] = v;
        }
    }
    const int* row = c.table + (size_t)b * c.ld_table;
    const size_t head_at = (size_t)kvh * c.head_stride;
    const __half* kbase = c.k + head_at;
    const __half* vbase = c.v + head_at;
    const float unit = a.scale * 1.44269504088896340736f;

    // Where an octet's slots begin.  Octets (and everything about them but the choice of a lane's) are the same for the whole wave: scalar work.  Tokens that do
    // not exist have some page of the pool all the same: what is read there is masked.
    auto slot_at = [&](int t) -> int64_t {
        const int p = c.by_page.of(t);
        const int page = min(max(row[min(p, c.table_pages - 1)], 0), c.pages - 1);
        return page * c.page_stride + (t - p * c.page_size) * c.token_stride;
    };
    struct Octets {
        int64_t at[4];
    };
    auto octets = [&](int t0) {
        Octets o;
#pragma unroll
        for (int x = 0; x < 4; ++x) o.at[x] = OCT ? slot_at(t0 + 8 * x) : 0;
        return o;
    };
    auto chosen = [&](const Octets& o, int x) {
        const int64_t lo = x & 1 ? o.at[1] : o.at[0], hi = x & 1 ? o.at[3] : o.at[2];
        return x & 2 ? hi : lo;
    };
    // the first lookups are asked for with the length, not after it
    int t0 = begin + STEP * wave;
    Octets next{};
    if (OCT && a.longest > 0) next = octets(t0);
    const int n = min(a.lens[b], a.longest), end = min(n, begin + ps.chunk);
    if (end <= begin && chunk > 0) return;   // (an empty sequence's first chunk writes the zeros)
    u4 K[2][KS];
    vreg V[8][VN];
    const int64_t krow = (int64_t)(col & 3) * c.token_stride + 8 * grp;
    auto load_k = [&](int t0, const Octets& o) {
        const __half* p[2];
        if (OCT) {
            p[0] = kbase + (chosen(o, col >> 2) + krow);
            p[1] = p[0] + 4 * (FULL ? DP : c.token_stride);
        } else {
            const int t = t0 + 8 * (col >> 2) + (col & 3);
            p[0] = kbase + (slot_at(t) + 8 * grp);
            p[1] = kbase + (slot_at(t + 4) + 8 * grp);
        }
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int s = 0; s < KS; ++s) {
                if (FULL) K[u][s] = *reinterpret_cast<const u4*>(p[u] + 32 * s);
                else {
                    K[u][s] = u4{0, 0, 0, 0};
                    if (32 * s + 8 * grp < c.d) K[u][s] = *reinterpret_cast<const u4*>(p[u] + 32 * s);
                }
            }
    };
    auto load_v = [&](int t0, const Octets& o) {
        const int dim = NV * col;
        const __half* p0 = OCT ? vbase + (chosen(o, grp) + dim) : nullptr;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const __half* p = OCT ? p0 + i * (FULL ? DP : c.token_stride) : vbase + (slot_at(t0 + 8 * grp + i) + dim);
#pragma unroll
            for (int x = 0; x < VN; ++x) {
                if (FULL) V[i][x] = *reinterpret_cast<const vreg*>(p + 8 * x);
                else {
                    V[i][x] = vreg{};
                    if (dim + 8 * x < c.d) V[i][x] = *reinterpret_cast<const vreg*>(p + 8 * x);
                }
            }
        }
    };

    float m = NEG_INF, l = 0.f;   // of head column col; l: this lane's tokens only
    f4 acc[NV];
#pragma unroll
    for (int j = 0; j < NV; ++j) acc[j] = f4{0.f, 0.f, 0.f, 0.f};

    if (t0 < end) {
        load_k(t0, next);
        load_v(t0, next);
        if (t0 + ROUND < end) next = octets(t0 + ROUND);   // (looked up a step ahead of the loads)
    }
    if (Q_IN_LDS) __syncthreads();   // (the first rows are on their way)
    for (; t0 < end; t0 += ROUND) {
        int at_q = lane;
        if (Q_IN_LDS) asm volatile("" : "+v"(at_q));   // (read in every step, not kept in registers after all)
        f4 st[2] = {f4{0.f, 0.f, 0.f, 0.f}, f4{0.f, 0.f, 0.f, 0.f}};
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            const h8 qs = Q_IN_LDS ? __builtin_bit_cast(h8, sq[Q_IN_LDS ? s : 0][at_q]) : q[s];
#pragma unroll
            for (int u = 0; u < 2; ++u) st[u] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h8, K[u][s]), qs, st[u], 0, 0, 0);
        }
        const bool more = t0 + ROUND < end;
        if (more) load_k(t0 + ROUND, next);   // K's registers are free: the next step's rows fly during the softmax and the second product

        float x[8];   // log2 of the weight, unnormalised; token t0 + 8 grp + e
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = st[e >> 2][e & 3] * unit;
        const bool tail = t0 + STEP > end;
        if (tail) {
            const int left = end - (t0 + 8 * grp);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                x[e] = e < left ? x[e] : NEG_INF;
#pragma unroll
                for (int y = 0; y < VN; ++y) V[e][y] = e < left ? V[e][y] : vreg{};   // whatever lies behind the end: 0 x NaN is NaN
            }
        }
        if (ps.raw && my_head < nh) {
            float* rp = ps.raw + ((size_t)b * a.heads + head0 + my_head) * ps.pitch + t0 + 8 * grp;
            *reinterpret_cast<f4*>(rp) = f4{x[0], x[1], x[2], x[3]};
            *reinterpret_cast<f4*>(rp + 4) = f4{x[4], x[5], x[6], x[7]};
        }
        float mx = x[0];
#pragma unroll
        for (int e = 1; e < 8; ++e) mx = fmaxf(mx, x[e]);
        if (__ballot(mx > m + SLACK)) {   // (m = -inf at first: taken for any score above it)
            const auto larger = [](float x, float y) { return fmaxf(x, y); };
            mx = fmaxf(m, across<true>(across<false>(mx, larger), larger));   // over the lanes of this column
            if (__ballot(m != NEG_INF)) {   // (nothing but zeros to scale before the first score)
                const float f = m == NEG_INF ? 0.f : exp2_fast(m - mx);
                l = l == 0.f ? 0.f : l * f;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float fr = __shfl(f, 4 * grp + i);
#pragma unroll
                    for (int j = 0; j < NV; ++j) acc[j][i] *= fr;
                }
            }
            m = mx;
        }
        const float base = m == NEG_INF ? 0.f : m;   // (every score so far was -inf: their weight is 0)
        h8 hi, lo;
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
            const float p0 = exp2_fast(x[e] - base), p1 = exp2_fast(x[e + 1] - base);
            l += p0;
            l += p1;
            const h2 h = __builtin_convertvector((f2{p0 * FACTOR, p1 * FACTOR}), h2);
            const h2 r = __builtin_convertvector((f2{fmaf(p0, FACTOR, -(float)h.x), fmaf(p1, FACTOR, -(float)h.y)}), h2);
            hi[e] = h.x, hi[e + 1] = h.y;
            lo[e] = r.x, lo[e + 1] = r.y;
        }
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            u4 col8;   // dimension NV col + j of the lane's 8 tokens
            const uint32_t sel = (j & 1) ? 0x07060302u : 0x05040100u;
#pragma unroll
            for (int y = 0; y < 4; ++y) col8[y] = __builtin_amdgcn_perm(V[2 * y + 1][j / (2 * VW)][(j / 2) % VW], V[2 * y][j / (2 * VW)][(j / 2) % VW], sel);
            acc[j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(hi, __builtin_bit_cast(h8, col8), acc[j], 0, 0, 0);
            acc[j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(lo, __builtin_bit_cast(h8, col8), acc[j], 0, 0, 0);
        }
        if (more) {
            load_v(t0 + ROUND, next);
            next = octets(t0 + 2 * ROUND);
        }
    }

    // ---- join the waves: maxima, sums and outputs as they are, four heads at a time; every thread that sums an output makes the factors itself ----
    l = across<true>(across<false>(l, Sum()), Sum());
    if (lane < 16) {
        sm[wave][lane] = m;
        sl[wave][lane] = l;
    }
    const bool direct = ps.chunks == 1 && ps.m == nullptr;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (4 * i >= nh) break;   // heads 4 i .. 4 i + 3
#pragma unroll
        for (int j = 0; j < NV; j += 4)
            *reinterpret_cast<f4*>(&so[wave][grp][NV * col + j]) = f4{acc[j][i], acc[j + 1][i], acc[j + 2][i], acc[j + 3][i]};
        __syncthreads();
        for (int e = threadIdx.x; e < 4 * DP; e += 64 * WAVES) {
            const int hl = e / DP, dim = e % DP, h = hl + 4 * i, r = 4 * hl + i;
            if (h < nh && (FULL || dim < c.d)) {
                float wm[WAVES], wl[WAVES], wo[WAVES], M = NEG_INF, L = 0.f, o = 0.f;
#pragma unroll
                for (int w = 0; w < WAVES; ++w) {
                    wm[w] = sm[w][r];
                    wl[w] = sl[w][r];
                    wo[w] = so[w][hl][dim];
                    M = fmaxf(M, wm[w]);
                }
#pragma unroll
                for (int w = 0; w < WAVES; ++w) {
                    const float f = wm[w] == NEG_INF ? 0.f : exp2_fast(wm[w] - M);
                    L += wl[w] == 0.f ? 0.f : wl[w] * f;
                    o = fmaf(wo[w], f, o);
                }
                if (direct) {
                    a.out[(size_t)b * a.ldo + (size_t)(head0 + h) * c.d + dim] = __float2half_rn(n > 0 ? o / (L * FACTOR) : 0.f);
                    if (dim == 0) {
                        sM[r] = M;
                        sL[r] = L;
                    }
                } else {
                    const size_t at = ((size_t)b * a.heads + head0 + h) * ps.chunks + chunk;
                    ps.o[at * c.d + dim] = o;
                    if (dim == 0) {
                        ps.m[at] = M;
                        ps.l[at] = L;
                    }
                }
            }
        }
        __syncthreads();
    }
    if (direct && a.score) {   // all of the kv head's query heads are this workgroup's; its scores were written before the barriers above
        const float* rp = ps.raw + ((size_t)b * a.heads + head0) * ps.pitch;
        float* out = a.score + ((size_t)b * c.kv + kvh) * a.ld_score;
        for (int t = threadIdx.x; t < n; t += 64 * WAVES) {
            float w = 0.f;
            for (int h = 0; h < nh; ++h) {
                const int at = 4 * (h & 3) + (h >> 2);
                w += exp2_fast(rp[(size_t)h * ps.pitch + t] - sM[at]) / sL[at];
            }
            out[t] = a.accumulate ? out[t] + w : w;
        }
    }
}

// Maximum and sum of a query head over its used chunks (a wave's work; the same in every lane).
__device__ __forceinline__ void join_stats(const Partials& ps, size_t at, int used, float& M, float& L) {
    const int lane = threadIdx.x & 63;
    // the first 64 chunks' are asked for before `used` is known
    float l = 0.f, m = NEG_INF;
    if (lane < ps.chunks) {
        l = ps.l[at + lane];
        m = ps.m[at + lane];
    }
    if (lane >= used || l == 0.f) m = NEG_INF, l = 0.f;
    M = m;
    for (int i = lane + 64; i < used; i += 64) M = fmaxf(M, ps.l[at + i] == 0.f ? NEG_INF : ps.m[at + i]);
    M = wave_reduce(M, [](float x, float y) { return fmaxf(x, y); });
    L = l == 0.f ? 0.f : l * exp2_fast(m - M);
    for (int i = lane + 64; i < used; i += 64) L += ps.l[at + i] == 0.f ? 0.f : ps.l[at + i] * exp2_fast(ps.m[at + i] - M);
    L = wave_reduce(L, Sum());
}

constexpr int JOIN_TOKENS = 512;   // tokens whose weights one workgroup of the second launch makes (4 x 4096 tokens, 64 heads on 8: 19.4 us with 1024, 18.7 with 256;
                                   // 16 x 4000, 32 on 8: 57.7 and 59.8, this 58.4)
constexpr int JOIN_HEADS = 8;      // heads whose scores and statistics are under way at a time (8 x 4000, 32 on 1: 23.8 us with 4, 20.5 with 16, this 20.8)

// The second launch.  Its first workgroups join the chunks of one query head, 32 dimensions each: 32 lanes of chunks x 8 of four dimensions.  The others
// make the weights of one kv head's tokens, JOIN_TOKENS at a time (weight_shares of them divide a kv head's), from the scores in the workspace.  Chunks are taken in order: the sums do not depend on who ran first.
__global__ __launch_bounds__(256) void attn_join_kernel(Cache c, Attention a, Partials ps, int g, int weight_shares) {
    const int slices = (c.d + 31) / 32;
    const int64_t outs = (int64_t)c.seqs * a.heads * slices;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    __shared__ __align__(16) float red[32][36];   // (rows four banks apart)
    __shared__ float part[2 * JOIN_HEADS];
    if ((int64_t)blockIdx.x < outs) {
        const int slice = (int)(blockIdx.x % slices), bh = (int)(blockIdx.x / slices), b = bh / a.heads, h = bh % a.heads;
        const size_t at = ((size_t)b * a.heads + h) * ps.chunks;
        const int quad = tid & 7, lane_c = tid >> 3, dim = 32 * slice + 4 * quad;
        const float* po = ps.o + at * c.d + dim;
        // Everything is asked for at once, before the length says how much of it was written (the rest is not looked at): one latency, not three.
        constexpr int AHEAD = 4;
        f4 v[AHEAD];
        float vl[AHEAD], vm[AHEAD];
#pragma unroll
        for (int x = 0; x < AHEAD; ++x) {
            const int i = lane_c + 32 * x;
            v[x] = f4{0.f, 0.f, 0.f, 0.f};
            vl[x] = vm[x] = 0.f;
            if (i < ps.chunks) {
                vl[x] = ps.l[at + i];
                vm[x] = ps.m[at + i];
                if (dim < c.d) v[x] = *reinterpret_cast<const f4*>(po + (size_t)i * c.d);
            }
        }
        const int n = min(a.lens[b], a.longest), used = n > 0 ? (n + ps.chunk - 1) / ps.chunk : 0;
        __half* out = a.out + (size_t)b * a.ldo + (size_t)h * c.d;
        float M, L;
        join_stats(ps, at, used, M, L);
        f4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int x = 0; x < AHEAD; ++x)
            if (lane_c + 32 * x < used && vl[x] != 0.f) o += v[x] * exp2_fast(vm[x] - M);
        if (dim < c.d)
            for (int i = lane_c + 32 * AHEAD; i < used; i += 32) {
                const float l = ps.l[at + i], f = exp2_fast(ps.m[at + i] - M);
                const f4 w = *reinterpret_cast<const f4*>(po + (size_t)i * c.d);
                if (l != 0.f) o += w * f;
            }
        *reinterpret_cast<f4*>(&red[lane_c][4 * quad]) = o;
        __syncthreads();
        if (tid < 32 && 32 * slice + tid < c.d) {
            float x = 0.f;
#pragma unroll
            for (int i = 0; i < 32; ++i) x += red[i][tid];
            out[32 * slice + tid] = __float2half_rn(n > 0 ? x / (L * FACTOR) : 0.f);
        }
        return;
    }
    int64_t id = (int64_t)blockIdx.x - outs;
    const int first = (int)(id % weight_shares);
    id /= weight_shares;
    const int kvh = (int)(id % c.kv), b = (int)(id / c.kv);
    const int n = min(a.lens[b], a.longest), used = (n + ps.chunk - 1) / ps.chunk;
    float* out = a.score + ((size_t)b * c.kv + kvh) * a.ld_score;
    for (int begin = first * JOIN_TOKENS; begin < n; begin += weight_shares * JOIN_TOKENS) {
        const int end = min(n, begin + JOIN_TOKENS);
        float w[JOIN_TOKENS / 256] = {};
        for (int h0 = 0; h0 < g; h0 += JOIN_HEADS) {   // a wave for the statistics of each fourth head
            float raw[JOIN_HEADS][JOIN_TOKENS / 256];   // (asked for with the statistics)
#pragma unroll
            for (int y = 0; y < JOIN_HEADS; ++y)
#pragma unroll
                for (int x = 0; x < JOIN_TOKENS / 256; ++x) {
                    const int t = begin + 256 * x + tid;
                    raw[y][x] = h0 + y < g && t < end ? ps.raw[((size_t)b * a.heads + (size_t)kvh * g + h0 + y) * ps.pitch + t] : 0.f;
                }
#pragma unroll
            for (int y = 0; y < JOIN_HEADS; y += 4) {
                const int h = h0 + y + wave;
                if (h < g) {
                    float M, L;
                    join_stats(ps, ((size_t)b * a.heads + (size_t)kvh * g + h) * ps.chunks, used, M, L);
                    if (lane == 0) {
                        part[y + wave] = M;
                        part[JOIN_HEADS + y + wave] = 1.f / L;
                    }
                }
            }
            __syncthreads();
#pragma unroll
            for (int y = 0; y < JOIN_HEADS; ++y) {
                if (h0 + y >= g) break;
                const float M = part[y], by = part[JOIN_HEADS + y];
#pragma unroll
                for (int x = 0; x < JOIN_TOKENS / 256; ++x) w[x] += exp2_fast(raw[y][x] - M) * by;
            }
            __syncthreads();
        }
#pragma unroll
        for (int x = 0; x < JOIN_TOKENS / 256; ++x) {
            const int t = begin + 256 * x + tid;
            if (t < end) out[t] = a.accumulate ? out[t] + w[x] : w[x];
        }
    }
}

// Tokens that one workgroup takes rather than two launches, 512 at head_dim 128: 32 heads of one sequence, 256 / 400 / 800 tokens: 6.2 / 8.5 / 12.3 us against 8.4 / 8.5 / 9.0; at 64,
// 4 sequences of 600 / 740 / 880: 7.5 / 8.2 / 8.9 against 10.0 / 10.3 / 10.3 (one sequence: 6.7 / 7.5 / 8.1 against 6.8); at 256, 285 / 400 / 500 of one: 10.1 / 13.2 / 15.3 against 9.9 / 10.2 / 10.5.
int short_row(int d) { return 128 + 49152 / d; }
constexpr int CUS = 256;

// Chunks of a row (a sequence's kv head, and 16 of its query heads) of `rounds` 128-token rounds of 64 KiB at head_dim 128.  A CU reads 20 bytes a ns
// at most, so what counts is that all have the same number of workgroups: one each for up to 16 rows (1 of 130000 tokens, 8 heads on 1: 21.1 us against 29.3 with two; 8 of 60000:
// 48.8 against 49.7), two for up to 128 if they are long (32 of 2048, with weights: 11.2 against 12.0; 128 of 2800: 35.8 against 38.0), or, between 128 and 512 rows, what the estimate finds
// (us: 160 rows of 2049 tokens in 1 / 2 / 3 chunks: 46.4 / 46.3 / 39.4; 256 of 2048: 48.2 / 52.6; 8 of 131001 in 32 / 64 / 128 / 256: 95.6 / 97.3 / 102.6 / 109.9).
// The second launch is 4 us, and more where many heads have many chunks.
int chunks_of(int64_t rows, int64_t rounds, int d, int g) {
    if (rounds <= 1 || rows >= 2 * CUS) return 1;
    if (rows <= CUS / 2) {
        // One chunk where its rounds, 1.7 us each by eight waves, cost no more than the second launch (more with many heads a kv head) and the rounds of two workgroups a CU, 2.75 us for all
        // rows': 128 rows of 700 / 1000 / 1400 tokens, 8 heads each: 12.8 / 15.8 / 20.6 us against 19.3 / 21.5 / 25.8; one head each: 11.5 / 15.0 / 19.6 against 13.7 / 15.9 / 20.0.
        if (rows >= CUS / 4 && (float)rounds * (1.7f - 2.75f * (float)rows / CUS) * (float)(d + 64) / 192.f <= 4.f + 0.35f * (float)g) return 1;
        const int64_t most = (rows <= 16 ? CUS : 2 * CUS) / rows;
        return (int)(most < rounds ? most : rounds);
    }
    int best = 1;
    float least = 0.f;
    for (int c = 1; c <= 8 && c <= rounds; ++c) {
        const float per_cu = (float)((rows * c + CUS - 1) / CUS), us = 3.2f * d / 128.f;   // (a round's time on a CU)
        const float t = per_cu * ((float)((rounds + c - 1) / c) * us + 0.5f) + (c > 1 ? 4.f : 0.f);
        if (c == 1 || t < least) best = c, least = t;
    }
    return best;
}

struct Plan {
    int waves, chunk, chunks, tiles;
    bool direct;
    size_t at_l, at_o, at_raw, bytes;
    int64_t pitch;
};

Plan plan_of(int kv, int d, int64_t seqs, int heads, int longest, bool weights) {
    Plan p;
    const int g = heads / kv;
    p.tiles = (g + 15) / 16;
    const int64_t rows = seqs * kv * p.tiles;
    // One wave for two steps of rows that fill the GPU several times (2048 rows of 1 / 32 / 64 tokens: 6.6 / 8.5 / 13.2 us against 11.0 / 11.7 / 14.9 with four waves; 512 rows of 20
    // tokens, 4 heads each: 5.4 against 4.7).  Eight waves for what is one chunk of few rows (256 rows of 1000 to 2048 tokens, 4 heads each: 41.2 us against 43.1), four else: a round of 128 tokens wastes
    // less at a row's end (2048 rows of 100 to 300 tokens: 44.9 us against 52.9).
    int chunks = longest <= short_row(d) ? 1 : chunks_of(rows, ((int64_t)longest + 4 * STEP - 1) / (4 * STEP), d, g);
    p.waves = longest <= 2 * STEP && rows >= 4 * CUS ? 1 : chunks == 1 && rows < 2 * CUS ? 8 : 4;
    const int round = p.waves * STEP;
    const int64_t rounds = ((int64_t)longest + round - 1) / round, per = rounds > 0 ? (rounds + chunks - 1) / chunks : 1;
    p.chunk = (int)(per * round);
    p.chunks = rounds > 0 ? (int)((rounds + per - 1) / per) : 1;   // (longest 0: the chunk that writes the zeros)
    p.direct = p.chunks == 1 && (p.tiles == 1 || !weights);
    const size_t parts = p.direct ? 0 : (size_t)seqs * heads * p.chunks;
    const auto up = [](size_t x) { return (x + 255) / 256 * 256; };
    p.at_l = up(parts * 4);
    p.at_o = 2 * p.at_l;
    p.at_raw = p.at_o + up(parts * d * 4);
    p.pitch = weights ? rounds * round : 0;
    p.bytes = p.at_raw + (size_t)seqs * heads * p.pitch * 4;
    return p;
}

template <int DP, bool FULL, bool OCT>
void launch(const Cache& c, const Attention& a, const Partials& ps, int g, const Plan& p, unsigned grid, hipStream_t s) {
    if (p.waves == 1) attn_chunk_kernel<DP, FULL, OCT, 1><<<grid, 64, 0, s>>>(c, a, ps, g, p.tiles);
    else if (p.waves == 8) attn_chunk_kernel<DP, FULL, OCT, 8><<<grid, 512, 0, s>>>(c, a, ps, g, p.tiles);
    else attn_chunk_kernel<DP, FULL, OCT, 4><<<grid, 256, 0, s>>>(c, a, ps, g, p.tiles);
}
template <int DP>
void launch_dim(const Cache& c, const Attention& a, const Partials& ps, int g, const Plan& p, unsigned grid, hipStream_t s) {
    if (c.page_size % 8 != 0) return launch<DP, false, false>(c, a, ps, g, p, grid, s);
    if (c.d == DP && c.token_stride == DP) return launch<DP, true, true>(c, a, ps, g, p, grid, s);
    launch<DP, false, true>(c, a, ps, g, p, grid, s);
}

}  // namespace

size_t attn_workspace(int kv, int d, int64_t seqs, int heads, int bound, bool weights) {
    return plan_of(kv, d, seqs, heads, bound, weights).bytes;
}

hipError_t attn_decode(const Cache& c, const Attention& a, hipStream_t s) {
    const bool weights = a.score != nullptr;
    const Plan p = plan_of(c.kv, c.d, c.seqs, a.heads, a.bound, weights);
    const int g = a.heads / c.kv;
    Partials ps{};
    ps.chunk = p.chunk;
    ps.chunks = p.chunks;
    if (!p.direct) {
        ps.m = (float*)a.ws;
        ps.l = (float*)(a.ws + p.at_l);
        ps.o = (float*)(a.ws + p.at_o);
    }
    if (weights) {
        ps.raw = (float*)(a.ws + p.at_raw);
        ps.pitch = p.pitch;
    }
    const unsigned grid = (unsigned)((int64_t)c.seqs * c.kv * ps.chunks * p.tiles);
    if (c.d <= 64) launch_dim<64>(c, a, ps, g, p, grid, s);
    else if (c.d <= 128) launch_dim<128>(c, a, ps, g, p, grid, s);
    else launch_dim<256>(c, a, ps, g, p, grid, s);
    if (!p.direct) {
        const int64_t rows = (int64_t)c.seqs * c.kv, most = rows < 32768 ? 65536 / rows : 1;   // (workgroups enough to fill the GPU, and a grid of bounded size)
        const int tiles = weights ? (a.longest + JOIN_TOKENS - 1) / JOIN_TOKENS : 0, shares = tiles < most ? tiles : (int)most;
        attn_join_kernel<<<(unsigned)((int64_t)c.seqs * a.heads * ((c.d + 31) / 32) + rows * shares), 256, 0, s>>>(c, a, ps, g, shares);
    }
    return hipGetLastError();
}

}  // namespace qeft
