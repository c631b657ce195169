// Norms of the heads of queries and keys with their rotation by position, the gradients, and the same for tokens that enter a cache (qeft_qk_norm_fwd,
// qeft_qk_norm_bwd, qeft_cache_append_norm).
//
//   y = x rs w, rs = 1 / sqrt(mean x^2 + eps)     z = R y:  (a, b) -> (a c - b s, b c + a s),  a = y[j], b = y[j + half], half = rot_dim / 2
//   g = R^T gz     dx = rs (a - xh mean(a xh)),  a = g w, xh = x rs     dw = sum g xh
//
// A wave takes a head, a lane values half apart.
#include "qeft_internal.h"
#include "wave.h"

namespace qeft {
namespace {

constexpr int MOST_PAIRS = QEFT_MAX_HEAD_DIM / 2 / 64;   // pairs of a lane
constexpr int SLABS = 1024;

// Lane's i-th pair of the head's d / 2: the rotated ones, then what is behind them two by two
struct Pair {
    int first, second;
    bool there, turned;
};
__device__ __forceinline__ Pair pair_of(int i, int d, int half) {
    const int p = 64 * i + (threadIdx.x & 63);
    if (p >= d / 2) return Pair{0, 0, false, false};
    if (p < half) return Pair{p, p + half, true, true};
    return Pair{2 * p, 2 * p + 1, true, false};
}
struct Turn {
    float c[MOST_PAIRS], s[MOST_PAIRS];
};
__device__ __forceinline__ Turn turn_of(const float* rot, int64_t ld, int positions, int pos, int d, int half) {
    Turn t;
#pragma unroll
    for (int i = 0; i < MOST_PAIRS; ++i) {
        const Pair p = pair_of(i, d, half);
        t.c[i] = 1.f, t.s[i] = 0.f;
        if (p.turned) {
            const float* r = rot + (size_t)min(max(pos, 0), positions - 1) * ld + p.first;
            t.c[i] = r[0];
            t.s[i] = r[half];
        }
    }
    return t;
}

// One head: x (and w, where it is normed) to dst, rotated
__device__ __forceinline__ void one_head(const __half* x, const __half* w, __half* dst, const Turn& t, int d, int half, float eps) {
    float a[MOST_PAIRS], b[MOST_PAIRS], ss = 0.f;
#pragma unroll
    for (int i = 0; i < MOST_PAIRS; ++i) {
        const Pair p = pair_of(i, d, half);
        a[i] = p.there ? __half2float(x[p.first]) : 0.f;
        b[i] = p.there ? __half2float(x[p.second]) : 0.f;
        ss = fmaf(a[i], a[i], fmaf(b[i], b[i], ss));
    }
    if (w) {
        ss = wave_reduce(ss, Sum());
        const float rs = 1.f / sqrtf(ss / (float)d + eps);
#pragma unroll
        for (int i = 0; i < MOST_PAIRS; ++i) {
            const Pair p = pair_of(i, d, half);
            if (!p.there) continue;
            a[i] *= rs * __half2float(w[p.first]);
            b[i] *= rs * __half2float(w[p.second]);
        }
    }
#pragma unroll
    for (int i = 0; i < MOST_PAIRS; ++i) {
        const Pair p = pair_of(i, d, half);
        if (!p.there) continue;
        dst[p.first] = __float2half(p.turned ? a[i] * t.c[i] - b[i] * t.s[i] : a[i]);
        dst[p.second] = __float2half(p.turned ? b[i] * t.c[i] + a[i] * t.s[i] : b[i]);
    }
}

// Workgroup = a token, four waves over its heads
__global__ __launch_bounds__(256) void heads_fwd_kernel(Heads a) {
    const int64_t t = blockIdx.x;
    const int half = a.rot_dim / 2;
    const Turn turn = turn_of(a.rot, a.ld_rot, a.positions, a.pos ? a.pos[t] : (int)t, a.d, half);
    for (int h = threadIdx.x >> 6; h < a.q.heads + a.k.heads; h += 4) {
        const bool is_q = h < a.q.heads;
        const HeadPart& p = is_q ? a.q : a.k;
        const int64_t at = (int64_t)(is_q ? h : h - a.q.heads) * a.d;
        one_head(p.x + t * p.ldx + at, p.w, p.out + t * p.ldout + at, turn, a.d, half, a.eps);
    }
}

__global__ __launch_bounds__(256) void heads_append_kernel(Cache c, Append a, const __half* w_q, const __half* w_k, float eps) {
    const int t = blockIdx.x;
    const int index = a.index[t], b = a.seq ? a.seq[t] : t, half = a.rot_dim / 2;
    const int64_t last = (int64_t)c.table_pages * c.page_size;
    __half *kd = nullptr, *vd = nullptr;
    if (b >= 0 && b < c.seqs && index >= 0 && index < last) {
        const int p = c.by_page.of(index);
        const int page = c.table[(size_t)b * c.ld_table + p];
        if (page >= 0 && page < c.pages) {
            const size_t at = (size_t)page * c.page_stride + (size_t)(index - p * c.page_size) * c.token_stride;
            kd = c.k + at;
            vd = c.v + at;
        }
    }
    const Turn turn = turn_of(a.rot, a.ld_rot, a.positions, a.pos ? a.pos[t] : index, c.d, half);
    const int hq = a.q ? a.heads : 0;
    for (int h = threadIdx.x >> 6; h < hq + 2 * c.kv; h += 4) {
        if (h < hq) {
            one_head(a.q + (size_t)t * a.ldq + (size_t)h * c.d, w_q, a.q_out + (size_t)t * a.ldq_out + (size_t)h * c.d, turn, c.d, half, eps);
        } else if (kd) {
            const int kh = (h - hq) % c.kv;
            if (h < hq + c.kv) {
                one_head(a.k + (size_t)t * a.ldk + (size_t)kh * c.d, w_k, kd + (size_t)kh * c.head_stride, turn, c.d, half, eps);
            } else {
                for (int j = threadIdx.x & 63; j < c.d; j += 64) vd[(size_t)kh * c.head_stride + j] = a.v[(size_t)t * a.ldv + (size_t)kh * c.d + j];
            }
        }
    }
}

// Workgroups stay for tokens blockIdx.x, + gridDim.x ...; slab [workgroup][2 (q, k)][d] of dw
__global__ __launch_bounds__(256) void heads_bwd_kernel(Heads a, float* slab) {
    __shared__ float joined[2][4][QEFT_MAX_HEAD_DIM];
    const int half = a.rot_dim / 2, wave = threadIdx.x >> 6;
    float sums[2][2][MOST_PAIRS] = {};
    for (int64_t t = blockIdx.x; t < a.m; t += gridDim.x) {
        const Turn turn = turn_of(a.rot, a.ld_rot, a.positions, a.pos ? a.pos[t] : (int)t, a.d, half);
#pragma unroll
        for (int which = 0; which < 2; ++which) {
            const HeadPart& p = which ? a.k : a.q;
            for (int h = wave; h < p.heads; h += 4) {
                const int64_t at = (int64_t)h * a.d;
                float ga[MOST_PAIRS], gb[MOST_PAIRS], xa[MOST_PAIRS], xb[MOST_PAIRS], s[2] = {};
#pragma unroll
                for (int i = 0; i < MOST_PAIRS; ++i) {
                    const Pair r = pair_of(i, a.d, half);
                    const __half* g = p.g + t * p.ldg + at;
                    const float u = r.there ? __half2float(g[r.first]) : 0.f, v = r.there ? __half2float(g[r.second]) : 0.f;
                    ga[i] = r.turned ? u * turn.c[i] + v * turn.s[i] : u;
                    gb[i] = r.turned ? v * turn.c[i] - u * turn.s[i] : v;
                    if (!p.w || !r.there) continue;
                    const __half* x = p.x + t * p.ldx + at;
                    xa[i] = __half2float(x[r.first]);
                    xb[i] = __half2float(x[r.second]);
                    s[0] = fmaf(xa[i], xa[i], fmaf(xb[i], xb[i], s[0]));
                    s[1] = fmaf(ga[i] * __half2float(p.w[r.first]), xa[i], fmaf(gb[i] * __half2float(p.w[r.second]), xb[i], s[1]));
                }
                float rs = 0.f, mean = 0.f;
                if (p.w) {
                    s[0] = wave_reduce(s[0], Sum());
                    s[1] = wave_reduce(s[1], Sum());
                    rs = 1.f / sqrtf(s[0] / (float)a.d + a.eps);
                    mean = s[1] * rs / (float)a.d;
                }
#pragma unroll
                for (int i = 0; i < MOST_PAIRS; ++i) {
                    const Pair r = pair_of(i, a.d, half);
                    if (!r.there) continue;
                    float da = ga[i], db = gb[i];
                    if (p.w) {
                        const float ha = xa[i] * rs, hb = xb[i] * rs;
                        sums[which][0][i] = fmaf(da, ha, sums[which][0][i]);
                        sums[which][1][i] = fmaf(db, hb, sums[which][1][i]);
                        da = rs * (da * __half2float(p.w[r.first]) - ha * mean);
                        db = rs * (db * __half2float(p.w[r.second]) - hb * mean);
                    }
                    if (p.dx) {
                        p.dx[t * p.lddx + at + r.first] = __float2half(da);
                        p.dx[t * p.lddx + at + r.second] = __float2half(db);
                    }
                }
            }
        }
    }
    if (!slab) return;
#pragma unroll
    for (int which = 0; which < 2; ++which)
#pragma unroll
        for (int i = 0; i < MOST_PAIRS; ++i) {
            const Pair r = pair_of(i, a.d, half);
            if (!r.there) continue;
            joined[which][wave][r.first] = sums[which][0][i];
            joined[which][wave][r.second] = sums[which][1][i];
        }
    __syncthreads();
    for (int i = threadIdx.x; i < 2 * a.d; i += 256) {
        const int which = i / a.d, j = i % a.d;
        slab[((size_t)blockIdx.x * 2 + which) * a.d + j] = ((joined[which][0][j] + joined[which][1][j]) + joined[which][2][j]) + joined[which][3][j];
    }
}

// dw[j] = the slabs' sum in their order
__global__ __launch_bounds__(256) void heads_sum_kernel(Heads a, const float* slab, int slabs) {
    const int j = blockIdx.x * 256 + threadIdx.x;
    if (j >= 2 * a.d) return;
    float* out = j < a.d ? a.q.dw : a.k.dw;
    if (!out) return;
    float s = 0.f;
    for (int i = 0; i < slabs; ++i) s += slab[(size_t)i * 2 * a.d + j];
    float* at = out + (j < a.d ? j : j - a.d);
    *at = a.accumulate ? *at + s : s;
}

}  // namespace

size_t heads_workspace(int d, int heads, int kv, int rot_dim, int64_t m) { return (size_t)(m < SLABS ? m : SLABS) * 2 * d * sizeof(float); }

hipError_t heads_fwd(const Heads& a, hipStream_t s) {
    heads_fwd_kernel<<<(unsigned)a.m, 256, 0, s>>>(a);
    return hipGetLastError();
}
hipError_t heads_append(const Cache& c, const Append& p, const __half* w_q, const __half* w_k, float eps, hipStream_t s) {
    heads_append_kernel<<<(unsigned)p.tokens, 256, 0, s>>>(c, p, w_q, w_k, eps);
    return hipGetLastError();
}
hipError_t heads_bwd(const Heads& a, hipStream_t s) {
    const bool sums = a.q.dw || a.k.dw;
    float* slab = sums ? (float*)a.ws : nullptr;
    const int slabs = (int)(a.m < SLABS ? a.m : SLABS);
    if (slabs > 0) heads_bwd_kernel<<<(unsigned)slabs, 256, 0, s>>>(a, slab);
    if (sums) heads_sum_kernel<<<(unsigned)(2 * a.d + 255) / 256, 256, 0, s>>>(a, slab, slabs);
    return hipGetLastError();
}

}  // namespace qeft
