// Log probabilities of given tokens, entropies and likeliest tokens from rows of logits, and the gradient of the logits (qeft_logprob_fwd, _bwd, _fwd_bwd).
//
//   c = scale log2(e)    K = max z c    s = sum 2^(z c - K)    lse = K ln 2 + ln s    logp = (z_t c - K) ln 2 - ln s    entropy = ln s - ln 2 sum 2^u u / s, u = z c - K
//   dz_j = scale (p_j (dlse - dlogp - dentropy (log p_j + entropy)) + [j = t] dlogp),   p_j = 2^u / s
//
// z c - K is one multiply-add, K as it was rounded: what rounding K costs is in lse alone.  K is finite where the row is empty, so that -infinity minus it stays what it is.
#include <math.h>
#include "octets.h"
#include "qeft_internal.h"
#include "wave.h"

namespace qeft {
namespace {

constexpr float LN2 = 0.693147180559945f, LOG2E = 1.44269504088896f;
constexpr float LEAST = -3e38f;      // a finite bound of K
constexpr float FAR = -200.f;        // 2^u is 0 from here down: u may stop here, where it is a factor beside 2^u

constexpr uint32_t RANK_NEG_INF = 0x007fffffu, RANK_NAN = 0xff800001u;      // (one above +infinity's)
// Order of alternatives: by value (-0 as +0, not-a-number highest), then lower index.  0: none.
__device__ __forceinline__ uint32_t rank_of(float x) {
    if (x != x) return RANK_NAN;
    const uint32_t b = __builtin_bit_cast(uint32_t, x + 0.f);
    return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float value_of(uint32_t rank) {
    if (rank == RANK_NAN) return __builtin_nanf("");
    return __builtin_bit_cast(float, rank & 0x80000000u ? rank ^ 0x80000000u : ~rank);
}

// Over a workgroup's waves; slots: 16 of LDS, free again behind the next barrier
template <class T, class Op>
__device__ __forceinline__ T group_reduce(T x, T* slots, T none, const Op& op) {
    x = wave_reduce(x, op);
    const int waves = blockDim.x >> 6;
    if (waves == 1) return x;
    __syncthreads();
    if ((threadIdx.x & 63) == 0) slots[threadIdx.x >> 6] = x;
    __syncthreads();
    return waves_reduce(slots, 0, waves, none, op);
}
struct MostFloat {
    __device__ __forceinline__ float operator()(float a, float b) const { return fmaxf(a, b); }   // (passes over not-a-number)
};

// What a row's gradient needs
struct Slope {
    float c, k2, scale, a, dh, at_token;      // u = z c - k2, p = 2^u, log p = u ln 2
    int token;
    bool empty;
};
__device__ __forceinline__ float slope_of(const Slope& g, float z, int j) {
    if (g.empty) return 0.f;
    const float u = fmaf(z, g.c, -g.k2), p = __builtin_amdgcn_exp2f(u);
    float d = g.a;
    if (g.dh != 0.f) d = fmaf(-g.dh * LN2, fmaxf(u, FAR), d);      // (p is not-a-number where u is)
    d *= p;
    if (j == g.token) d += g.at_token;
    return g.scale * d;
}
__device__ __forceinline__ Slope make_slope(const Logprob& a, int64_t row, int token, float k2, float entropy, bool empty) {
    const float dl = a.dlogp ? a.dlogp[row] : 0.f, ds = a.dlse ? a.dlse[row] : 0.f, dh = a.dentropy ? a.dentropy[row] : 0.f;
    return Slope{a.scale * LOG2E, k2, a.scale, ds - dl - (dh != 0.f ? dh * entropy : 0.f), dh, dl, token, empty};
}
template <bool F32>
__device__ __forceinline__ void zero_row(void* row, int n) {
    for (int at = 8 * threadIdx.x; at < n; at += 8 * blockDim.x) {
        float x[8] = {};
        store<F32>(row, at, min(8, n - at), x);
    }
}
// a row without a token: no probability, no alternatives
__device__ __forceinline__ void left_out(const Logprob& a, int64_t row) {
    if (threadIdx.x == 0) {
        if (a.logp) a.logp[row] = 0.f;
        if (a.lse) a.lse[row] = 0.f;
        if (a.entropy) a.entropy[row] = 0.f;
    }
    for (int i = threadIdx.x; i < a.top; i += blockDim.x) {
        a.top_index[row * a.ld_top + i] = -1;
        a.top_logp[row * a.ld_top + i] = -INFINITY;
    }
}

// Rows of any length, read again for each step: the maximum, the sums, each alternative, the gradient.
template <bool F32, bool GRAD>
__global__ __launch_bounds__(1024) void logprob_long_kernel(Logprob a) {
    __shared__ float buf[3][16];
    __shared__ uint64_t best_buf[16];
    const int64_t row = blockIdx.x;
    const char* z = row_of(a.z, row, a.ldz, F32);
    void* dz = GRAD ? row_of(a.dz, row, a.lddz, F32) : nullptr;
    const int token = a.token ? a.token[row] : -1;
    if (a.token && (token < 0 || token >= a.n)) {
        left_out(a, row);
        if (GRAD) zero_row<F32>(dz, a.n);
        return;
    }
    const float c = a.scale * LOG2E;
    float most = -INFINITY;
    for (int at = 8 * threadIdx.x; at < a.n; at += 8 * blockDim.x) {
        const int left = a.n - at;
        Raw<F32> v;
        v.load(z, at, left);
#pragma unroll
        for (int e = 0; e < 8; ++e) most = e < left ? fmaxf(most, v[e]) : most;
    }
    most = group_reduce(most, buf[0], -INFINITY, MostFloat());
    const float k = fmaxf(most * c, LEAST);
    float s = 0.f, t = 0.f;
    for (int at = 8 * threadIdx.x; at < a.n; at += 8 * blockDim.x) {
        const int left = a.n - at;
        Raw<F32> v;
        v.load(z, at, left);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            if (e >= left) continue;
            const float u = fmaf(v[e], c, -k), x = __builtin_amdgcn_exp2f(u);
            s += x;
            t = fmaf(x, fmaxf(u, FAR), t);
        }
    }
    s = group_reduce(s, buf[1], 0.f, Sum());
    t = group_reduce(t, buf[2], 0.f, Sum());
    const bool empty = s == 0.f;
    const float ln_s = logf(s), entropy = empty ? 0.f : ln_s - LN2 * (t / s);
    if (threadIdx.x == 0) {
        if (a.lse) a.lse[row] = empty ? -INFINITY : fmaf(k, LN2, ln_s);
        if (a.entropy) a.entropy[row] = entropy;
        if (a.logp) {
            const float zt = F32 ? ((const float*)z)[token] : (float)((const _Float16*)z)[token];
            a.logp[row] = empty ? -INFINITY : fmaf(fmaf(zt, c, -k), LN2, -ln_s);
        }
    }
    uint64_t last = ~0ull;
    for (int i = 0; i < a.top; ++i) {
        uint64_t best = 0;
        for (int at = 8 * threadIdx.x; at < a.n; at += 8 * blockDim.x) {
            const int left = a.n - at;
            Raw<F32> v;
            v.load(z, at, left);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                if (e >= left) continue;
                const uint64_t x = (uint64_t)rank_of(v[e]) << 32 | (uint32_t)~(at + e);
                if (x < last && x > best) best = x;
            }
        }
        best = group_reduce(best, best_buf, (uint64_t)0, Most());
        const bool there = (uint32_t)(best >> 32) > RANK_NEG_INF;
        last = there ? best : 0;
        if (threadIdx.x == 0) {
            a.top_index[row * a.ld_top + i] = there ? (int)~(uint32_t)best : -1;
            a.top_logp[row * a.ld_top + i] = there ? fmaf(fmaf(value_of(best >> 32), c, -k), LN2, -ln_s) : -INFINITY;
        }
    }
    if (GRAD) {
        const Slope g = make_slope(a, row, token, k + log2f(s), entropy, empty);
        for (int at = 8 * threadIdx.x; at < a.n; at += 8 * blockDim.x) {
            const int left = a.n - at;
            Raw<F32> v;
            v.load(z, at, left);
            float x[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = slope_of(g, v[e], at + e);
            store<F32>(dz, at, left, x);
        }
    }
}

template <bool F32>
__global__ __launch_bounds__(1024) void logprob_bwd_kernel(Logprob a) {
    const int64_t row = blockIdx.x;
    const char* z = row_of(a.z, row, a.ldz, F32);
    char* dz = row_of(a.dz, row, a.lddz, F32);
    const int token = a.token ? a.token[row] : -1;
    if (a.token && (token < 0 || token >= a.n)) return zero_row<F32>(dz, a.n);
    const float lse = a.lse_in[row];
    const Slope g = make_slope(a, row, token, lse * LOG2E, a.entropy_in ? a.entropy_in[row] : 0.f, lse == -INFINITY);
    for (int at = 8 * threadIdx.x; at < a.n; at += 8 * blockDim.x) {
        const int left = a.n - at;
        Raw<F32> v;
        v.load(z, at, left);
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = slope_of(g, v[e], at + e);
        store<F32>(dz, at, left, x);
    }
}

}  // namespace

size_t logprob_workspace(int n, bool f32, int64_t m, int top) { return 0; }

hipError_t logprob_fwd(const Logprob& a, hipStream_t s) {
    const dim3 grid((unsigned)a.m), threads(1024);
    if (a.f32) {
        if (a.dz) logprob_long_kernel<true, true><<<grid, threads, 0, s>>>(a);
        else logprob_long_kernel<true, false><<<grid, threads, 0, s>>>(a);
    } else {
        if (a.dz) logprob_long_kernel<false, true><<<grid, threads, 0, s>>>(a);
        else logprob_long_kernel<false, false><<<grid, threads, 0, s>>>(a);
    }
    return hipGetLastError();
}

hipError_t logprob_bwd(const Logprob& a, hipStream_t s) {
    const dim3 grid((unsigned)a.m), threads(1024);
    if (a.f32) logprob_bwd_kernel<true><<<grid, threads, 0, s>>>(a);
    else logprob_bwd_kernel<false><<<grid, threads, 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace qeft
