// The optimizer's step over a list of tensors, states in 32 or 8 bits, and the norm of all gradients (qeft_adamw_step, qeft_grad_norm).
//
//   g = factor grad    m = b1 m + (1 - b1) g    v = b2 v + (1 - b2) g^2    w -= lr decay w + lr r m / (sqrt v + eps q),   q = sqrt(1 - b2^t), r = q / (1 - b1^t)
//
// Bytes bound it: every value is read and written once.  A workgroup takes a piece of a tensor, a thread eight values at a time; 16 lanes have a block of an
// 8-bit state, whose largest value they find without LDS.
#include <math.h>
#include "octets.h"
#include "qeft_internal.h"
#include "wave.h"

namespace qeft {
namespace {

constexpr int THREADS = 256, STEP = 8 * THREADS;
constexpr int SUM_GROUPS = 1024;     // workgroups of the norm
static_assert(PIECE % STEP == 0 && PIECE % QEFT_STATE_BLOCK == 0, "whole blocks");

// 32 bits stirred: two products with odd constants between shifts (every bit of x flips every bit of the result about half the time)
__host__ __device__ __forceinline__ uint32_t stir(uint32_t x) {
    x ^= x >> 16;
    x *= 0x5c3c9ccdu;
    x ^= x >> 15;
    x *= 0xfa1b1bf1u;
    return x ^ x >> 16;
}

// Code of a >= 0 in a format of BITS mantissa bits and exponent bias BIAS, up where the bits that are cut and r (of SIZE bits, at their top) carry: below the
// smallest binade the float's bits are not the code's, there a is cut as a fixed-point number.
template <int BITS, int BIAS, int SIZE>
__device__ __forceinline__ uint32_t cut(float a, uint32_t r) {
    constexpr int DROP = 23 - BITS;
    constexpr float TINIEST = BIAS == 7 ? 0x1p-6f : 0x1p-14f, UNIT = BIAS == 7 ? 0x1p+29f : 0x1p+37f;
    static_assert(BIAS == 7 || BIAS == 15, "e4m3, or e5m2 and fp16");
    r <<= DROP - SIZE;
    const uint32_t normal = ((__builtin_bit_cast(uint32_t, a) + r) >> DROP) - ((127 - BIAS) << BITS);
    const uint32_t low = ((uint32_t)(fminf(a, TINIEST) * UNIT) + r) >> DROP;
    return a >= TINIEST ? normal : low;
}

// Eight 8-bit codes
struct Codes {
    uint32_t x, y;
    __device__ __forceinline__ void load(const uint8_t* p, int left) {
        x = y = 0;
        if (left >= 8) {
            const uint2 v = *reinterpret_cast<const uint2*>(p);
            x = v.x;
            y = v.y;
            return;
        }
#pragma unroll 1
        for (int e = left - 1; e >= 0; --e) {
            y = y << 8 | x >> 24;
            x = x << 8 | p[e];
        }
    }
    __device__ __forceinline__ void store(uint8_t* p, int left) const {
        if (left >= 8) {
            *reinterpret_cast<uint2*>(p) = uint2{x, y};
            return;
        }
        uint32_t lo = x, hi = y;
#pragma unroll 1
        for (int e = 0; e < left; ++e) {
            p[e] = (uint8_t)lo;
            lo = lo >> 8 | hi << 24;
            hi >>= 8;
        }
    }
    template <bool E4M3>
    __device__ __forceinline__ void values(float (&v)[8]) const {
        typedef float f2 __attribute__((ext_vector_type(2)));
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int w = (int)(i < 2 ? x : y);
            f2 p;
            if constexpr (E4M3) p = i & 1 ? __builtin_amdgcn_cvt_pk_f32_fp8(w, true) : __builtin_amdgcn_cvt_pk_f32_fp8(w, false);
            else p = i & 1 ? __builtin_amdgcn_cvt_pk_f32_bf8(w, true) : __builtin_amdgcn_cvt_pk_f32_bf8(w, false);
            v[2 * i] = p.x;
            v[2 * i + 1] = p.y;
        }
    }
};
__device__ __forceinline__ float power_of(uint32_t byte) {   // e8m0
    return __builtin_bit_cast(float, byte == 0 ? 0x00400000u : byte == 255 ? 0x7fc00000u : byte << 23);
}
// Codes of eight values, and the power of two of the block that 16 lanes have; r: 16 random bits each
template <bool E4M3>
__device__ __forceinline__ void encode(const float (&v)[8], const uint32_t (&r)[8], Codes& codes, uint32_t& byte) {
    constexpr int TOP = E4M3 ? 7 : 14;
    uint32_t most = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const uint32_t a = __builtin_bit_cast(uint32_t, v[e]) & 0x7fffffffu;
        most = a > most ? a : most;      // (bits of floats >= 0 are in their order, not-a-number above infinity)
    }
    most = row_reduce(most, Most());
    const bool finite = most < 0x7f800000u;
    const int power = max((int)(most >> 23) - 127 - TOP, -110);
    byte = most == 0 ? 0 : finite ? (uint32_t)(power + 127) : 255;
    const float inverse = __builtin_bit_cast(float, (uint32_t)(127 - power) << 23);
    uint32_t c[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float a = fabsf(v[e]) * inverse;
        c[e] = E4M3 ? cut<3, 7, 16>(a, r[e]) : cut<2, 15, 16>(a, r[e]);
        if (!E4M3 && c[e] == 0 && a > 0.f) c[e] = 1;      // (a state that became zero under a first moment that is not would make a huge step)
        if (E4M3 && v[e] < 0.f) c[e] |= 0x80;
        if (!finite) c[e] = 0x7f;
    }
    codes.x = c[0] | c[1] << 8 | c[2] << 16 | c[3] << 24;
    codes.y = c[4] | c[5] << 8 | c[6] << 16 | c[7] << 24;
}
// fp16 values rounded up or down by 13 random bits each; not-a-number stays one, what reaches 2^16 is infinite
__device__ __forceinline__ _Float16 cut_half(float x, uint32_t r) {
    uint32_t c = cut<10, 15, 13>(fabsf(x), r);
    c = c < 0x7c00u ? c : 0x7c00u;
    c |= __builtin_bit_cast(uint32_t, x) >> 16 & 0x8000u;
    return x != x ? (_Float16)x : __builtin_bit_cast(_Float16, (uint16_t)c);
}

struct Now {      // what the step's number makes
    float lr, size, eps;
};
__device__ __forceinline__ Now now_of(const Adamw& a) {
    float c1 = a.c1, c2 = a.c2;
    if (a.step_at) {
        const float t = (float)max(*a.step_at, 1);
        c1 = -expm1f(t * a.log_beta1);
        c2 = -expm1f(t * a.log_beta2);
    }
    const float lr = a.lr_at ? *a.lr_at : a.lr, q = sqrtf(c2);
    return Now{lr, lr * q / c1, a.eps * q};
}

// m and v: each product and sum rounded for itself, so that the codes do not depend on how a compiler joins them
__device__ __forceinline__ void moments(const Adamw& a, float g, float& m, float& v) {
#pragma clang fp contract(off)
    m = a.beta1 * m + a.one_minus_beta1 * g;
    v = a.beta2 * v + a.one_minus_beta2 * (g * g);
}

template <bool GRAD32, bool STATE8, bool WEIGHT, bool MASTER>
__global__ __launch_bounds__(THREADS) void adamw_kernel(Tensors t, Adamw a) {
    const float factor = a.factor ? *a.factor : 1.f;
    if (!(fabsf(factor) < INFINITY)) return;
    const TensorRecord& rec = t.records[t.piece_of[blockIdx.x]];
    const int64_t from = (int64_t)((int)blockIdx.x - rec.first_piece) * PIECE;
    const int n = (int)min((int64_t)PIECE, rec.n - from);
    const Now now = now_of(a);
    const float decay = now.lr * rec.decay;
    const bool dice = STATE8 || (!MASTER && a.stochastic);
    const int64_t place = rec.first_block * QEFT_STATE_BLOCK + from;
    const uint32_t step = (uint32_t)(a.step_at ? max(*a.step_at, 1) : a.step);
    const uint32_t key = stir(step + stir(a.seed_low + stir(a.seed_high)));
    for (int at = 8 * threadIdx.x; (at & -QEFT_STATE_BLOCK) < n; at += STEP) {      // (the 16 lanes of a block stay together)
        const int left = n - at;
        Raw<GRAD32> grad;
        grad.load((const char*)rec.grad + from * (GRAD32 ? 4 : 2), at, left);
        Raw<MASTER> weight;
        if (MASTER) weight.load(rec.master + from, at, left);
        else weight.load((const char*)rec.weight + from * 2, at, left);
        float m[8], v[8], w[8];
        const int64_t block = (from + at) / QEFT_STATE_BLOCK;
        if (STATE8) {
            Codes cm, cv;
            cm.load((const uint8_t*)rec.m + from + at, left);
            cv.load((const uint8_t*)rec.v + from + at, left);
            const float pm = power_of(rec.m_scale[block]), pv = power_of(rec.v_scale[block]);
            cm.values<true>(m);
            cv.values<false>(v);
#pragma unroll
            for (int e = 0; e < 8; ++e) m[e] *= pm, v[e] *= pv;
        } else {
            Raw<true> rm, rv;
            rm.load((const float*)rec.m + from, at, left);
            rv.load((const float*)rec.v + from, at, left);
#pragma unroll
            for (int e = 0; e < 8; ++e) m[e] = rm[e], v[e] = rv[e];
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            moments(a, factor * grad[e], m[e], v[e]);
            const float x = weight[e];
            w[e] = fmaf(-decay, x, x) - now.size * (m[e] / (sqrtf(v[e]) + now.eps));
            if (e >= left) m[e] = v[e] = 0.f;      // (no part of a block's largest)
        }
        uint32_t r[8] = {};
        if (dice) {
            const int64_t first = place + at;
            const uint32_t base = (uint32_t)first + stir((uint32_t)(first >> 32) + key);
#pragma unroll
            for (int e = 0; e < 8; ++e) r[e] = stir(base + e);
        }
        if (STATE8) {
            Codes cm, cv;
            uint32_t bm, bv, dm[8], dv[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) dm[e] = r[e] >> 16, dv[e] = r[e] & 0xffffu;
            encode<true>(m, dm, cm, bm);
            encode<false>(v, dv, cv, bv);
            cm.store((uint8_t*)rec.m + from + at, left);
            cv.store((uint8_t*)rec.v + from + at, left);
            if ((threadIdx.x & 15) == 0) {
                rec.m_scale[block] = (uint8_t)bm;
                rec.v_scale[block] = (uint8_t)bv;
            }
        } else {
            store<true>((float*)rec.m + from, at, left, m);
            store<true>((float*)rec.v + from, at, left, v);
        }
        if (MASTER) store<true>(rec.master + from, at, left, w);
        if (WEIGHT) {
            if (!MASTER && a.stochastic) {
#pragma unroll
                for (int e = 0; e < 8; ++e) w[e] = (float)cut_half(w[e], r[e] * 0x5c3c9ccdu >> 19);
            }
            store<false>((__half*)rec.weight + from, at, left, w);
        }
    }
}

// One partial sum a workgroup, pieces blockIdx.x, + gridDim.x ...
template <bool GRAD32>
__global__ __launch_bounds__(THREADS) void square_sums_kernel(Tensors t, double* part) {
    __shared__ double slots[16];
    double s = 0.;
    for (int p = blockIdx.x; p < t.work; p += gridDim.x) {
        const TensorRecord& rec = t.records[t.piece_of[p]];
        const int64_t from = (int64_t)(p - rec.first_piece) * PIECE;
        const int n = (int)min((int64_t)PIECE, rec.n - from);
        for (int at = 8 * threadIdx.x; at < n; at += STEP) {
            Raw<GRAD32> g;
            g.load((const char*)rec.grad + from * (GRAD32 ? 4 : 2), at, n - at);
#pragma unroll
            for (int e = 0; e < 8; ++e) s = fma((double)g[e], (double)g[e], s);      // (what does not exist was loaded as 0)
        }
    }
    s = wave_reduce(s, Sum());
    if ((threadIdx.x & 63) == 0) slots[threadIdx.x >> 6] = s;
    __syncthreads();
    if (threadIdx.x == 0) part[blockIdx.x] = ((slots[0] + slots[1]) + slots[2]) + slots[3];
}
__global__ __launch_bounds__(SUM_GROUPS) void norm_finish_kernel(const double* part, int parts, float scale, float max_norm, float* out, int* steps) {
    __shared__ double slots[16];
    double s = threadIdx.x < parts ? part[threadIdx.x] : 0.;
    s = wave_reduce(s, Sum());
    if ((threadIdx.x & 63) == 0) slots[threadIdx.x >> 6] = s;
    __syncthreads();
    if (threadIdx.x != 0) return;
    s = 0.;
    for (int i = 0; i < SUM_GROUPS / 64; ++i) s += slots[i];
    const double norm = (double)scale * sqrt(s);
    out[0] = (float)norm;
    const bool finite = fabsf((float)norm) < INFINITY;
    out[1] = !finite ? __builtin_nanf("") : norm > (double)max_norm ? (float)(scale * ((double)max_norm / norm)) : scale;
    if (steps && finite) *steps += 1;
}

template <bool GRAD32, bool STATE8>
void launch(const Tensors& t, const Adamw& a, hipStream_t s) {
    const unsigned grid = (unsigned)t.work;
    if (!t.has_master) adamw_kernel<GRAD32, STATE8, true, false><<<grid, THREADS, 0, s>>>(t, a);
    else if (t.has_weight) adamw_kernel<GRAD32, STATE8, true, true><<<grid, THREADS, 0, s>>>(t, a);
    else adamw_kernel<GRAD32, STATE8, false, true><<<grid, THREADS, 0, s>>>(t, a);
}

}  // namespace

hipError_t adamw_step(const Tensors& t, const Adamw& a, hipStream_t s) {
    if (t.grad_f32) {
        if (t.bits == 8) launch<true, true>(t, a, s);
        else launch<true, false>(t, a, s);
    } else {
        if (t.bits == 8) launch<false, true>(t, a, s);
        else launch<false, false>(t, a, s);
    }
    return hipGetLastError();
}

size_t grad_norm_workspace(int work) { return (size_t)(work < SUM_GROUPS ? work : SUM_GROUPS) * sizeof(double); }

hipError_t grad_norm(const Tensors& t, float scale, float max_norm, float* out, int* steps, unsigned char* ws, hipStream_t s) {
    const int parts = t.work < SUM_GROUPS ? t.work : SUM_GROUPS;
    if (parts > 0) {
        if (t.grad_f32) square_sums_kernel<true><<<(unsigned)parts, THREADS, 0, s>>>(t, (double*)ws);
        else square_sums_kernel<false><<<(unsigned)parts, THREADS, 0, s>>>(t, (double*)ws);
    }
    norm_finish_kernel<<<1, SUM_GROUPS, 0, s>>>((const double*)ws, parts, scale, max_norm, out, steps);
    return hipGetLastError();
}

}  // namespace qeft
