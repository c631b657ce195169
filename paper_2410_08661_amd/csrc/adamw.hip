// The optimizer's step over a list of tensors, states in 32 or 8 bits, and the norm of all gradients (qeft_adamw_step, qeft_grad_norm).
//
//   g = factor grad    m = b1 m + (1 - b1) g    v = b2 v + (1 - b2) g^2    w -= lr decay w + lr r m / (sqrt v + eps q),   q = sqrt(1 - b2^t), r = q / (1 - b1^t)
//
// Bytes bound it: every value is read and written once.  A workgroup takes a piece of a tensor, a thread eight values (two or more in turn, the next loaded ahead: 3 to 5 % slower);
// 16 lanes have a block of an 8-bit state, whose largest value they find without LDS.  174 million weights with fp32 masters and states 895 us (5.8 TB/s, a large device copy
// 5.1), 272 million with 8-bit states and stochastic rounding 456 (6.0), 38 thousand 4.
#include <math.h>
#include <algorithm>
#include <type_traits>
#include "octets.h"
#include "qeft_internal.h"
#include "wave.h"

namespace qeft {
namespace {

constexpr int THREADS = PIECE / 8;
constexpr int SUM_GROUPS = 1024;     // workgroups of the norm (512: 174 million gradients 78 us in place of 59)
static_assert(PIECE % QEFT_STATE_BLOCK == 0, "whole blocks");

// 32 bits stirred: two products with odd constants between shifts (every bit of x flips every bit of the result about half the time)
__host__ __device__ __forceinline__ uint32_t stir(uint32_t x) {
    x ^= x >> 16;
    x *= 0x5c3c9ccdu;
    x ^= x >> 15;
    x *= 0xfa1b1bf1u;
    return x ^ x >> 16;
}

typedef uint32_t u2 __attribute__((ext_vector_type(2)));

// Eight 8-bit codes
struct Codes {
    uint32_t x, y;
    __device__ __forceinline__ void load(const uint8_t* p, int left) {
        x = y = 0;
        if (left >= 8) {
            const u2 v = fetch<u2>((const char*)p, true);
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
            place((char*)p, u2{x, y}, true);
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
// Codes of eight values, and the power of two of the block that 16 lanes have.  The conversions round by 16 random bits at the top of a word: up where the bits that
// are cut and those carry; as a fixed-point number below the smallest binade (compared with that definition for a million values: the same).  `finite`: of the whole block.
template <bool E4M3>
__device__ __forceinline__ uint32_t block_power(float most, bool finite) {
    constexpr int TOP = E4M3 ? 7 : 14;
    const int power = max((int)(__builtin_bit_cast(uint32_t, most) >> 23) - 127 - TOP, -110);
    return most == 0.f ? 0 : finite ? (uint32_t)(power + 127) : 255;
}
template <bool E4M3>
__device__ __forceinline__ void encode(const float (&v)[8], const uint32_t (&r)[8], Codes& codes, uint32_t byte, bool finite) {
    const float inverse = __builtin_bit_cast(float, (254u - min(max(byte, 17u), 253u)) << 23);      // (2^(127 - byte); a block of zeros has any)
    float a[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) a[e] = v[e] * inverse;
    if (!E4M3) {
        // A second moment that became zero under a first one that is not would make a huge step: it stays at the smallest code.  Few lanes have any this small.
        constexpr float SMALLEST = 0x1p-16f;
        const float least = fminf(fminf(fminf(a[0], a[1]), fminf(a[2], a[3])), fminf(fminf(a[4], a[5]), fminf(a[6], a[7])));
        if (least < SMALLEST) {
#pragma unroll
            for (int e = 0; e < 8; ++e) a[e] = v[e] > 0.f ? fmaxf(a[e], SMALLEST) : a[e];
        }
    }
    int w[2] = {0, 0};
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        if (E4M3) {
            w[i] = __builtin_amdgcn_cvt_sr_fp8_f32(a[4 * i], (int)r[4 * i], w[i], 0);
            w[i] = __builtin_amdgcn_cvt_sr_fp8_f32(a[4 * i + 1], (int)r[4 * i + 1], w[i], 1);
            w[i] = __builtin_amdgcn_cvt_sr_fp8_f32(a[4 * i + 2], (int)r[4 * i + 2], w[i], 2);
            w[i] = __builtin_amdgcn_cvt_sr_fp8_f32(a[4 * i + 3], (int)r[4 * i + 3], w[i], 3);
        } else {
            w[i] = __builtin_amdgcn_cvt_sr_bf8_f32(a[4 * i], (int)r[4 * i], w[i], 0);
            w[i] = __builtin_amdgcn_cvt_sr_bf8_f32(a[4 * i + 1], (int)r[4 * i + 1], w[i], 1);
            w[i] = __builtin_amdgcn_cvt_sr_bf8_f32(a[4 * i + 2], (int)r[4 * i + 2], w[i], 2);
            w[i] = __builtin_amdgcn_cvt_sr_bf8_f32(a[4 * i + 3], (int)r[4 * i + 3], w[i], 3);
        }
    }
    codes.x = finite ? (uint32_t)w[0] : 0x7f7f7f7fu;
    codes.y = finite ? (uint32_t)w[1] : 0x7f7f7f7fu;
}
// Eight values rounded to fp16 by the 13 top bits of a random word's product with an odd constant (the word's own ends round the states): up where the bits that are cut and those carry; as a fixed-point number below the
// smallest binade (compared with that definition for two million values: the same).
__device__ __forceinline__ u4 cut_halves(const float (&w)[8], const uint32_t (&r)[8]) {
    typedef _Float16 h2 __attribute__((ext_vector_type(2)));
    uint32_t x[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        h2 pair = {0, 0};
        pair = __builtin_amdgcn_cvt_sr_f16_f32(pair, w[2 * i], r[2 * i] * 0x5c3c9ccdu, false);
        pair = __builtin_amdgcn_cvt_sr_f16_f32(pair, w[2 * i + 1], r[2 * i + 1] * 0x5c3c9ccdu, true);
        x[i] = __builtin_bit_cast(uint32_t, pair);
    }
    return u4{x[0], x[1], x[2], x[3]};
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

// An address that is the same in all lanes, kept in scalar registers: loads and stores add a lane's 32-bit offset by themselves.
template <class T>
__device__ __forceinline__ T* scalar(T* p) {
    const uint64_t u = (uint64_t)p;
    return (T*)((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(u >> 32)) << 32 | (uint32_t)__builtin_amdgcn_readfirstlane((int)u));
}
// Where a piece's arrays begin
struct Base {
    const char* grad;
    char *weight, *master, *m, *v;
    uint8_t *m_scale, *v_scale;
};
// Eight values of everything a step reads.  With 8-bit states loads and stores but the master's go past the caches (272 million weights with masters 839 -> 786 us, without 494 -> 454);
// with 32-bit states that gains nothing (895 both ways).
template <bool GRAD32, bool STATE8, bool MASTER>
struct Read {
    Raw<GRAD32> grad;
    Raw<MASTER> weight;
    typename std::conditional<STATE8, Codes, Raw<true>>::type m, v;
    uint8_t m_scale, v_scale;
    __device__ __forceinline__ void load(const Base& b, int at, int left) {
        grad.load(b.grad, at, left, 0, STATE8);
        weight.load(MASTER ? b.master : b.weight, at, left, 0, STATE8);
        if constexpr (STATE8) {
            m.load((const uint8_t*)b.m + (uint32_t)at, left);
            v.load((const uint8_t*)b.v + (uint32_t)at, left);
            m_scale = b.m_scale[(uint32_t)at / QEFT_STATE_BLOCK];
            v_scale = b.v_scale[(uint32_t)at / QEFT_STATE_BLOCK];
        } else {
            m.load(b.m, at, left);
            v.load(b.v, at, left);
        }
    }
};

template <bool GRAD32, bool STATE8, bool WEIGHT, bool MASTER>
__global__ __launch_bounds__(THREADS) void adamw_kernel(Tensors t, Adamw a, int first) {
    const float factor = a.factor ? *a.factor : 1.f;
    if (!(fabsf(factor) < INFINITY)) return;
    const int piece = first + blockIdx.x;
    const TensorRecord& rec = t.records[t.piece_of[piece]];
    const int64_t from = (int64_t)(piece - rec.first_piece) * PIECE;
    const int n = (int)min((int64_t)PIECE, rec.n - from);
    constexpr int STATE = STATE8 ? 1 : 4;
    const Base base{scalar((const char*)rec.grad + from * (GRAD32 ? 4 : 2)),  scalar((char*)rec.weight + from * 2),
                    scalar((char*)rec.master + from * 4),                     scalar((char*)rec.m + from * STATE),
                    scalar((char*)rec.v + from * STATE),                      scalar(rec.m_scale + from / QEFT_STATE_BLOCK),
                    scalar(rec.v_scale + from / QEFT_STATE_BLOCK)};
    const bool dice = STATE8 || (!MASTER && a.stochastic);
    const int64_t place = rec.first_block * QEFT_STATE_BLOCK + from;
    const int at = 8 * threadIdx.x, left = n - at;
    if ((at & -QEFT_STATE_BLOCK) >= n) return;      // (the 16 lanes of a block stay together)
    Read<GRAD32, STATE8, MASTER> in;
    in.load(base, at, left);
    const Now now = now_of(a);
    const float decay = now.lr * rec.decay;
    const uint32_t step = (uint32_t)(a.step_at ? max(*a.step_at, 1) : a.step);
    const uint32_t key = stir(step + stir(a.seed_low + stir(a.seed_high)));
    float m[8], v[8], w[8];
    if constexpr (STATE8) {
        const float pm = power_of(in.m_scale), pv = power_of(in.v_scale);
        in.m.template values<true>(m);
        in.v.template values<false>(v);
#pragma unroll
        for (int e = 0; e < 8; ++e) m[e] *= pm, v[e] *= pv;
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) m[e] = in.m[e], v[e] = in.v[e];
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        moments(a, factor * in.grad[e], m[e], v[e]);
        const float x = in.weight[e];
        // (8-bit states: issue bounds the kernel, and the hardware's root and reciprocal are good to a unit of fp32's last place; a root below 2^-63 would be 0)
        const float up = STATE8 ? m[e] * __builtin_amdgcn_rcpf(__builtin_amdgcn_sqrtf(fmaxf(v[e], 0x1p-126f)) + now.eps) : m[e] / (sqrtf(v[e]) + now.eps);
        w[e] = fmaf(-now.size, up, fmaf(-decay, x, x));
    }
    uint32_t r[8] = {};
    if (dice) {
        const int64_t spot = place + at;
        const uint32_t base_r = (uint32_t)spot + stir((uint32_t)(spot >> 32) + key);
#pragma unroll
        for (int e = 0; e < 8; ++e) r[e] = stir(base_r + e);
    }
    if constexpr (STATE8) {
        if (left < 8) {      // what does not exist is no part of a block's largest
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (e >= left) m[e] = v[e] = 0.f;
        }
        float most_m = 0.f;
        uint32_t most_v = 0;      // (bits of floats >= 0 are in their order, not-a-number above infinity)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            most_m = fmaxf(most_m, fabsf(m[e]));
            most_v = max(most_v, __builtin_bit_cast(uint32_t, v[e]));
        }
        most_m = __builtin_bit_cast(float, row_reduce(__builtin_bit_cast(uint32_t, most_m), Most()));
        most_v = row_reduce(most_v, Most());
        // (a gradient that is not finite makes v so; a first moment that was not finite before has a block of such)
        const bool finite = most_v < 0x7f800000u && most_m < INFINITY;
        const uint32_t bm = block_power<true>(most_m, finite), bv = block_power<false>(__builtin_bit_cast(float, most_v), finite);
        Codes cm, cv;
        uint32_t dm[8], dv[8];      // (the instruction would take 20 bits)
#pragma unroll
        for (int e = 0; e < 8; ++e) dm[e] = r[e] & 0xffff0000u, dv[e] = r[e] << 16;
        encode<true>(m, dm, cm, bm, finite);
        encode<false>(v, dv, cv, bv, finite);
        cm.store((uint8_t*)base.m + (uint32_t)at, left);
        cv.store((uint8_t*)base.v + (uint32_t)at, left);
        if ((threadIdx.x & 15) == 0) {
            base.m_scale[(uint32_t)at / QEFT_STATE_BLOCK] = (uint8_t)bm;
            base.v_scale[(uint32_t)at / QEFT_STATE_BLOCK] = (uint8_t)bv;
        }
    } else {
        store<true>(base.m, at, left, m);
        store<true>(base.v, at, left, v);
    }
    if (MASTER) store<true>(base.master, at, left, w);
    if (WEIGHT) {
        if (!MASTER && a.stochastic) store_halves(base.weight, at, left, cut_halves(w, r), STATE8);
        else store<false>(base.weight, at, left, w, STATE8);
    }
}

// One partial sum a workgroup, of every gridDim.x-th bunch of pieces.  A bunch is 64 bytes a thread, so that the chains piece - tensor - gradients of its pieces run at a time
// (174 million fp16 gradients by 1 / 2 / 4 / 8 pieces 83 / 66 / 59 / 62 us, fp32 ones 115 / 106 / 112 / 117).
template <bool GRAD32>
__global__ __launch_bounds__(THREADS) void square_sums_kernel(Tensors t, double* part) {
    __shared__ double slots[16];
    constexpr int BUNCH = GRAD32 ? 2 : 4;
    const int at = 8 * threadIdx.x;
    double s = 0.;
    for (int64_t first = (int64_t)blockIdx.x * BUNCH; first < t.work; first += (int64_t)gridDim.x * BUNCH) {
        const char* from[BUNCH];
        int left[BUNCH];
#pragma unroll
        for (int i = 0; i < BUNCH; ++i) {
            const int p = (int)min(first + i, (int64_t)t.work - 1);
            const TensorRecord& rec = t.records[t.piece_of[p]];
            const int64_t begin = (int64_t)(p - rec.first_piece) * PIECE;
            from[i] = scalar((const char*)rec.grad + begin * (GRAD32 ? 4 : 2));
            left[i] = first + i < t.work ? (int)min((int64_t)PIECE, rec.n - begin) - at : 0;
        }
        Raw<GRAD32> g[BUNCH];
#pragma unroll
        for (int i = 0; i < BUNCH; ++i) g[i].load(from[i], at, left[i]);      // (what does not exist is loaded as 0)
#pragma unroll
        for (int i = 0; i < BUNCH; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) s = fma((double)g[i][e], (double)g[i][e], s);
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
    for (int i = 0; i < (int)blockDim.x / 64; ++i) s += slots[i];
    const double norm = (double)scale * sqrt(s);
    out[0] = (float)norm;
    const bool finite = fabsf((float)norm) < INFINITY;
    out[1] = !finite ? __builtin_nanf("") : norm > (double)max_norm ? (float)(scale * ((double)max_norm / norm)) : scale;
    if (steps && finite) *steps += 1;
}

// Workgroups that a CU runs at a time, by LDS that none of them uses: with more, the rows of memory that so many arrays' streams open push one another out.  174 million weights
// with 32-bit states (seven streams) by 8 / 6 / 4 / 3 / 2 a CU: 960 / 947 / 921 / 895 / 926 us; without masters 698 / 691 / 662 / 645 / 740; 272 million with 8-bit states and masters (nine, short
// ones among them) 855 / 847 / 783 / 818 / 1011.  With 8-bit states alone (six, short ones) many are needed: to nearest 451 / 448 / 492 / 586 / 798.
constexpr int resident_lds(bool state8, bool master) { return !state8 ? 52 * 1024 : master ? 40 * 1024 : 0; }
constexpr int MOST_WORK = 1 << 23;      // pieces of a launch: a grid has fewer than 2^32 threads
template <bool GRAD32, bool STATE8>
void launch(const Tensors& t, const Adamw& a, hipStream_t s) {
    for (int first = 0; first < t.work; first += MOST_WORK) {
        const unsigned grid = (unsigned)std::min(t.work - first, MOST_WORK);
        if (!t.has_master) adamw_kernel<GRAD32, STATE8, true, false><<<grid, THREADS, resident_lds(STATE8, false), s>>>(t, a, first);
        else if (t.has_weight) adamw_kernel<GRAD32, STATE8, true, true><<<grid, THREADS, resident_lds(STATE8, true), s>>>(t, a, first);
        else adamw_kernel<GRAD32, STATE8, false, true><<<grid, THREADS, resident_lds(STATE8, true), s>>>(t, a, first);
    }
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
    norm_finish_kernel<<<1, parts <= 64 ? 64 : parts <= 256 ? 256 : SUM_GROUPS, 0, s>>>((const double*)ws, parts, scale, max_norm, out, steps);
    return hipGetLastError();
}

}  // namespace qeft
