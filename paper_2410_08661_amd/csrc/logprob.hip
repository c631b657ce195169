// Log probabilities of given tokens, entropies and likeliest tokens from rows of logits, and the gradient of the logits (qeft_logprob_fwd, _bwd, _fwd_bwd).
//
//   M = max z    u = (z - M) scale log2(e)    s = sum 2^u    lse = scale M + ln s    logp = scale (z_t - M) - ln s    entropy = ln s - ln 2 sum 2^u u / s
//   dz_j = scale (p_j (dlse - dlogp - dentropy (log p_j + entropy)) + [j = t] dlogp),   p_j = 2^u (1 / s), or exp(scale z_j - lse) of a given lse
//
// Bytes bound it: a row is read once into registers, by a workgroup or, the longest, by several whose statistics a second launch joins.  2003 x 32003 fp32, a third of the entries
// -infinity, 48 us (5.3 TB/s; a large device copy 5.1); 4096 x 32000 fp16 with the gradient in the same call 85 (5.2), without but with entropies and 20 alternatives 66.  Few rows: one of
// 32000 with 5 alternatives 6.4 us, of which 3.8 a launch that does nothing, 57 x 130001 with 20 13.1.
// u is exact to roundings of its own size, 0 for the largest logit, so that what a large scale z costs is in lse alone: one multiply-add z c - K, c = scale log2(e), K = M c as rounded, which
// leaves all u off by K's error r, known exactly; r goes into the factor that brings a wave's sums to the row's M.  Where K is so large that r would not be small, (z - M) c: an instruction
// more (4096 x 32000 with 20 alternatives 66 -> 71 us).  M is finite where the row is empty, so that -infinity minus it stays what it is.
#include <math.h>
#include <algorithm>
#include "octets.h"
#include "qeft_internal.h"
#include "wave.h"

namespace qeft {
namespace {

constexpr float LN2 = 0.693147180559945f, LOG2E = 1.44269504088896f;
constexpr float LEAST = -3.402823466e38f;      // the lowest finite number: a finite bound of M, which a row of nothing but it reaches
constexpr float FAR = -200.f;        // 2^u is 0 from here down: u may stop here, where it is a factor beside 2^u

constexpr uint32_t RANK_NEG_INF = 0x007fffffu, RANK_NAN = 0xff800001u;      // (one above +infinity's)
// A row's address, the same in all lanes
__host__ __device__ __forceinline__ const char* row_at(const void* p, int64_t row, int64_t ld, bool f32) { return (const char*)p + row * ld * (f32 ? 4 : 2); }
__device__ __forceinline__ char* row_at(void* p, int64_t row, int64_t ld, bool f32) { return (char*)p + row * ld * (f32 ? 4 : 2); }

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

// What a row's gradient needs: u = (z by - off) c, p = 2^u share, dz = 2^u (a - dh u), and at_token more at the token
struct Slope {
    float by, off, c, a, dh, at_token;
    int token;
};
// distance: entropy + log share, so that log p + entropy = u ln 2 + distance.  The share stays a factor: as a summand beside the largest logit it would be rounded at that size,
// and all probabilities be off by one factor.
__device__ __forceinline__ Slope make_slope(const Logprob& a, int64_t row, int token, float by, float off, float c, float share, float distance) {
    const float dl = a.dlogp ? a.dlogp[row] : 0.f, ds = a.dlse ? a.dlse[row] : 0.f, dh = a.dentropy ? a.dentropy[row] : 0.f;
    return Slope{by, off, c, a.scale * (ds - dl - (dh != 0.f ? dh * distance : 0.f)) * share, a.scale * dh * LN2 * share, a.scale * dl, a.token ? token : -1};
}
__device__ __forceinline__ float u_of(const Slope& g, float z) { return fmaf(z, g.by, -g.off) * g.c; }
__device__ __forceinline__ float slope_of(const Slope& g, float z) {
    const float u = u_of(g, z);
    return __builtin_amdgcn_exp2f(u) * fmaf(-g.dh, fmaxf(u, FAR), g.a);      // (p is 0 where u is far, not-a-number where u is)
}
template <bool F32>
__device__ __forceinline__ void put_slopes(const Slope& g, const Raw<F32>& v, char* dz, int at, int left) {
    if (left <= 0) return;
    float x[8];
    if (g.dh != 0.f) {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = slope_of(g, v[e]);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = __builtin_amdgcn_exp2f(u_of(g, v[e])) * g.a;
    }
    if ((uint32_t)(g.token - at) < 8u) {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (at + e == g.token) x[e] += g.at_token;
    }
    store<F32>(dz, at, left, x);
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

// ---- rows in registers ------------------------------------------------------------------------------------------------
struct Stats {       // of a part of a row, relative to its own largest logit
    float most, s, t;
};
constexpr float NEAR = 0x1p23f;      // K below which its error is at most 1/2
// K's error where it is below that
__device__ __forceinline__ float residue(float most, float c) {
    const float k = most * c;
    return fabsf(k) < NEAR ? fmaf(most, c, -k) : 0.f;
}
__device__ __forceinline__ float shrink(float from, float to, float c) { return fmaxf((from - to) * c, FAR); }      // (2^FAR is 0: what is further away adds nothing)

// A term of a sum over lanes: rounded for itself.  Joined with the sum's first addition it would be rounded otherwise in the lane that adds it than in the lane it is added
// to, and the lanes' sums would differ.
__device__ __forceinline__ float term(float a, float b) {
#pragma clang fp contract(off)
    return a * b;
}

// Of a row whose statistics are at hand
__device__ __forceinline__ Slope make_slope(const Logprob& a, int64_t row, int token, const Stats& x) {
    const float share = 1.f / x.s;
    return make_slope(a, row, token, 1.f, x.most, a.scale * LOG2E, share, -LN2 * x.t * share);
}

// Where a workgroup's part of a row goes: to the call's outputs, or, one of several parts, to the workspace
struct Part {
    int parts, len;        // parts of a row, values of one
    Stats* stats;          // [m][parts]
    uint64_t* keys;        // [m][parts][top], largest first
    Stats* joined;         // [m] of whole rows, for a gradient that follows
};
constexpr int CANDIDATES = 1024;

__device__ __forceinline__ float logit_at(const Logprob& a, const char* row, int j) { return a.f32 ? ((const float*)row)[j] : (float)((const _Float16*)row)[j]; }
// A row's numbers from its joined statistics, by one thread; zt: the token's logit
__device__ __forceinline__ void put_row(const Logprob& a, const Part& p, int64_t row, float zt, const Stats& x, float ln_s, float entropy) {
    const bool empty = x.s == 0.f;
    const float lse = empty ? -INFINITY : fmaf(x.most, a.scale, ln_s);
    if (a.lse) a.lse[row] = lse;
    if (a.entropy) a.entropy[row] = entropy;
    if (p.joined) p.joined[row] = x;
    if (a.logp) a.logp[row] = empty ? -INFINITY : fmaf(zt - x.most, a.scale, -ln_s);
}
__device__ __forceinline__ void put_top(const Logprob& a, int64_t row, int i, uint64_t key, float most, float ln_s) {
    const bool there = (uint32_t)(key >> 32) > RANK_NEG_INF;
    a.top_index[row * a.ld_top + i] = there ? (int)~(uint32_t)key : -1;
    a.top_logp[row * a.ld_top + i] = there ? fmaf(value_of(key >> 32) - most, a.scale, -ln_s) : -INFINITY;
}

// The largest `top` keys of a workgroup, by rounds: each() calls its argument with every key of the thread.  For what the list of candidates does not hold.
template <class Each, class Put>
__device__ __forceinline__ void top_by_rounds(int top, uint64_t* slots, const Each& each, const Put& put) {
    uint64_t last = ~0ull;
    for (int i = 0; i < top; ++i) {
        uint64_t best = 0;
        each([&](uint64_t x) {
            if (x < last && x > best) best = x;
        });
        best = group_reduce(best, slots, (uint64_t)0, Most());
        if ((uint32_t)(best >> 32) <= RANK_NEG_INF) best = 0;
        last = best;
        if (threadIdx.x == 0) put(i, best);
    }
}
// The largest `top` of the `count` keys in a list: each key's place is the number of larger ones, counted by 16 lanes.
template <class Put>
__device__ __forceinline__ void top_of_list(int top, const uint64_t* list, int count, const Put& put) {
    const int share = threadIdx.x & 15;
    for (int i = threadIdx.x >> 4; i < count; i += blockDim.x >> 4) {      // (a row of lanes together)
        const uint64_t mine = list[i];
        int place = 0;
        for (int j = share; j < count; j += 16) place += list[j] > mine;
        place = row_reduce(place, Sum());
        if (share == 0 && place < top) put(place, mine);
    }
    for (int i = count + threadIdx.x; i < top; i += blockDim.x) put(i, 0);
}
// x of the lanes that want it, behind what `used` counts, one atomic a wave; more than `room` are counted only.  All lanes of the wave call it.
template <class T>
__device__ __forceinline__ void append(bool want, T x, T* list, int room, int* used) {
    const uint64_t who = __ballot(want);
    if (who == 0) return;
    const int lane = threadIdx.x & 63, leader = __builtin_ctzll(who);
    int at = 0;
    if (lane == leader) at = atomicAdd(used, __popcll(who));
    at = __builtin_amdgcn_readlane(at, leader) + __popcll(who & ((1ull << lane) - 1));
    if (want && at < room) list[at] = x;
}

// Workgroup = a row, or a part of one: V octets a thread.
template <int V, bool F32, bool GRAD>
__global__ __launch_bounds__(1024) void logprob_row_kernel(Logprob a, Part p) {
    __shared__ float buf[3][16];
    __shared__ uint32_t maxima[GRAD ? 1 : 256], border;
    __shared__ uint64_t list[GRAD ? 1 : CANDIDATES], slots[16];
    __shared__ uint16_t reached[GRAD ? 1 : 1024];
    __shared__ int used[2];
    const int64_t row = p.parts == 1 ? blockIdx.x : blockIdx.x / p.parts;
    const int part = p.parts == 1 ? 0 : (int)(blockIdx.x - row * p.parts), from = part * p.len, n = min(p.len, a.n - from), T = blockDim.x;
    const char* begin = row_at(a.z, row, a.ldz, F32);
    const char* z = begin + (size_t)from * (F32 ? 4 : 2);
    const int token = a.token ? a.token[row] : -1;
    if (a.token && (token < 0 || token >= a.n)) {
        if (p.parts > 1) return;      // (the join leaves it out)
        left_out(a, row);
        if (GRAD) zero_row<F32>(row_at(a.dz, row, a.lddz, F32), a.n);
        return;
    }
    // (before the gradient's first store, which may go to z itself)
    const float zt = a.logp && p.parts == 1 && threadIdx.x == 0 ? logit_at(a, begin, token) : 0.f;
    // Whole octets by one load each; a partial one is some thread's v[i] (the code for it once, not V times).
    const int whole = n / 8, last = threadIdx.x == (whole & (T - 1)) && (n & 7) ? whole / T : -1;
    Raw<F32> v[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        v[i].fill(Raw<F32>::NEG_INF);
        if ((int)threadIdx.x + T * i < whole) v[i].load(z, 8 * (threadIdx.x + T * i), 8);
    }
    if (last >= 0) {
        Raw<F32> x;
        x.load(z, 8 * whole, n & 7, Raw<F32>::NEG_INF);
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (i == last) v[i] = x;
    }
    const float c = a.scale * LOG2E;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = T >> 6;
    float mine = -INFINITY;
#pragma unroll
    for (int i = 0; i < V; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) mine = fmaxf(mine, v[i][e]);
    Stats x{fmaxf(wave_reduce(mine, MostFloat()), LEAST), 0.f, 0.f};
    // (kept as loaded between the steps, not as twice the registers of converted values)
    auto pin = [&] {
#pragma unroll
        for (int i = 0; i < V; ++i) v[i].hold();
    };
    pin();
    uint32_t rank = 0;
    if constexpr (!GRAD) {      // for the alternatives, see there: shared with the statistics' barrier
        if (a.top > 0) {
            rank = rank_of(mine);
            uint32_t group = rank;
            const int side = T > 256 ? 4 : 1;      // threads of a group: neighbours
            if (side == 4) {
                group = max(group, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)group, 0xb1, 0xf, 0xf, false));      // quad_perm 1 0 3 2
                group = max(group, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)group, 0x4e, 0xf, 0xf, false));      // quad_perm 2 3 0 1
            }
            if (threadIdx.x % side == 0) maxima[threadIdx.x / side] = group;
            for (int i = T / side + threadIdx.x; i < 256; i += T) maxima[i] = 0;
            if (threadIdx.x < 2) used[threadIdx.x] = 0;
        }
    }
    const bool wants_t = a.entropy || a.dentropy;
    {
        float s[2] = {}, t[2] = {};
        auto sums = [&](const auto& far) {
#pragma unroll
            for (int i = 0; i < V; ++i) {
                if (wants_t) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float u = far(v[i][e]), y = __builtin_amdgcn_exp2f(u);
                        s[e & 1] += y;
                        t[e & 1] = fmaf(y, fmaxf(u, FAR), t[e & 1]);
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e) s[e & 1] += __builtin_amdgcn_exp2f(far(v[i][e]));
                }
            }
        };
        const float k = x.most * c;
        if (fabsf(k) < NEAR) sums([&](float z) { return fmaf(z, c, -k); });
        else sums([&](float z) { return (z - x.most) * c; });
        x.s = wave_reduce(s[0] + s[1], Sum());
        if (wants_t) x.t = wave_reduce(t[0] + t[1], Sum());
    }
    if (lane == 0) {
        buf[0][wave] = x.most;
        buf[1][wave] = x.s;
        buf[2][wave] = x.t;
    }
    __syncthreads();
    if (waves > 1) {      // the waves' statistics joined, a lane per wave
        const int w = lane & 15;
        const bool there = w < waves;
        const Stats y{there ? buf[0][w] : LEAST, there ? buf[1][w] : 0.f, there ? buf[2][w] : 0.f};
        x.most = row_reduce(y.most, MostFloat());
        const float d = shrink(y.most, x.most, c) - residue(y.most, c), f = __builtin_amdgcn_exp2f(d);
        x.s = row_reduce(term(y.s, f), Sum());
        x.t = row_reduce(term(f, fmaf(d, y.s, y.t)), Sum());
    } else {
        const float d = -residue(x.most, c), f = __builtin_amdgcn_exp2f(d);
        x.t = f * fmaf(d, x.s, x.t);
        x.s *= f;
    }
    pin();
    const bool empty = x.s == 0.f;
    const float ln_s = logf(x.s), entropy = empty ? 0.f : ln_s - LN2 * (x.t / x.s);
    if (p.parts == 1) {
        if (threadIdx.x == 0) put_row(a, p, row, zt, x, ln_s, entropy);
    } else if (threadIdx.x == 0) p.stats[blockIdx.x] = x;
    if constexpr (!GRAD) {
        if (a.top == 0) return;
        // Candidates: whatever reaches the top-th largest of the maxima of groups of threads (64 groups for up to 32 alternatives, 256 for more).  Few threads have any, and few of
        // their values are: the threads are listed, then all look through the listed ones' values, read again.  The few candidates are ordered by comparing each with each.  Rows where
        // many are (equal logits) or with not-a-number, which no maximum shows, go by rounds.
        auto put = [&](int i, uint64_t key) {
            if (p.parts == 1) put_top(a, row, i, key, x.most, ln_s);
            else p.keys[(size_t)blockIdx.x * a.top + i] = key;
        };
        uint32_t bound = 0;
        {
            uint32_t g[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) g[i] = maxima[lane + 64 * i];
            if (a.top <= 32 && waves >= 4) {
                // each wave looks at a share of the 64: is it the one with fewer than `top` above it and `top` with it?
                const uint32_t most = max(max(g[0], g[1]), max(g[2], g[3]));
                for (int i = 64 / waves * wave; i < 64 / waves * (wave + 1); ++i) {
                    const uint32_t x = (uint32_t)__builtin_amdgcn_readlane((int)most, i);
                    if ((int)__popcll(__ballot(most > x)) < a.top && (int)__popcll(__ballot(most >= x)) >= a.top && lane == 0) border = x;      // (the same, if several)
                }
                __syncthreads();
                bound = border;
            } else {
#pragma unroll 1
                for (uint32_t bit = 0x80000000u; bit >= 0x10000u; bit >>= 1) {      // cut to 16 bits
                    int count = 0;
#pragma unroll
                    for (int i = 0; i < 4; ++i) count += __popcll(__ballot(g[i] >= (bound | bit)));
                    if (count >= a.top) bound |= bit;
                }
            }
        }
        bound = max(bound, RANK_NEG_INF + 1);
        append(rank >= bound, (uint16_t)threadIdx.x, reached, 1024, &used[0]);
        __syncthreads();
        const int looked = used[0] * 8 * V;
        for (int i0 = 0; i0 < looked; i0 += T) {
            const int i = i0 + threadIdx.x;
            uint64_t key = 0;
            if (i < looked) {
                const int j = 8 * (reached[i / (8 * V)] + T * (i / 8 % V)) + i % 8;
                if (j < n) key = (uint64_t)rank_of(logit_at(a, z, j)) << 32 | (uint32_t)~(from + j);
            }
            append((uint32_t)(key >> 32) >= bound, key, list, CANDIDATES, &used[1]);
        }
        __syncthreads();
        const int count = used[1];
        if (count <= CANDIDATES && x.s == x.s) top_of_list(a.top, list, count, put);
        else {
            auto each = [&](auto&& f) {      // (from memory: every value's key would stay in registers through the rounds)
                for (int at = 8 * threadIdx.x; at < n; at += 8 * T) {
                    Raw<F32> x;
                    x.load(z, at, n - at, Raw<F32>::NEG_INF);
#pragma unroll
                    for (int e = 0; e < 8; ++e) f((uint64_t)rank_of(x[e]) << 32 | (uint32_t)~(from + at + e));
                }
            };
            top_by_rounds(a.top, slots, each, put);
        }
    } else {
        char* dz = row_at(a.dz, row, a.lddz, F32);
        if (empty) return zero_row<F32>(dz, a.n);
        const Slope g = make_slope(a, row, token, x);
        Raw<F32> x = v[0];
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int o = threadIdx.x + T * i;
            if (o < whole) put_slopes(g, v[i], dz, 8 * o, 8);
            if (i == last) x = v[i];
        }
        if (last >= 0) put_slopes(g, x, dz, 8 * whole, n & 7);
    }
}

// The parts of a row joined: a lane a part where a wave has lanes for them (each wave for itself, no barrier), else a thread a part (256 at most).
__global__ __launch_bounds__(256) void logprob_join_kernel(Logprob a, Part p) {
    __shared__ float buf[3][16];
    __shared__ uint64_t list[CANDIDATES], slots[16];
    __shared__ int used;
    const int64_t row = blockIdx.x;
    const int token = a.token ? a.token[row] : -1;
    if (a.token && (token < 0 || token >= a.n)) {
        left_out(a, row);
        return;
    }
    const bool alone = p.parts <= 64;
    const int t = threadIdx.x, i = alone ? t & 63 : t;
    const float zt = a.logp && t == 0 ? logit_at(a, row_at(a.z, row, a.ldz, a.f32), token) : 0.f;
    const Stats y = i < p.parts ? p.stats[row * p.parts + i] : Stats{LEAST, 0.f, 0.f};
    const uint64_t* keys = p.keys + (size_t)row * p.parts * a.top;
    const int total = p.parts * a.top;
    // (asked for together with the statistics: a part's last key, and this thread's first)
    const uint64_t last = a.top > 0 && i < p.parts ? keys[(size_t)i * a.top + a.top - 1] : 0, first = t < total ? keys[t] : 0;
    if (t == 0) used = 0;
    auto joined = [&](auto v, auto* slots, auto none, const auto& op) { return alone ? wave_reduce(v, op) : group_reduce(v, slots, none, op); };
    Stats x;
    x.most = joined(y.most, buf[0], LEAST, MostFloat());
    const float d = shrink(y.most, x.most, a.scale * LOG2E), f = __builtin_amdgcn_exp2f(d);
    x.s = joined(term(y.s, f), buf[1], 0.f, Sum());
    x.t = joined(term(f, fmaf(d, y.s, y.t)), buf[2], 0.f, Sum());
    const float ln_s = logf(x.s), entropy = x.s == 0.f ? 0.f : ln_s - LN2 * (x.t / x.s);
    if (t == 0) put_row(a, p, row, zt, x, ln_s, entropy);
    if (a.top == 0) return;
    // a part whose last key is this large has enough of them
    const uint64_t bound = max(joined(last, slots, (uint64_t)0, Most()), (uint64_t)1);
    __syncthreads();
    for (int j0 = 0; j0 < total; j0 += blockDim.x) {
        const uint64_t key = j0 == 0 ? first : j0 + t < total ? keys[j0 + t] : 0;
        append(key >= bound, key, list, CANDIDATES, &used);
    }
    __syncthreads();
    const int count = used;
    auto put = [&](int at, uint64_t key) { put_top(a, row, at, key, x.most, ln_s); };
    if (count <= CANDIDATES) top_of_list(a.top, list, count, put);
    else top_by_rounds(a.top, slots, [&](auto&& g) {
        for (int j = t; j < total; j += blockDim.x) g(keys[j]);
    }, put);
}

// ---- the gradient alone -------------------------------------------------------------------------------------------------
constexpr int CHUNK = 8192;      // values of a workgroup
template <bool F32, bool JOINED>
__global__ __launch_bounds__(256) void logprob_bwd_kernel(Logprob a, const Stats* joined, int chunks, int64_t first) {
    const int64_t row = first + blockIdx.x / chunks;
    const int from = (int)(blockIdx.x % chunks) * CHUNK, n = min(CHUNK, a.n - from);
    const char* z = row_at(a.z, row, a.ldz, F32) + (size_t)from * (F32 ? 4 : 2);
    char* dz = row_at(a.dz, row, a.lddz, F32) + (size_t)from * (F32 ? 4 : 2);
    const int token = a.token ? a.token[row] : -1;
    bool none = a.token && (token < 0 || token >= a.n);
    Slope g;
    Raw<F32> v[CHUNK / 2048];
    if (!none) {
#pragma unroll
        for (int i = 0; i < CHUNK / 2048; ++i) v[i].load(z, 8 * threadIdx.x + 2048 * i, n - (int)(8 * threadIdx.x + 2048 * i));
        if constexpr (JOINED) {
            const Stats x = joined[row];
            none = x.s == 0.f;
            g = make_slope(a, row, token - from, x);
        } else {
            const float lse = a.lse_in[row];
            none = lse == -INFINITY;
            g = make_slope(a, row, token - from, a.scale, lse, LOG2E, 1.f, a.entropy_in ? a.entropy_in[row] : 0.f);
        }
    }
    if (none) return zero_row<F32>(dz, n);
#pragma unroll
    for (int i = 0; i < CHUNK / 2048; ++i) put_slopes(g, v[i], dz, 8 * threadIdx.x + 2048 * i, n - (int)(8 * threadIdx.x + 2048 * i));
}

// ---- what goes where ----------------------------------------------------------------------------------------------------
struct Plan {
    int threads, octets;     // of a workgroup, a thread
    int parts, len;          // parts of a row
    int64_t rows;            // that the workspace holds the parts of
    size_t keys_at, joined_at, bytes;
};
constexpr size_t PARTS_BYTES = 64 << 20;      // of a workspace at most: more rows go in rounds
constexpr int64_t MOST_THREADS = (int64_t)1 << 31;      // of a launch (a grid has fewer than 2^32): more go in rounds too
constexpr int FINER = 32768, FINER_FROM = 65536, FINER_GROUPS = 256;
Plan plan_of(int n, bool f32, int64_t m, int top) {
    const int most = f32 ? 8 : 16;      // octets that a thread of 1024 holds beside its work: 64 registers
    Plan p{};
    const int octets = ceil_div(n, 8), fit = 1024 * most;
    int parts = ceil_div(octets, fit);
    // A CU takes 9 us for 130000 values (exponentials and sums, 260 KB): where there are CUs for all of them, parts of 32768 values save more than the join's launch
    // costs.  1 x 130001 with 20 alternatives 15.7 -> 12.5 us, 57 x 130001 16.2 -> 14.4, 16 x 262144 18.7 -> 11.9, 1 x 68849 13.0 -> 11.3, without alternatives 10.0 -> 8.6; 1 x 50257 would go
    // 8.8 -> 10.4.  With the gradient in the same call the parts mean a third launch and a second read, and gain all the same: waited for, 1 x 68849 14.6 -> 12.7, 1 x 130001 17.8 -> 12.5,
    // 60 x 100001 18.6 -> 17.6; behind one another 11.9 -> 12.0, 15.2 -> 12.1, 60 x 115001 17.1 -> 15.6 (60 x 68849 13.3 -> 13.5).
    const int finer = ceil_div(n, FINER);
    if (n > FINER_FROM && finer > parts && m * finer <= FINER_GROUPS) parts = finer;
    p.parts = parts;
    int per = ceil_div(octets, parts);
    // As few threads as hold a row in some octets each, where rows are many; where they are few more would be quicker.  With 64 / 256 / 1024 threads 4000 fp16 rows of 500: 5.6 / 7.8 / 22.7 us,
    // of 2000: 6.3 / 7.8 / 22.9, of 8000: 16.9 / 14.4 / 24.8; 64 rows of 4000 with 5 alternatives 8.1 / 5.4, of 8000 10.4 / 5.8 / 5.4; of 16000 with 256 / 1024 threads 6.7 / 5.9, 4000 of them 24.2 / 30.6.
    const int threads = per <= 256 ? 64 : per <= 2048 ? 256 : 1024;
    int v = 1;
    while (v * threads < per) v *= 2;
    p.threads = threads;
    p.octets = v;
    p.len = parts > 1 ? 8 * threads * v : n;
    if (parts == 1) return p;
    p.parts = parts = ceil_div(n, p.len);
    const size_t row = (size_t)parts * (sizeof(Stats) + top * sizeof(uint64_t));
    p.rows = std::min({m, (int64_t)(PARTS_BYTES / row), MOST_THREADS / 1024 / parts});
    p.keys_at = (size_t)p.rows * parts * sizeof(Stats) + 15 & ~(size_t)15;
    p.joined_at = p.rows < m ? PARTS_BYTES + 16 : p.keys_at + (size_t)p.rows * parts * top * sizeof(uint64_t);
    p.bytes = p.joined_at + (size_t)m * sizeof(Stats);
    return p;
}

template <bool F32, bool GRAD>
void launch_rows(const Plan& q, const Logprob& a, const Part& p, hipStream_t s) {
    const unsigned grid = (unsigned)(a.m * p.parts);
    switch (q.octets) {
        case 1: logprob_row_kernel<1, F32, GRAD><<<grid, q.threads, 0, s>>>(a, p); break;
        case 2: logprob_row_kernel<2, F32, GRAD><<<grid, q.threads, 0, s>>>(a, p); break;
        case 4: logprob_row_kernel<4, F32, GRAD><<<grid, q.threads, 0, s>>>(a, p); break;
        case 8: logprob_row_kernel<8, F32, GRAD><<<grid, q.threads, 0, s>>>(a, p); break;
        default:
            if constexpr (!F32) logprob_row_kernel<16, F32, GRAD><<<grid, q.threads, 0, s>>>(a, p);
    }
}
template <bool F32>
void launch_bwd(const Logprob& a, const Stats* joined, hipStream_t s) {
    const int chunks = ceil_div(a.n, CHUNK);
    const int64_t most = (MOST_THREADS / 256) / chunks;
    for (int64_t first = 0; first < a.m; first += most) {
        const unsigned grid = (unsigned)(std::min(most, a.m - first) * chunks);
        if (joined) logprob_bwd_kernel<F32, true><<<grid, 256, 0, s>>>(a, joined, chunks, first);
        else logprob_bwd_kernel<F32, false><<<grid, 256, 0, s>>>(a, joined, chunks, first);
    }
}
template <bool F32>
void launch_fwd(const Logprob& a, hipStream_t s) {
    const Plan q = plan_of(a.n, F32, a.m, a.top);
    Part p{q.parts, q.len, nullptr, nullptr, nullptr};
    if (q.parts == 1) {
        if (a.dz) launch_rows<F32, true>(q, a, p, s);
        else launch_rows<F32, false>(q, a, p, s);
        return;
    }
    p.stats = (Stats*)a.ws;
    p.keys = (uint64_t*)(a.ws + q.keys_at);
    Stats* const joined = a.dz ? (Stats*)(a.ws + q.joined_at) : nullptr;
    for (int64_t from = 0; from < a.m; from += q.rows) {
        Logprob b = a;
        b.m = std::min(q.rows, a.m - from);
        b.z = row_at(a.z, from, a.ldz, F32);
        auto later = [&](auto*& at, int64_t by) {
            if (at) at += by;
        };
        later(b.token, from), later(b.logp, from), later(b.lse, from), later(b.entropy, from);
        later(b.top_logp, from * a.ld_top), later(b.top_index, from * a.ld_top);
        p.joined = joined ? joined + from : nullptr;
        launch_rows<F32, false>(q, b, p, s);
        logprob_join_kernel<<<(unsigned)b.m, q.parts <= 64 && a.top == 0 ? 64 : 256, 0, s>>>(b, p);
    }
    if (a.dz) launch_bwd<F32>(a, joined, s);
}

}  // namespace

// What m rows need, or fewer: finer parts are for few rows only, and a workspace for many has to do for them.
size_t logprob_workspace(int n, bool f32, int64_t m, int top) {
    const int64_t few = FINER_GROUPS / ceil_div(n, FINER);
    return std::max(plan_of(n, f32, m, top).bytes, few > 0 && few < m ? plan_of(n, f32, few, top).bytes : 0);
}

hipError_t logprob_fwd(const Logprob& a, hipStream_t s) {
    if (a.f32) launch_fwd<true>(a, s);
    else launch_fwd<false>(a, s);
    return hipGetLastError();
}

hipError_t logprob_bwd(const Logprob& a, hipStream_t s) {
    if (a.f32) launch_bwd<true>(a, nullptr, s);
    else launch_bwd<false>(a, nullptr, s);
    return hipGetLastError();
}

}  // namespace qeft
