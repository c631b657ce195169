// The norms around a decoder block (qeft_norm_fwd, qeft_norm_bwd): residual addition with gate and scale, the norm after a block and the norm before the next,
// in one pass over the data, and their gradients in another.
//
//   u = y or unit(y) w_post      h = r + scale gate u      x = unit(h) w_pre      unit(z) = z / sqrt(mean z^2 + eps)
//   t  = dh + rs (a - hh mean(a hh)),     a = dx w_pre, hh = unit(h), rs = 1 / sqrt(mean h^2 + eps);    dr = t
//   du = scale gate t;   dy = du, or rs_y (a' - yh mean(a' yh)) with a' = du w_post, yh = unit(y)
//   dw_pre = sum dx hh     dw_post = sum du yh     dgate = scale u t
//
// Bytes bound both: a row stays in registers from its one load to its one store.  Rows of up to 512 values are a wave's (sums by shuffles); longer ones up to
// 8192 have a thread per 8 values, so that a load is 16 or 32 bytes a lane; longer still two and (forward) four times 8 values a thread, and beyond FWD_MAX
// or BWD_MAX values the row is read again for each step.
// The gradient's workgroups stay for many rows: the column sums are kept in registers, a workgroup's row groups join theirs in LDS, and one slab per
// workgroup goes to the workspace, summed by a second launch in a fixed order.  The next row's loads are issued before the current one's sums: a
// CU has one or two workgroups and nothing else to hide them.
// Measured: forward 4096 x 4096, fp32 residual: 39 us, 5.2 TB/s; gradient 4096 x 8192 with both norms and a channel gate: 122 - 125 us, 5 TB/s, 6 of it the slabs' sum;
// 333 x 5120, token gate: 15 us, where the bytes take 5.3 (two rows a workgroup and the second launch, latencies).
#include <algorithm>
#include "qeft_internal.h"
#include "wave.h"

namespace qeft {
namespace {

typedef uint32_t u4 __attribute__((ext_vector_type(4)));
typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef float f4 __attribute__((ext_vector_type(4)));

constexpr int FWD_MAX = 32768;    // values of a row that the forward keeps in registers (1024 threads x 4 octets)
constexpr int BWD_MAX = 16384;    // and the gradient (1024 x 2: beside three column sums)

// A row's address, the same in all lanes: kept from the optimiser, which would otherwise add a lane's offset to every array's base outside the loop over
// the rows and hold those sums, two registers each (the gradient has eight arrays), instead of adding in the load.
__device__ __forceinline__ const char* row_of(const void* p, int64_t row, int64_t ld, bool f32) {
    const char* r = (const char*)p + row * ld * (f32 ? 4 : 2);
    asm volatile("" : "+s"(r));
    return r;
}
__device__ __forceinline__ char* row_of(void* p, int64_t row, int64_t ld, bool f32) { return const_cast<char*>(row_of((const void*)p, row, ld, f32)); }

// Eight values of a row as loaded.  left: how many of them exist; a row's last octet may be partial, and is read value by value, the last one first.
template <bool F32> struct Raw;
template <> struct Raw<false> {
    u4 v;
    __device__ __forceinline__ void load(const void* row, uint32_t at, int left) {
        const char* p = (const char*)row + 2 * at;
        if (left >= 8) {
            v = *reinterpret_cast<const u4*>(p);
            return;
        }
        v = u4{0, 0, 0, 0};
#pragma unroll 1
        for (int e = left - 1; e >= 0; --e) {
            const uint32_t x = *reinterpret_cast<const uint16_t*>(p + 2 * e);
            v = u4{v.x << 16 | x, v.y << 16 | v.x >> 16, v.z << 16 | v.y >> 16, v.w << 16 | v.z >> 16};
        }
    }
    __device__ __forceinline__ float operator[](int e) const { return (float)__builtin_bit_cast(h8, v)[e]; }
    __device__ __forceinline__ void clear() { v = u4{0, 0, 0, 0}; }
    // Eight values stay four registers: without this the compiler converts once and keeps eight (across a loop for a row of weights).
    __device__ __forceinline__ void pin() { asm volatile("" : "+v"(v)); }
};
template <> struct Raw<true> {
    f4 a, b;
    __device__ __forceinline__ void load(const void* row, uint32_t at, int left) {
        const char* p = (const char*)row + 4 * at;
        if (left >= 8) {
            a = *reinterpret_cast<const f4*>(p);
            b = *reinterpret_cast<const f4*>(p + 16);
            return;
        }
        clear();
#pragma unroll 1
        for (int e = left - 1; e >= 0; --e) {
            b = f4{a.w, b.x, b.y, b.z};
            a = f4{*reinterpret_cast<const float*>(p + 4 * e), a.x, a.y, a.z};
        }
    }
    __device__ __forceinline__ float operator[](int e) const { return e < 4 ? a[e & 3] : b[e & 3]; }
    __device__ __forceinline__ void clear() { a = b = f4{0.f, 0.f, 0.f, 0.f}; }
    __device__ __forceinline__ void pin() {}
};
typedef Raw<false> Half8;

// x goes to the row, rounded to its type (which x then is too)
template <bool F32>
__device__ __forceinline__ void store(void* row, uint32_t at, int left, float (&x)[8]) {
    if (F32) {
        char* p = (char*)row + 4 * at;
        f4 a = {x[0], x[1], x[2], x[3]}, b = {x[4], x[5], x[6], x[7]};
        if (left >= 8) {
            *reinterpret_cast<f4*>(p) = a;
            *reinterpret_cast<f4*>(p + 16) = b;
            return;
        }
#pragma unroll 1
        for (int e = 0; e < left; ++e) {
            *reinterpret_cast<float*>(p + 4 * e) = a.x;
            a = f4{a.y, a.z, a.w, b.x};
            b = f4{b.y, b.z, b.w, b.w};
        }
        return;
    }
    h8 h;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        h[e] = (_Float16)x[e];
        x[e] = (float)h[e];
    }
    u4 v = __builtin_bit_cast(u4, h);
    char* p = (char*)row + 2 * at;
    if (left >= 8) {
        *reinterpret_cast<u4*>(p) = v;
        return;
    }
#pragma unroll 1
    for (int e = 0; e < left; ++e) {
        *reinterpret_cast<uint16_t*>(p + 2 * e) = (uint16_t)v.x;
        v = u4{v.x >> 16 | v.y << 16, v.y >> 16 | v.z << 16, v.z >> 16 | v.w << 16, v.w >> 16};
    }
}
template <bool F32>
__device__ __forceinline__ void round_to(float (&x)[8]) {
    if (F32) return;
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = (float)(_Float16)x[e];
}
// N sums over the `waves` waves from `first` on of a workgroup (a row's), the same for every thread of them.  buf: the LDS slots of this call; the
// call before it on the same slots must lie behind a barrier.
template <int N>
__device__ __forceinline__ void row_sums(float (&s)[N], float (*buf)[16], int first, int waves) {
#pragma unroll
    for (int i = 0; i < N; ++i) s[i] = wave_reduce(s[i], Sum());
    if (waves == 1) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    if (lane == 0)
#pragma unroll
        for (int i = 0; i < N; ++i) buf[i][wave] = s[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) s[i] = waves_reduce(buf[i], first, waves, 0.f, Sum());
}

// ---- forward ----------------------------------------------------------------------------------------------------------
// A row by `waves` waves, V octets a thread; workgroups of one row, or of four one-wave rows.
template <int V, bool F32>
__global__ __launch_bounds__(1024) void norm_fwd_kernel(Norm a, int waves) {
    __shared__ float buf[2][1][16];
    const int T = 64 * waves, group = __builtin_amdgcn_readfirstlane(threadIdx.x / T), tid = threadIdx.x - group * T;
    const int64_t row = (int64_t)blockIdx.x * (blockDim.x / T) + group;
    if (row >= a.m) return;   // (whole waves of one-wave rows only: no barrier follows for them)
    const int first = group * waves;
    const float inv = 1.f / (float)a.n;
    const void* r = row_of(a.r, row, a.ldr, F32);
    float h[V][8];
    Raw<F32> rr[V];
    Half8 yy[V], gg[V];
    const bool has_y = a.y != nullptr, has_g = a.gate_kind != QEFT_GATE_NONE && has_y;
    const __half* y = has_y ? a.y + row * a.ldy : nullptr;
    const __half* gate = has_g ? a.gate + (a.gate_kind == QEFT_GATE_TOKEN ? row * a.ldg : 0) : nullptr;
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const int at = 8 * (tid + T * v), left = a.n - at;
        rr[v].clear();
        yy[v].clear();
        if (left > 0) {
            rr[v].load(r, at, left);
            if (has_y) yy[v].load(y, at, left);
            if (has_g) gg[v].load(gate, at, left);
        }
    }
    float post = 1.f;
    if (a.w_post) {
        float s[1] = {0.f};
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
            for (int e = 0; e < 8; ++e) s[0] = fmaf(yy[v][e], yy[v][e], s[0]);
        row_sums(s, buf[0], first, waves);
        post = 1.f / sqrtf(fmaf(s[0], inv, a.eps));
    }
    float s[1] = {0.f};
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const int at = 8 * (tid + T * v), left = a.n - at;
        if (left <= 0) continue;
        if (has_y) {
            Half8 wp;
            if (a.w_post) wp.load(a.w_post, at, left);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                float u = yy[v][e];
                if (a.w_post) u = u * post * wp[e];
                if (has_g) u *= gg[v][e];
                h[v][e] = fmaf(a.scale, u, rr[v][e]);
            }
            if (a.h) store<F32>(row_of(a.h, row, a.ldh, F32), at, left, h[v]);
            else round_to<F32>(h[v]);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) h[v][e] = rr[v][e];
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) s[0] = e < left ? fmaf(h[v][e], h[v][e], s[0]) : s[0];
    }
    row_sums(s, buf[1], first, waves);
    const float rs = 1.f / sqrtf(fmaf(s[0], inv, a.eps));
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const int at = 8 * (tid + T * v), left = a.n - at;
        if (left <= 0) continue;
        Half8 w;
        w.load(a.w_pre, at, left);
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = h[v][e] * rs * w[e];
        store<false>(row_of((void*)a.x, row, a.ldx, false), at, left, x);
    }
}

// Rows longer than the registers of a workgroup: read once for unit(y), once for h, once more for x.
template <bool F32>
__global__ __launch_bounds__(1024) void norm_fwd_long_kernel(Norm a) {
    __shared__ float buf[2][1][16];
    const int64_t row = blockIdx.x;
    const float inv = 1.f / (float)a.n;
    const void* r = row_of(a.r, row, a.ldr, F32);
    const __half* y = a.y ? a.y + row * a.ldy : nullptr;
    const __half* gate = a.gate_kind != QEFT_GATE_NONE && y ? a.gate + (a.gate_kind == QEFT_GATE_TOKEN ? row * a.ldg : 0) : nullptr;
    void* hrow = a.h ? row_of(a.h, row, a.ldh, F32) : nullptr;
    float post = 1.f;
    if (a.w_post) {
        float s[1] = {0.f};
        for (int at = 8 * threadIdx.x; at < a.n; at += 8192) {
            Half8 v;
            v.load(y, at, min(8, a.n - at));
#pragma unroll
            for (int e = 0; e < 8; ++e) s[0] = fmaf(v[e], v[e], s[0]);
        }
        row_sums(s, buf[0], 0, 16);
        post = 1.f / sqrtf(fmaf(s[0], inv, a.eps));
    }
    auto make_h = [&](int at, int left, float (&h)[8]) {
        Raw<F32> rr;
        rr.load(r, at, left);
        if (!y) {
#pragma unroll
            for (int e = 0; e < 8; ++e) h[e] = rr[e];
            return;
        }
        Half8 yy, wp, gg;
        yy.load(y, at, left);
        if (a.w_post) wp.load(a.w_post, at, left);
        if (gate) gg.load(gate, at, left);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            float u = yy[e];
            if (a.w_post) u = u * post * wp[e];
            if (gate) u *= gg[e];
            h[e] = fmaf(a.scale, u, rr[e]);
        }
        round_to<F32>(h);
    };
    float s[1] = {0.f};
    for (int at = 8 * threadIdx.x; at < a.n; at += 8192) {
        const int left = min(8, a.n - at);
        float h[8];
        make_h(at, left, h);
        if (hrow) store<F32>(hrow, at, left, h);
        for (int e = 0; e < 8; ++e) s[0] = e < left ? fmaf(h[e], h[e], s[0]) : s[0];
    }
    row_sums(s, buf[1], 0, 16);
    const float rs = 1.f / sqrtf(fmaf(s[0], inv, a.eps));
    for (int at = 8 * threadIdx.x; at < a.n; at += 8192) {
        const int left = min(8, a.n - at);
        float h[8], x[8];
        if (hrow) {   // (r may be the same row; a thread reads back what it wrote)
            Raw<F32> hh;
            hh.load(hrow, at, left);
#pragma unroll
            for (int e = 0; e < 8; ++e) h[e] = hh[e];
        } else make_h(at, left, h);
        Half8 w;
        w.load(a.w_pre, at, left);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = h[e] * rs * w[e];
        store<false>(row_of((void*)a.x, row, a.ldx, false), at, left, x);
    }
}

// ---- gradient -----------------------------------------------------------------------------------------------------------
// The column sums of one slab: dw_pre, dw_post, dgate, each [slabs][pitch] in the workspace, or the outputs themselves where one workgroup made it all.
struct Sums {
    float* slab[3];
    int64_t pitch;
    int slabs;
};

template <int V, bool F32>
struct RowIn {
    Half8 dx[V], y[V], g[V];
    Raw<F32> h[V], dh[V];
};

// Workgroup = `groups` rows at a time, `waves` waves a row, V octets a thread.  POST: w_post is given; GATE: 0 none, 1 channel, 2 token.
template <int V, bool F32, bool POST, int GATE>
__global__ __launch_bounds__(1024) void norm_bwd_kernel(Norm a, Sums S, int waves, int groups, int rounds) {
    extern __shared__ __align__(16) float joined[];   // [groups][64 waves][8 V] if groups > 1, then held
    __shared__ float buf[4][3][16];
    const int T = 64 * waves, group = __builtin_amdgcn_readfirstlane(threadIdx.x / T), tid = threadIdx.x - group * T;   // (rows' addresses are then scalar)
    const int first = group * waves;
    const float inv = 1.f / (float)a.n;
    const bool has_y = a.y != nullptr, has_dh = a.dh != nullptr;
    // With both norms (and V == 1) the weights and a channel gate, 12 registers a thread, lie in LDS, read again by each step.
    constexpr bool IN_LDS = POST && V == 1;
    u4* held = reinterpret_cast<u4*>(joined + (groups > 1 ? blockDim.x * 8 * V : 0));   // [3][64 waves]
    Half8 wpre[V], wpost[V], gch[V];
    // Two octets a thread leave no registers for two of the three sums: they lie in LDS, where every thread adds to its own columns.
    constexpr bool SUMS_IN_LDS = V > 1;
    f4* sums_at = reinterpret_cast<f4*>(joined) + threadIdx.x;   // [w_pre, w_post][octet][half][threads]
    auto add_to = [&](int which, int v, const float (&x)[8]) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            f4& s = sums_at[(size_t)((which * V + v) * 2 + h) * blockDim.x];
            s += f4{x[4 * h], x[4 * h + 1], x[4 * h + 2], x[4 * h + 3]};
        }
    };
    if (SUMS_IN_LDS)
        for (int i = 0; i < (POST ? 2 : 1) * V * 2; ++i) sums_at[(size_t)i * blockDim.x] = f4{0.f, 0.f, 0.f, 0.f};
    float spre[V][8] = {}, spost[V][8] = {}, sgate[V][8] = {};
    const int64_t step = (int64_t)gridDim.x * groups;
    // what a row's first sums need, and the rest: the next row's are loaded apart, as registers fall free
    auto load_sums = [&](int64_t row, RowIn<V, F32>& in) {
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int at = 8 * (tid + T * v), left = a.n - at;
            in.dx[v].clear();
            in.y[v].clear();
            in.h[v].clear();
            if (left > 0 && row < a.m) {
                in.h[v].load(row_of(a.r, row, a.ldr, F32), at, left);
                in.dx[v].load(row_of(a.dx, row, a.lddx, false), at, left);
                if (has_y) in.y[v].load(row_of(a.y, row, a.ldy, false), at, left);
            }
        }
    };
    auto load_rest = [&](int64_t row, RowIn<V, F32>& in) {
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int at = 8 * (tid + T * v), left = a.n - at;
            in.g[v].clear();
            in.dh[v].clear();
            if (left > 0 && row < a.m) {
                if (has_dh) in.dh[v].load(row_of(a.dh, row, a.lddh, F32), at, left);
                if (GATE == QEFT_GATE_TOKEN) in.g[v].load(row_of(a.gate, row, a.ldg, false), at, left);
            }
        }
    };
    int64_t row = (int64_t)blockIdx.x * groups + group;
    RowIn<V, F32> in;
    load_sums(row, in);
    load_rest(row, in);
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const int at = 8 * (tid + T * v), left = a.n - at;
        wpre[v].clear();
        wpost[v].clear();
        gch[v].clear();
        if (left > 0) {
            wpre[v].load(a.w_pre, at, left);
            if (POST) wpost[v].load(a.w_post, at, left);
            if (GATE == QEFT_GATE_CHANNEL) gch[v].load(a.gate, at, left);
        }
    }
    if (IN_LDS) {
        if (group == 0) {
            held[tid] = wpre[0].v;
            held[T + tid] = wpost[0].v;
            if (GATE == QEFT_GATE_CHANNEL) held[2 * T + tid] = gch[0].v;
        }
        __syncthreads();
    }
    for (int round = 0; round < rounds; ++round, row += step) {
        RowIn<V, F32> next;
        if (V == 1 && round + 1 < rounds) load_sums(row + step, next);
        auto pin = [&] {
#pragma unroll
            for (int v = 0; v < V; ++v) {
                if (IN_LDS) {
                    wpre[v].v = held[tid];
                    wpost[v].v = held[T + tid];
                    if (GATE == QEFT_GATE_CHANNEL) gch[v].v = held[2 * T + tid];
                } else {
                    wpre[v].pin();
                    if (POST) wpost[v].pin();
                    if (GATE == QEFT_GATE_CHANNEL) gch[v].pin();
                }
                in.dx[v].pin();
                in.h[v].pin();
                in.dh[v].pin();
                in.y[v].pin();
                if (GATE == QEFT_GATE_TOKEN) in.g[v].pin();
            }
        };
        pin();
        float s[3] = {0.f, 0.f, 0.f};   // h^2, a h, y^2
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float h = in.h[v][e];
                s[0] = fmaf(h, h, s[0]);
                s[1] = fmaf(in.dx[v][e] * wpre[v][e], h, s[1]);
                if (POST) s[2] = fmaf(in.y[v][e], in.y[v][e], s[2]);
            }
        if (POST) row_sums(s, buf[2 * (round & 1)], first, waves);
        else {
            float two[2] = {s[0], s[1]};
            row_sums(two, buf[2 * (round & 1)], first, waves);
            s[0] = two[0], s[1] = two[1];
        }
        // (a row beyond the last has no norm: with eps == 0 its hh would be 0 / 0, and dw_pre's sums take it)
        const float rs = row < a.m ? 1.f / sqrtf(fmaf(s[0], inv, a.eps)) : 0.f, c = s[1] * inv * rs;   // c = mean(a hh)
        const float rsy = POST ? 1.f / sqrtf(fmaf(s[2], inv, a.eps)) : 1.f;
        pin();
        float t[V][8], q[1] = {0.f};
#pragma unroll
        for (int v = 0; v < V; ++v) {
            float pre[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float hh = in.h[v][e] * rs, dx = in.dx[v][e];
                t[v][e] = fmaf(rs, fmaf(-hh, c, dx * wpre[v][e]), in.dh[v][e]);
                if (SUMS_IN_LDS) pre[e] = dx * hh;
                else spre[v][e] = fmaf(dx, hh, spre[v][e]);
                if (POST) {
                    const float g = GATE == QEFT_GATE_CHANNEL ? gch[v][e] : GATE == QEFT_GATE_TOKEN ? in.g[v][e] : 1.f;
                    q[0] = fmaf(a.scale * g * t[v][e] * wpost[v][e], in.y[v][e], q[0]);
                }
            }
            if (SUMS_IN_LDS) add_to(0, v, pre);
        }
        if (V == 1 && round + 1 < rounds) load_rest(row + step, next);
        if (POST) row_sums(q, buf[2 * (round & 1) + 1], first, waves);
        pin();
        const float cy = POST ? q[0] * inv * rsy : 0.f;   // mean(a' yh)
        if (row < a.m) {
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const int at = 8 * (tid + T * v), left = a.n - at;
                if (left <= 0) continue;
                float dy[8], dg[8], post[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float g = GATE == QEFT_GATE_CHANNEL ? gch[v][e] : GATE == QEFT_GATE_TOKEN ? in.g[v][e] : 1.f;
                    const float st = a.scale * t[v][e], du = st * g, yh = in.y[v][e] * rsy;
                    dy[e] = POST ? rsy * fmaf(-yh, cy, du * wpost[v][e]) : du;
                    if (POST && SUMS_IN_LDS) post[e] = du * yh;
                    else if (POST) spost[v][e] = fmaf(du, yh, spost[v][e]);
                    const float u = POST ? yh * wpost[v][e] : yh;
                    if (GATE == QEFT_GATE_CHANNEL) sgate[v][e] = fmaf(st, u, sgate[v][e]);
                    if (GATE == QEFT_GATE_TOKEN) dg[e] = st * u;
                    }
                if (POST && SUMS_IN_LDS) add_to(1, v, post);
                if (a.dr) store<F32>(row_of(a.dr, row, a.lddr, F32), at, left, t[v]);
                if (a.dy) store<false>(row_of((void*)a.dy, row, a.lddy, false), at, left, dy);
                if (GATE == QEFT_GATE_TOKEN && a.dgate) store<false>(row_of(a.dgate, row, a.lddg, false), at, left, dg);
            }
        }
        if (round + 1 < rounds) {
            if (V == 1) in = next;
            else {
                load_sums(row + step, in);
                load_rest(row + step, in);
            }
        }
    }
    // this workgroup's slab: its row groups in order
#pragma unroll
    for (int w = 0; w < 3; ++w) {
        if (!S.slab[w]) continue;
        float* out = S.slab[w] + (size_t)blockIdx.x * S.pitch;
        const bool add = S.slabs == 1 && a.accumulate;   // (the slab is the output)
        if (groups == 1) {
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const int at = 8 * (tid + T * v), left = a.n - at;
                float(&x)[8] = w == 0 ? spre[v] : w == 1 ? spost[v] : sgate[v];
                if (SUMS_IN_LDS && w < 2) {
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const f4 s = sums_at[(size_t)((w * V + v) * 2 + h) * blockDim.x];
                        x[4 * h] = s.x, x[4 * h + 1] = s.y, x[4 * h + 2] = s.z, x[4 * h + 3] = s.w;
                    }
                }
                if (add)
                    for (int e = 0; e < 8; ++e) x[e] = e < left ? out[at + e] + x[e] : 0.f;
                if (left > 0) store<true>(out, at, left, x);
            }
            continue;
        }
        __syncthreads();
#pragma unroll
        for (int v = 0; v < V; ++v) {
            float* p = joined + (size_t)group * T * 8 * V + 8 * (tid + T * v);
            const float(&x)[8] = w == 0 ? spre[v] : w == 1 ? spost[v] : sgate[v];
            *reinterpret_cast<f4*>(p) = f4{x[0], x[1], x[2], x[3]};
            *reinterpret_cast<f4*>(p + 4) = f4{x[4], x[5], x[6], x[7]};
        }
        __syncthreads();
        for (int col = threadIdx.x; col < a.n; col += blockDim.x) {
            float x = joined[col];
            for (int g = 1; g < groups; ++g) x += joined[(size_t)g * T * 8 * V + col];
            out[col] = add ? out[col] + x : x;
        }
    }
}

// out[col] = the sum of the slabs, in their order within 16 interleaved shares, then the shares in order
__global__ __launch_bounds__(256) void norm_slabs_kernel(Sums S, float* o0, float* o1, float* o2, int n, int accumulate) {
    __shared__ __align__(16) float red[16][64];
    const int which = blockIdx.y;
    const float* slab = S.slab[which];
    float* out = which == 0 ? o0 : which == 1 ? o1 : o2;
    if (!slab) return;
    const int quad = threadIdx.x & 15, share = threadIdx.x >> 4, col = 64 * blockIdx.x + 4 * quad;
    f4 s = {0.f, 0.f, 0.f, 0.f};
    if (col < n)   // (a slab's pitch is a multiple of 8)
        for (int i0 = share; i0 < S.slabs; i0 += 16 * 8) {
            f4 x[8];   // eight loads before the first sum
#pragma unroll
            for (int y = 0; y < 8; ++y) {
                const int i = i0 + 16 * y;
                x[y] = i < S.slabs ? *reinterpret_cast<const f4*>(slab + (size_t)i * S.pitch + col) : f4{0.f, 0.f, 0.f, 0.f};
            }
#pragma unroll
            for (int y = 0; y < 8; ++y) s += x[y];
        }
    *reinterpret_cast<f4*>(&red[share][4 * quad]) = s;
    __syncthreads();
    if (threadIdx.x < 64) {
        const int x = 64 * blockIdx.x + threadIdx.x;
        float v = red[0][threadIdx.x];
#pragma unroll
        for (int i = 1; i < 16; ++i) v += red[i][threadIdx.x];
        if (x < n) out[x] = accumulate ? out[x] + v : v;
    }
}

// Rows beyond BWD_MAX: their statistics first (all of them sums over one reading: mean(a' yh) is linear in t's three terms) ...
struct RowStat {
    float rs, c, rsy, cy;
};
template <bool F32>
__global__ __launch_bounds__(1024) void norm_bwd_stats_kernel(Norm a, RowStat* out) {
    __shared__ float buf[6][16];
    const int64_t row = blockIdx.x;
    const float inv = 1.f / (float)a.n;
    float s[6] = {};   // h^2, a h, y^2; with k = scale gate w_post: k y dh, k y a, k y h
    for (int at = 8 * threadIdx.x; at < a.n; at += 8192) {
        const int left = min(8, a.n - at);
        Raw<F32> h, dh;
        Half8 dx, w;
        h.load(row_of(a.r, row, a.ldr, F32), at, left);
        dx.load(a.dx + row * a.lddx, at, left);
        w.load(a.w_pre, at, left);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            s[0] = fmaf(h[e], h[e], s[0]);
            s[1] = fmaf(dx[e] * w[e], h[e], s[1]);
        }
        if (!a.w_post) continue;
        Half8 y, wp, g;
        dh.clear();
        if (a.dh) dh.load(row_of(a.dh, row, a.lddh, F32), at, left);
        y.load(a.y + row * a.ldy, at, left);
        wp.load(a.w_post, at, left);
        if (a.gate_kind != QEFT_GATE_NONE) g.load(a.gate + (a.gate_kind == QEFT_GATE_TOKEN ? row * a.ldg : 0), at, left);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float k = a.scale * (a.gate_kind != QEFT_GATE_NONE ? g[e] : 1.f) * wp[e] * y[e];
            s[2] = fmaf(y[e], y[e], s[2]);
            s[3] = fmaf(k, dh[e], s[3]);
            s[4] = fmaf(k, dx[e] * w[e], s[4]);
            s[5] = fmaf(k, h[e], s[5]);
        }
    }
    row_sums(s, buf, 0, 16);
    if (threadIdx.x == 0) {
        RowStat r;
        r.rs = 1.f / sqrtf(fmaf(s[0], inv, a.eps));
        r.c = s[1] * inv * r.rs;
        r.rsy = a.w_post ? 1.f / sqrtf(fmaf(s[2], inv, a.eps)) : 1.f;
        r.cy = (s[3] + r.rs * (s[4] - r.rs * r.c * s[5])) * inv * r.rsy;
        out[row] = r;
    }
}
// ... then gradients and column sums: a workgroup has 2048 columns and the rows blockIdx.y, blockIdx.y + slabs, ...
template <bool F32>
__global__ __launch_bounds__(256) void norm_bwd_long_kernel(Norm a, Sums S, const RowStat* stats) {
    const int at = 2048 * blockIdx.x + 8 * threadIdx.x;
    if (at >= a.n) return;
    const int left = min(8, a.n - at);
    Half8 w, wp, gc;
    w.load(a.w_pre, at, left);
    if (a.w_post) wp.load(a.w_post, at, left);
    if (a.gate_kind == QEFT_GATE_CHANNEL) gc.load(a.gate, at, left);
    float sums[3][8] = {};
    for (int64_t row = blockIdx.y; row < a.m; row += gridDim.y) {
        const RowStat r = stats[row];
        Raw<F32> h, dh;
        Half8 dx, y, g = gc;
        dh.clear();
        y.clear();
        h.load(row_of(a.r, row, a.ldr, F32), at, left);
        dx.load(a.dx + row * a.lddx, at, left);
        if (a.dh) dh.load(row_of(a.dh, row, a.lddh, F32), at, left);
        if (a.y) y.load(a.y + row * a.ldy, at, left);
        if (a.gate_kind == QEFT_GATE_TOKEN) g.load(a.gate + row * a.ldg, at, left);
        float t[8], dy[8], dg[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float hh = h[e] * r.rs;
            t[e] = fmaf(r.rs, fmaf(-hh, r.c, dx[e] * w[e]), dh[e]);
            sums[0][e] = fmaf(dx[e], hh, sums[0][e]);
            const float st = a.scale * t[e], du = a.gate_kind != QEFT_GATE_NONE ? st * g[e] : st, yh = y[e] * r.rsy;
            dy[e] = a.w_post ? r.rsy * fmaf(-yh, r.cy, du * wp[e]) : du;
            const float u = a.w_post ? yh * wp[e] : yh;
            dg[e] = st * u;
            sums[1][e] = fmaf(du, yh, sums[1][e]);
            sums[2][e] = fmaf(st, u, sums[2][e]);
        }
        if (a.dr) store<F32>(row_of(a.dr, row, a.lddr, F32), at, left, t);
        if (a.dy) store<false>(row_of((void*)a.dy, row, a.lddy, false), at, left, dy);
        if (a.gate_kind == QEFT_GATE_TOKEN && a.dgate) store<false>(row_of(a.dgate, row, a.lddg, false), at, left, dg);
    }
#pragma unroll
    for (int x = 0; x < 3; ++x)
        if (S.slab[x])
            for (int e = 0; e < 8; ++e)
                if (e < left) S.slab[x][(size_t)blockIdx.y * S.pitch + at + e] = sums[x][e];
}

// How the gradient divides its rows.
struct BwdPlan {
    int waves, groups, v, grid, rounds;
    bool in_registers;
    size_t at_slabs, slab_bytes;   // one of the three sums' slabs
    int64_t pitch;
};
BwdPlan bwd_plan(int n, int64_t m) {
    BwdPlan p{};
    const int octets = (n + 7) / 8;
    p.pitch = 8 * (int64_t)octets;
    p.in_registers = n <= BWD_MAX;
    if (p.in_registers) {
        p.v = n <= 8192 ? 1 : 2;
        p.waves = (octets + 64 * p.v - 1) / (64 * p.v);
        // Rows side by side in a workgroup: all that fit where one workgroup then takes the whole call (13 x 488: 5.6 us against 8.8), else no more than fill the CUs (200 x 4096:
        // 10.5 us with one, 11.2 with two; 101 x 3856 with both norms and a token gate 9.6 and 11.4).
        const int most = 16 / p.waves;
        p.groups = m <= most ? most : (int)std::min<int64_t>(most, (m + 255) / 256);
        // One workgroup of up to 1024 threads per CU: a slab costs 24 bytes a column however many rows it sums.
        const int64_t teams = (m + p.groups - 1) / p.groups;
        p.rounds = (int)((teams + 255) / 256);
        p.grid = (int)((teams + p.rounds - 1) / (p.rounds > 0 ? p.rounds : 1));
    } else {
        p.grid = (int)(m < 64 ? m : 64);   // slabs
        p.at_slabs = ((size_t)m * sizeof(RowStat) + 255) / 256 * 256;
    }
    p.slab_bytes = (size_t)p.grid * p.pitch * sizeof(float);
    return p;
}

template <int V, bool F32, bool POST, int GATE>
hipError_t launch_gate(const Norm& a, const Sums& S, const BwdPlan& p, int threads, size_t lds, hipStream_t s) {
    const hipError_t e = allow_lds((const void*)norm_bwd_kernel<V, F32, POST, GATE>, lds, 128 * 1024);
    if (e == hipSuccess) norm_bwd_kernel<V, F32, POST, GATE><<<p.grid, threads, lds, s>>>(a, S, p.waves, p.groups, p.rounds);
    return e;
}
template <int V, bool F32, bool POST>
hipError_t launch_bwd(const Norm& a, const Sums& S, const BwdPlan& p, hipStream_t s) {
    const int threads = 64 * p.waves * p.groups;
    const size_t lds = V > 1 ? (size_t)threads * (POST ? 2 : 1) * 8 * V * sizeof(float)
                             : (p.groups > 1 ? (size_t)threads * 8 * sizeof(float) : 0) + (POST ? 3 * 64 * (size_t)p.waves * sizeof(u4) : 0);
    if (a.gate_kind == QEFT_GATE_CHANNEL) return launch_gate<V, F32, POST, QEFT_GATE_CHANNEL>(a, S, p, threads, lds, s);
    if (a.gate_kind == QEFT_GATE_TOKEN) return launch_gate<V, F32, POST, QEFT_GATE_TOKEN>(a, S, p, threads, lds, s);
    return launch_gate<V, F32, POST, QEFT_GATE_NONE>(a, S, p, threads, lds, s);
}
template <int V>
hipError_t launch_bwd_of(const Norm& a, const Sums& S, const BwdPlan& p, hipStream_t s) {
    if (a.f32) return a.w_post ? launch_bwd<V, true, true>(a, S, p, s) : launch_bwd<V, true, false>(a, S, p, s);
    return a.w_post ? launch_bwd<V, false, true>(a, S, p, s) : launch_bwd<V, false, false>(a, S, p, s);
}

template <int V>
void launch_fwd(const Norm& a, hipStream_t s) {
    const int octets = (a.n + 7) / 8, waves = (octets + 64 * V - 1) / (64 * V), rows = waves == 1 ? 4 : 1;
    const unsigned grid = (unsigned)((a.m + rows - 1) / rows);
    if (a.f32) norm_fwd_kernel<V, true><<<grid, 64 * waves * rows, 0, s>>>(a, waves);
    else norm_fwd_kernel<V, false><<<grid, 64 * waves * rows, 0, s>>>(a, waves);
}

__global__ __launch_bounds__(256) void zero_kernel(float* a, float* b, float* c, int n) {
    const int i = blockIdx.x * 256 + threadIdx.x;
    if (i >= n) return;
    if (a) a[i] = 0.f;
    if (b) b[i] = 0.f;
    if (c) c[i] = 0.f;
}

}  // namespace

hipError_t norm_fwd(const Norm& a, hipStream_t s) {
    if (a.n <= 8192) launch_fwd<1>(a, s);
    else if (a.n <= 16384) launch_fwd<2>(a, s);
    else if (a.n <= FWD_MAX) launch_fwd<4>(a, s);
    else if (a.f32) norm_fwd_long_kernel<true><<<(unsigned)a.m, 1024, 0, s>>>(a);
    else norm_fwd_long_kernel<false><<<(unsigned)a.m, 1024, 0, s>>>(a);
    return hipGetLastError();
}

size_t norm_workspace(int n, int64_t m) {
    if (m <= 0) return 0;
    const BwdPlan p = bwd_plan(n, m);
    return p.at_slabs + 3 * p.slab_bytes;
}
size_t norm_bwd_workspace(int n, int64_t m, bool sums) { return sums || n > BWD_MAX ? norm_workspace(n, m) : 0; }   // (rows too long for registers leave their statistics there)

hipError_t norm_bwd(const Norm& a, hipStream_t s) {
    float* gate = a.gate_kind == QEFT_GATE_CHANNEL ? (float*)a.dgate : nullptr;
    if (a.m == 0) {
        if (!a.accumulate && (a.dw_pre || a.dw_post || gate)) zero_kernel<<<(a.n + 255) / 256, 256, 0, s>>>(a.dw_pre, a.dw_post, gate, a.n);
        return hipGetLastError();
    }
    const BwdPlan p = bwd_plan(a.n, a.m);
    Sums S{};
    S.pitch = p.pitch;
    S.slabs = p.grid;
    float* outs[3] = {a.dw_pre, a.dw_post, gate};
    const bool one = p.in_registers && p.grid == 1;   // its slab is the output
    for (int i = 0; i < 3; ++i)
        if (outs[i]) S.slab[i] = one ? outs[i] : (float*)(a.ws + p.at_slabs + i * p.slab_bytes);
    if (p.in_registers) {
        const hipError_t e = p.v == 1 ? launch_bwd_of<1>(a, S, p, s) : launch_bwd_of<2>(a, S, p, s);
        if (e != hipSuccess) return e;
    } else {
        RowStat* stats = (RowStat*)a.ws;
        const dim3 grid((a.n + 2047) / 2048, p.grid);
        if (a.f32) {
            norm_bwd_stats_kernel<true><<<(unsigned)a.m, 1024, 0, s>>>(a, stats);
            norm_bwd_long_kernel<true><<<grid, 256, 0, s>>>(a, S, stats);
        } else {
            norm_bwd_stats_kernel<false><<<(unsigned)a.m, 1024, 0, s>>>(a, stats);
            norm_bwd_long_kernel<false><<<grid, 256, 0, s>>>(a, S, stats);
        }
    }
    if (!one && (outs[0] || outs[1] || outs[2]))
        norm_slabs_kernel<<<dim3((a.n + 63) / 64, 3), 256, 0, s>>>(S, outs[0], outs[1], outs[2], a.n, a.accumulate);
    return hipGetLastError();
}

}  // namespace qeft
