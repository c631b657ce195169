// Norms of the heads of queries and keys with their rotation by position, the gradients, and the same for tokens that enter a cache (qeft_qk_norm_fwd,
// qeft_qk_norm_bwd, qeft_cache_append_norm).
//
//   y = x rs w, rs = 1 / sqrt(mean x^2 + eps)     z = R y:  (a, b) -> (a c - b s, b c + a s),  a = y[j], b = y[j + half], half = rot_dim / 2
//   g = R^T gz     dx = rs (a - xh mean(a xh)),  a = g w, xh = x rs     dw = sum g xh
//
// Bytes bound all three (4096 tokens of 40 + 40 heads of 128 39 us, 4.4 TB/s, or 33 where the caches hold some of it; the gradient of 4001 tokens of 64 + 8 heads 48, 4.6 TB/s;
// 8 tokens of 32 + 32 heads into a cache 4.8, of which 3.8 a launch that does nothing).  A head is L lanes', each with two pieces of VW values half apart, so that pairs meet in a lane and the head's sums stay within a row of lanes
// (no LDS); a wave has 64 / L heads side by side.  Heads of all tokens form one sequence that the grid walks through: no lane waits for a token's last heads.  The
// gradient's workgroups keep their sums for dw in registers and leave one slab each, summed by a second launch in a fixed order.
#include "pieces.h"
#include "qeft_internal.h"
#include "wave.h"

namespace qeft {
namespace {

constexpr int THREADS = 256;
// Workgroups at most.  Forward: as many as run at a time, five a CU (4096 tokens of 40 + 40 heads 38.8 us; 2048 41.7, 10240 - one head a lane - 38.3, but 4096 tokens of 32 + 1 heads
// of 40, 20 of them turned, 13.9 -> 16.0; 768 33.3 in place of 33.0 where the caches hold some, 16.2 / 13.9).  The append's grid is the same (41.9, by 768 44.6).  Gradient: two a CU, each leaves a slab (4001 tokens of 64 + 8 heads with 256 / 512 / 768 / 1024 / 2048: 55 / 45 / 47 / 49 / 59 us).
constexpr int FWD_GROUPS = 1280, BWD_GROUPS = 512;

// Lane's r-th two pieces of a head: the rotated ones, half apart, then what is behind them two by two
template <int VW>
struct Place {
    int first, second;      // values
    bool turned, one, two;  // two pieces that are a pair; there is a first, a second one
};
template <int VW>
__device__ __forceinline__ Place<VW> place_of(int p, int d, int half) {
    const int pairs = half / VW, whole = d / VW;
    if (p < pairs) return Place<VW>{VW * p, half + VW * p, true, true, true};
    const int at = 2 * pairs + 2 * (p - pairs);
    return Place<VW>{VW * at, VW * (at + 1), false, at < whole, at + 1 < whole};
}
template <int VW>
struct Two {
    _Float16 a[VW], b[VW];
    __device__ __forceinline__ void load(const __half* head, const Place<VW>& p) {
        if (p.two) {
            get<VW>(head + p.first, a);
            get<VW>(head + p.second, b);
        } else {
#pragma unroll
            for (int e = 0; e < VW; ++e) a[e] = b[e] = 0;
            if (p.one) get<VW>(head + p.first, a);
        }
    }
    __device__ __forceinline__ void store(__half* head, const Place<VW>& p) const {
        if (p.one) put<VW>(head + p.first, a);
        if (p.two) put<VW>(head + p.second, b);
    }
    // one of two, word by word (a choice between the objects goes through memory)
    static __device__ __forceinline__ Two choose(bool first, const Two& x, const Two& y) {
        uint32_t u[VW], v[VW];
        __builtin_memcpy(u, &x, sizeof u);
        __builtin_memcpy(v, &y, sizeof v);
#pragma unroll
        for (int i = 0; i < VW; ++i) u[i] = first ? u[i] : v[i];
        Two o;
        __builtin_memcpy(&o, u, sizeof u);
        return o;
    }
};
template <int N, int CTRL>
__device__ __forceinline__ float moved(float x) { return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CTRL, 0xf, 0xf, false)); }
// Sum over L neighbouring lanes, the same in each of them
template <int L>
__device__ __forceinline__ float head_sum(float x) {
    if (L >= 2) x += moved<1, 0xb1>(x);       // quad_perm 1 0 3 2
    if (L >= 4) x += moved<2, 0x4e>(x);       // quad_perm 2 3 0 1
    if (L >= 8) x += moved<4, 0x141>(x);      // row_half_mirror
    if (L >= 16) x += moved<8, 0x140>(x);     // row_mirror
    if (L >= 32) x = across<false>(x, Sum());
    if (L >= 64) x = across<true>(x, Sum());
    return x;
}
// Sum over the heads side by side in a wave: lanes L apart
template <int L>
__device__ __forceinline__ float side_sum(float x) {
    if (L <= 4) x += row_rotated<4>(x);
    if (L <= 8) x += row_rotated<8>(x);
    if (L <= 16) x = across<false>(x, Sum());
    if (L <= 32) x = across<true>(x, Sum());
    return x;
}

// Where the grid's walk over `heads` heads of every token begins for this lane, and its step
struct Walk {
    int t, h, dt, dh, heads;
    __device__ __forceinline__ Walk(int slot, int slots, int heads_) : heads(heads_) {
        t = (int)((uint32_t)slot / (uint32_t)heads);
        h = slot - t * heads;
        dt = (int)((uint32_t)slots / (uint32_t)heads);
        dh = slots - dt * heads;
    }
    __device__ __forceinline__ void next() {
        t += dt;
        h += dh;
        if (h >= heads) h -= heads, ++t;
    }
};

// cosines and sines of a lane's pairs
template <int VW>
struct Turn {
    float c[VW], s[VW];
    __device__ __forceinline__ void load(const float* rot, int64_t ld, int positions, int pos, int first, int half) {
        const float* r = rot + (size_t)min(max(pos, 0), positions - 1) * ld + first;
#pragma unroll
        for (int e = 0; e < VW; ++e) {
            c[e] = r[e];
            s[e] = r[half + e];
        }
    }
};

// A head's values (x, and the weights w where it is normed) into what goes out
template <int VW, int R, int L>
__device__ __forceinline__ void forward(Two<VW> (&x)[R], const Two<VW> (&w)[R], bool normed, const Place<VW> (&place)[R], const Turn<VW> (&turn)[R], int d, float eps) {
    float rs = 1.f;
    if (normed) {
        float ss = 0.f;
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int e = 0; e < VW; ++e) {
                const float a = x[r].a[e], b = x[r].b[e];
                ss = fmaf(a, a, ss);
                ss = fmaf(b, b, ss);
            }
        rs = 1.f / sqrtf(head_sum<L>(ss) / (float)d + eps);
    }
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int e = 0; e < VW; ++e) {
            float a = x[r].a[e], b = x[r].b[e];
            if (normed) {
                a = a * rs * (float)w[r].a[e];
                b = b * rs * (float)w[r].b[e];
            }
            x[r].a[e] = (_Float16)(place[r].turned ? a * turn[r].c[e] - b * turn[r].s[e] : a);
            x[r].b[e] = (_Float16)(place[r].turned ? b * turn[r].c[e] + a * turn[r].s[e] : b);
        }
}

template <int VW, int R, int L>
struct Lane {
    Place<VW> place[R];
    Two<VW> wq[R], wk[R];
    __device__ __forceinline__ Lane(int d, int half, const __half* w_q, const __half* w_k) {
#pragma unroll
        for (int r = 0; r < R; ++r) {
            place[r] = place_of<VW>((int)(threadIdx.x % L) + L * r, d, half);
            if (w_q) wq[r].load(w_q, place[r]);
            if (w_k) wk[r].load(w_k, place[r]);
        }
    }
};

template <int VW, int R, int L>
__global__ __launch_bounds__(THREADS) void heads_fwd_kernel(Heads a) {
    const int half = a.rot_dim / 2, hq = a.q.heads;
    const Lane<VW, R, L> lane(a.d, half, a.q.w, a.k.w);
    Walk at((blockIdx.x * THREADS + threadIdx.x) / L, gridDim.x * (THREADS / L), hq + a.k.heads);
    Two<VW> x[R], ahead[R];
    int pos = 0, pos_ahead = 0;
    auto fetch = [&](Two<VW>(&to)[R], int& p) {
        if (at.t >= a.m) return;
        const bool is_q = at.h < hq;
        const __half* head = (is_q ? a.q.x + at.t * a.q.ldx : a.k.x + at.t * a.k.ldx) + (size_t)(is_q ? at.h : at.h - hq) * a.d;
#pragma unroll
        for (int r = 0; r < R; ++r) to[r].load(head, lane.place[r]);
        p = a.pos && half ? a.pos[at.t] : at.t;
    };
    fetch(ahead, pos_ahead);
    while (at.t < a.m) {
        const int t = at.t, h = at.h;
        pos = pos_ahead;
#pragma unroll
        for (int r = 0; r < R; ++r) x[r] = ahead[r];
        Turn<VW> turn[R];
#pragma unroll
        for (int r = 0; r < R; ++r)
            if (lane.place[r].turned) turn[r].load(a.rot, a.ld_rot, a.positions, pos, lane.place[r].first, half);
        at.next();
        fetch(ahead, pos_ahead);
        const bool is_q = h < hq;
        Two<VW> w[R];
#pragma unroll
        for (int r = 0; r < R; ++r) w[r] = Two<VW>::choose(is_q, lane.wq[r], lane.wk[r]);
        forward<VW, R, L>(x, w, is_q ? a.q.w != nullptr : a.k.w != nullptr, lane.place, turn, a.d, a.eps);
        __half* out = (is_q ? a.q.out + t * a.q.ldout : a.k.out + t * a.k.ldout) + (size_t)(is_q ? h : h - hq) * a.d;
#pragma unroll
        for (int r = 0; r < R; ++r) x[r].store(out, lane.place[r]);
    }
}

// The heads of q, k and v of tokens that enter a cache; as qeft_cache_append otherwise.
template <int VW, int R, int L>
__global__ __launch_bounds__(THREADS) void heads_append_kernel(Cache c, Append a, const __half* w_q, const __half* w_k, float eps) {
    const int half = a.rot_dim / 2, hq = a.q ? a.heads : 0;
    const Lane<VW, R, L> lane(c.d, half, w_q, w_k);
    const int64_t last = (int64_t)c.table_pages * c.page_size;
    for (Walk at((blockIdx.x * THREADS + threadIdx.x) / L, gridDim.x * (THREADS / L), hq + 2 * c.kv); at.t < a.tokens; at.next()) {
        const int t = at.t;
        const bool is_q = at.h < hq, is_v = at.h >= hq + c.kv;
        const int h = is_q ? at.h : is_v ? at.h - hq - c.kv : at.h - hq;
        const __half* head = (is_q ? a.q + t * a.ldq : is_v ? a.v + t * a.ldv : a.k + t * a.ldk) + (size_t)h * c.d;
        Two<VW> x[R];
#pragma unroll
        for (int r = 0; r < R; ++r) x[r].load(head, lane.place[r]);
        const int index = a.index[t], b = a.seq ? a.seq[t] : t;
        __half* out = is_q ? a.q_out + t * a.ldq_out + (size_t)h * c.d : nullptr;
        if (!is_q && b >= 0 && b < c.seqs && index >= 0 && index < last) {
            const int p = c.by_page.of(index);
            const int page = c.table[(size_t)b * c.ld_table + p];
            if (page >= 0 && page < c.pages)
                out = (is_v ? c.v : c.k) + (size_t)page * c.page_stride + (size_t)(index - p * c.page_size) * c.token_stride + (size_t)h * c.head_stride;
        }
        if (!is_v) {
            Turn<VW> turn[R];
            Two<VW> w[R];
#pragma unroll
            for (int r = 0; r < R; ++r) {
                if (lane.place[r].turned) turn[r].load(a.rot, a.ld_rot, a.positions, a.pos ? a.pos[t] : index, lane.place[r].first, half);
                w[r] = Two<VW>::choose(is_q, lane.wq[r], lane.wk[r]);
            }
            forward<VW, R, L>(x, w, is_q ? w_q != nullptr : w_k != nullptr, lane.place, turn, c.d, eps);
        }
        if (!out) continue;   // (a token without a slot)
#pragma unroll
        for (int r = 0; r < R; ++r) x[r].store(out, lane.place[r]);
    }
}

// Gradient: first the heads of q, then those of k.  slab [workgroup][q, k][d], or NULL
template <int VW, int R, int L>
__global__ __launch_bounds__(THREADS) void heads_bwd_kernel(Heads a, float* slab) {
    __shared__ float joined[THREADS / 64][QEFT_MAX_HEAD_DIM];
    const int half = a.rot_dim / 2, wave = threadIdx.x >> 6;
#pragma unroll 1
    for (int which = 0; which < 2; ++which) {
        const HeadPart& p = which ? a.k : a.q;
        float sa[R][VW] = {}, sb[R][VW] = {};
        const Lane<VW, R, L> lane(a.d, half, p.w, nullptr);
        const bool normed = p.w != nullptr;
        if (p.heads > 0 && (p.dx || p.dw)) {
            Walk at((blockIdx.x * THREADS + threadIdx.x) / L, gridDim.x * (THREADS / L), p.heads);
            Two<VW> g[R], x[R], g_ahead[R], x_ahead[R];
            int pos = 0, pos_ahead = 0;
            auto fetch = [&] {
                if (at.t >= a.m) return;
                const __half* gh = p.g + at.t * p.ldg + (size_t)at.h * a.d;
                const __half* xh = p.x + at.t * p.ldx + (size_t)at.h * a.d;
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    g_ahead[r].load(gh, lane.place[r]);
                    if (normed) x_ahead[r].load(xh, lane.place[r]);
                }
                pos_ahead = a.pos && half ? a.pos[at.t] : at.t;
            };
            fetch();
            while (at.t < a.m) {
                const int t = at.t, h = at.h;
                pos = pos_ahead;
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    g[r] = g_ahead[r];
                    x[r] = x_ahead[r];
                }
                Turn<VW> turn[R];
#pragma unroll
                for (int r = 0; r < R; ++r)
                    if (lane.place[r].turned) turn[r].load(a.rot, a.ld_rot, a.positions, pos, lane.place[r].first, half);
                at.next();
                fetch();
                float ga[R][VW], gb[R][VW], ss = 0.f, dot = 0.f;
#pragma unroll
                for (int r = 0; r < R; ++r)
#pragma unroll
                    for (int e = 0; e < VW; ++e) {
                        const float u = g[r].a[e], v = g[r].b[e];
                        ga[r][e] = lane.place[r].turned ? u * turn[r].c[e] + v * turn[r].s[e] : u;
                        gb[r][e] = lane.place[r].turned ? v * turn[r].c[e] - u * turn[r].s[e] : v;
                    }
                if (normed) {
#pragma unroll
                    for (int r = 0; r < R; ++r)
#pragma unroll
                        for (int e = 0; e < VW; ++e) {
                            const float xa = x[r].a[e], xb = x[r].b[e];
                            ss = fmaf(xa, xa, ss);
                            ss = fmaf(xb, xb, ss);
                            dot = fmaf(ga[r][e] * (float)lane.wq[r].a[e], xa, dot);
                            dot = fmaf(gb[r][e] * (float)lane.wq[r].b[e], xb, dot);
                        }
                    const float rs = 1.f / sqrtf(head_sum<L>(ss) / (float)a.d + a.eps), mean = head_sum<L>(dot) * rs / (float)a.d;
#pragma unroll
                    for (int r = 0; r < R; ++r)
#pragma unroll
                        for (int e = 0; e < VW; ++e) {
                            const float ha = x[r].a[e] * rs, hb = x[r].b[e] * rs;
                            sa[r][e] = fmaf(ga[r][e], ha, sa[r][e]);
                            sb[r][e] = fmaf(gb[r][e], hb, sb[r][e]);
                            ga[r][e] = rs * (ga[r][e] * (float)lane.wq[r].a[e] - ha * mean);
                            gb[r][e] = rs * (gb[r][e] * (float)lane.wq[r].b[e] - hb * mean);
                        }
                }
                if (!p.dx) continue;
                __half* out = p.dx + t * p.lddx + (size_t)h * a.d;
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    Two<VW> o;
#pragma unroll
                    for (int e = 0; e < VW; ++e) {
                        o.a[e] = (_Float16)ga[r][e];
                        o.b[e] = (_Float16)gb[r][e];
                    }
                    o.store(out, lane.place[r]);
                }
            }
        }
        if (!slab) continue;
        // the heads side by side, then the waves
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int e = 0; e < VW; ++e) {
                const float x = side_sum<L>(sa[r][e]), y = side_sum<L>(sb[r][e]);
                if ((threadIdx.x & 63) < L) {
                    if (lane.place[r].one) joined[wave][lane.place[r].first + e] = x;
                    if (lane.place[r].two) joined[wave][lane.place[r].second + e] = y;
                }
            }
        __syncthreads();
        for (int j = threadIdx.x; j < a.d; j += THREADS)
            slab[((size_t)blockIdx.x * 2 + which) * a.d + j] = ((joined[0][j] + joined[1][j]) + joined[2][j]) + joined[3][j];
        __syncthreads();
    }
}

// dw: the slabs' sum in a fixed order, 32 columns a workgroup, 32 threads a column: few loads one after the other
constexpr int SHARES = 32;
__global__ __launch_bounds__(32 * SHARES) void heads_sum_kernel(Heads a, const float* slab, int slabs) {
    __shared__ float joined[SHARES][33];
    const int column = threadIdx.x & 31, share = threadIdx.x >> 5, j = blockIdx.x * 32 + column;
    float s = 0.f;
    if (j < 2 * a.d) {
#pragma unroll 8
        for (int i = share; i < slabs; i += SHARES) s += slab[(size_t)i * 2 * a.d + j];
    }
    joined[share][column] = s;
    __syncthreads();
    if (share != 0 || j >= 2 * a.d) return;
    float* out = j < a.d ? a.q.dw : a.k.dw;
    if (!out) return;
#pragma unroll
    for (int i = 1; i < SHARES; ++i) s += joined[i][column];
    float* at = out + (j < a.d ? j : j - a.d);
    *at = a.accumulate ? *at + s : s;
}

// The widest pieces that both halves of a pair consist of, and the lanes of a head: f.template operator()<VW, R, L>().  Pieces of 16 bytes against 8: 4096 tokens of 40 + 40 heads 33 -> 41 us,
// gradient 49 -> 64.
struct Form {
    int vw, lanes;
};
Form form_of(int d, int rot_dim) {
    const int half = rot_dim / 2, vw = half % 8 == 0 ? 8 : half % 4 == 0 ? 4 : half % 2 == 0 ? 2 : 1;
    const int pairs = half / vw, pieces = pairs + (d / vw - 2 * pairs + 1) / 2;
    if (vw == 8) return Form{8, pieces <= 4 ? 4 : pieces <= 8 ? 8 : 16};
    if (vw == 4) return Form{4, pieces <= 8 ? 8 : pieces <= 16 ? 16 : 32};
    if (vw == 2) return Form{2, pieces <= 16 ? 16 : 64};
    return Form{1, 64};
}
template <class F>
void with_form(const Form& f, const F& go) {
    if (f.vw == 8) {
        if (f.lanes == 4) go.template operator()<8, 1, 4>();
        else if (f.lanes == 8) go.template operator()<8, 1, 8>();
        else go.template operator()<8, 1, 16>();
    } else if (f.vw == 4) {
        if (f.lanes == 8) go.template operator()<4, 1, 8>();
        else if (f.lanes == 16) go.template operator()<4, 1, 16>();
        else go.template operator()<4, 1, 32>();
    } else if (f.vw == 2) {
        if (f.lanes == 16) go.template operator()<2, 1, 16>();
        else go.template operator()<2, 1, 64>();
    } else go.template operator()<1, 2, 64>();
}
// workgroups for so many heads of so many lanes
int groups_for(int64_t heads, int lanes, int most) {
    const int64_t n = (heads * lanes + THREADS - 1) / THREADS;
    return (int)(n < most ? n : most);
}
struct Fwd {
    const Heads& a;
    unsigned grid;
    hipStream_t s;
    template <int VW, int R, int L>
    void operator()() const { heads_fwd_kernel<VW, R, L><<<grid, THREADS, 0, s>>>(a); }
};
struct App {
    const Cache& c;
    const Append& a;
    const __half *w_q, *w_k;
    float eps;
    unsigned grid;
    hipStream_t s;
    template <int VW, int R, int L>
    void operator()() const { heads_append_kernel<VW, R, L><<<grid, THREADS, 0, s>>>(c, a, w_q, w_k, eps); }
};
struct Bwd {
    const Heads& a;
    float* slab;
    unsigned grid;
    hipStream_t s;
    template <int VW, int R, int L>
    void operator()() const { heads_bwd_kernel<VW, R, L><<<grid, THREADS, 0, s>>>(a, slab); }
};
int bwd_groups(int d, int heads, int kv, int rot_dim, int64_t m) { return groups_for(m * (heads > kv ? heads : kv), form_of(d, rot_dim).lanes, BWD_GROUPS); }

}  // namespace

size_t heads_workspace(int d, int heads, int kv, int rot_dim, int64_t m) { return (size_t)bwd_groups(d, heads, kv, rot_dim, m) * 2 * d * sizeof(float); }

hipError_t heads_fwd(const Heads& a, hipStream_t s) {
    const Form f = form_of(a.d, a.rot_dim);
    with_form(f, Fwd{a, (unsigned)groups_for(a.m * (a.q.heads + a.k.heads), f.lanes, FWD_GROUPS), s});
    return hipGetLastError();
}
hipError_t heads_append(const Cache& c, const Append& p, const __half* w_q, const __half* w_k, float eps, hipStream_t s) {
    const Form f = form_of(c.d, p.rot_dim);
    with_form(f, App{c, p, w_q, w_k, eps, (unsigned)groups_for((int64_t)p.tokens * (p.heads + 2 * (int64_t)c.kv), f.lanes, FWD_GROUPS), s});
    return hipGetLastError();
}
hipError_t heads_bwd(const Heads& a, hipStream_t s) {
    const bool sums = a.q.dw || a.k.dw;
    float* slab = sums ? (float*)a.ws : nullptr;
    const int slabs = a.m > 0 ? bwd_groups(a.d, a.q.heads, a.k.heads, a.rot_dim, a.m) : 0;
    if (slabs > 0) with_form(form_of(a.d, a.rot_dim), Bwd{a, slab, (unsigned)slabs, s});
    if (sums) heads_sum_kernel<<<(unsigned)(2 * a.d + 31) / 32, 32 * SHARES, 0, s>>>(a, slab, slabs);
    return hipGetLastError();
}

}  // namespace qeft
