// New tokens into a paged cache (qeft_cache_append): queries and keys rotated by their positions, keys and values stored in their slots.
//
//   (x[j], x[j + half]) -> (x[j] c - x[j + half] s, x[j + half] c + x[j] s),   half = rot_dim / 2, c and s of the token's position and j
//
// Nothing but bytes: every value is read and written once, so a thread takes whole pieces of VW values of both halves and keeps the cosines and sines of its
// piece, fp32 and as many bytes as the pieces themselves, for all heads of the token: a workgroup takes one token and runs over its heads.  4001 tokens, 64 / 8 heads of 128: 34.5 us, 4.8 TB/s.
#include "pieces.h"
#include "qeft_internal.h"

namespace qeft {
namespace {

// Workgroup = token x one of `parts` shares of its heads.  Threads: `pieces` of a head x as many heads side by side as fit.  The pieces of a head: rot_dim / 2 / VW
// pairs (half apart), then what is not rotated, d - rot_dim, in pieces of VW.  Heads: those of q, then k's, then v's (whose d is all "not rotated").
template <int VW>
__global__ __launch_bounds__(256) void append_kernel(Cache c, Append a, int parts, int pieces, int side) {
    const int t = blockIdx.x / parts, part = blockIdx.x % parts;
    const int piece = threadIdx.x % pieces, first = threadIdx.x / pieces;
    if (first >= side) return;
    const int half = a.rot_dim / 2, pairs = half / VW, whole = c.d / VW;

    const int index = a.index[t], b = a.seq ? a.seq[t] : t;
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
    float cs[VW] = {}, sn[VW] = {};
    if (piece < pairs) {
        const int pos = min(max(a.pos ? a.pos[t] : index, 0), a.positions - 1);
        const float* r = a.rot + (size_t)pos * a.ld_rot + VW * piece;
#pragma unroll
        for (int e = 0; e < VW; ++e) {
            cs[e] = r[e];
            sn[e] = r[half + e];
        }
    }
    const int hq = a.q ? a.heads : 0, total = hq + 2 * c.kv;
    for (int h = part * side + first; h < total; h += parts * side) {
        const bool is_q = h < hq, is_v = h >= hq + c.kv;
        const int hh = is_q ? h : is_v ? h - hq - c.kv : h - hq;
        const __half* src = is_q ? a.q + (size_t)t * a.ldq : is_v ? a.v + (size_t)t * a.ldv : a.k + (size_t)t * a.ldk;
        src += (size_t)hh * c.d;
        __half* dst = is_q ? a.q_out + (size_t)t * a.ldq_out + (size_t)hh * c.d : is_v ? vd : kd;
        if (!dst) continue;   // (a token without a slot)
        if (!is_q) dst += (size_t)hh * c.head_stride;
        _Float16 x[VW], y[VW];
        if (piece < pairs) {
            get<VW>(src + VW * piece, x);
            get<VW>(src + half + VW * piece, y);
            if (!is_v) {
#pragma unroll
                for (int e = 0; e < VW; ++e) {
                    const float p = (float)x[e], q = (float)y[e];
                    x[e] = (_Float16)(p * cs[e] - q * sn[e]);
                    y[e] = (_Float16)(q * cs[e] + p * sn[e]);
                }
            }
            put<VW>(dst + VW * piece, x);
            put<VW>(dst + half + VW * piece, y);
        } else {
            // behind the pairs: two pieces at a time, like a pair
            const int p0 = 2 * pairs + 2 * (piece - pairs);
            if (p0 + 1 < whole) {
                get<VW>(src + VW * p0, x);
                get<VW>(src + VW * (p0 + 1), y);
                put<VW>(dst + VW * p0, x);
                put<VW>(dst + VW * (p0 + 1), y);
            } else {
                get<VW>(src + VW * p0, x);
                put<VW>(dst + VW * p0, x);
            }
        }
    }
}

template <int VW>
void launch(const Cache& c, const Append& a, hipStream_t s) {
    const int pairs = a.rot_dim / 2 / VW, whole = c.d / VW;
    const int pieces = pairs + (whole - 2 * pairs + 1) / 2;   // (d is a multiple of 8, so d / VW and both halves are whole pieces)
    const int total = (a.q ? a.heads : 0) + 2 * c.kv;
    const int side = min(256 / pieces, total);
    // A token's heads go to one workgroup where there are tokens enough to fill the GPU, else to as many as have a round of heads each.
    const int rounds = (total + side - 1) / side;
    const int parts = a.tokens >= 2048 ? 1 : min(rounds, (2048 + a.tokens - 1) / a.tokens);
    append_kernel<VW><<<(unsigned)((int64_t)a.tokens * parts), (unsigned)(side * pieces + 63) / 64 * 64, 0, s>>>(c, a, parts, pieces, side);
}

}  // namespace

hipError_t cache_append(const Cache& c, const Append& a, hipStream_t s) {
    // The widest pieces that both halves of a pair consist of; every row and head starts on 16 bytes.
    const int half = a.rot_dim / 2;
    if (half % 8 == 0) launch<8>(c, a, s);
    else if (half % 4 == 0) launch<4>(c, a, s);
    else if (half % 2 == 0) launch<2>(c, a, s);
    else launch<1>(c, a, s);
    return hipGetLastError();
}

}  // namespace qeft
