// Eviction from a paged cache by accumulated attention weight (qeft_cache_evict).
//
// A row is one kv head of one sequence: n tokens with a weight and a position each, of which `budget` stay.  Order of preference: rank (weight as an ordered
// 32-bit key, or the key of +infinity for the first and last positions) from high to low, then slot from low to high.  The kept set is everything before
// one border in that order, (key, slot), which a workgroup finds with its row's keys in LDS:
//   few to go (a sequence one token over its budget): the least preferred token, so many times;
//   else a selection by digits of 8 bits from the top, each from a histogram of what still agrees with the border's digits; where the border cuts through
//   equal keys, the same again over the slots.
// Then kept tokens behind the budget are matched with freed slots before it, both counted off in slot order (a wave per share of the row, ballots).
// Bytes bound it: 16 a token for weights and positions, and 8 head_dim per token that moves.  Few moves are made by the same workgroup; where there can be many,
// they go into lists and a second launch spreads them over the GPU.
#include "qeft_internal.h"

namespace qeft {
namespace {

typedef uint32_t u4 __attribute__((ext_vector_type(4)));

constexpr int BINS = 256, COPIES = 16;          // a digit's histogram: counters of a bin side by side, a lane adds to its own of 16 (equal weights are common:
                                                // one counter would take a wave's 64 additions one after the other)
constexpr int FEW = 4;                          // tokens to go that are found one by one
constexpr int INLINE_MOVES = 32;                // moves that the selecting workgroup makes itself
constexpr int MAX_KEYS = 35 * 1024;             // keys that fit LDS beside the histogram and the lists
constexpr uint32_t KEY_INF = 0xff800000u;

__device__ __forceinline__ uint32_t key_of(float x) {
    const uint32_t u = __builtin_bit_cast(uint32_t, x + 0.f);   // (-0 becomes +0)
    if (x != x) return 0xffffffffu;
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

struct Moves {
    int* count;   // [rows]
    int* src;     // [rows][cap]
    int* dst;
    int cap;
};

__device__ __forceinline__ __half* slot_ptr(const Cache& c, __half* pool, int b, int h, int t) {
    const int p = c.by_page.of(t);
    const int page = min(max(c.table[(size_t)b * c.ld_table + p], 0), c.pages - 1);
    return pool + (size_t)page * c.page_stride + (size_t)h * c.head_stride + (size_t)(t - p * c.page_size) * c.token_stride;
}

// Moves number first, first + step, ... of a row: `lane` of the 16 that share a move takes pieces lane, lane + 16, ... of both rows.
__device__ __forceinline__ void move_rows(const Cache& c, int b, int h, const int* src, const int* dst, int count, int first, int step, int lane) {
    for (int i = first; i < count; i += step) {
        const int s = src[i], t = dst[i];
        const __half *ks = slot_ptr(c, c.k, b, h, s), *vs = slot_ptr(c, c.v, b, h, s);
        __half *kd = slot_ptr(c, c.k, b, h, t), *vd = slot_ptr(c, c.v, b, h, t);
        for (int x = 8 * lane; x < c.d; x += 128) {
            const u4 k = *reinterpret_cast<const u4*>(ks + x), v = *reinterpret_cast<const u4*>(vs + x);
            *reinterpret_cast<u4*>(kd + x) = k;
            *reinterpret_cast<u4*>(vd + x) = v;
        }
    }
}

// The digit at `shift` of the border, among the values that agree with `prefix` above it: from the top down, the bin in which the `want`-th value lies.
// `each(f)` calls f(value) for every value of this thread.  Returns prefix with the digit; want becomes the rank within the bin, size its values.
template <class Each>
__device__ __forceinline__ uint32_t border_digit(int* hist, int* bins, int* found, uint32_t prefix, int shift, int& want, int& size, const Each& each) {
    const int tid = threadIdx.x, lane = tid & 63;
    for (int i = tid; i < BINS * COPIES; i += blockDim.x) hist[i] = 0;
    __syncthreads();
    const uint32_t above = shift == 24 ? 0u : 0xffffffffu << (shift + 8);
    each([&](uint32_t v) {
        if ((v & above) == (prefix & above)) atomicAdd(&hist[((v >> shift) & 255) * COPIES + (lane & (COPIES - 1))], 1);
    });
    __syncthreads();
    for (int i = tid; i < BINS; i += blockDim.x) {
        int s = 0;
#pragma unroll
        for (int x = 0; x < COPIES; ++x) s += hist[i * COPIES + x];
        bins[i] = s;
    }
    __syncthreads();
    if (tid < 64) {   // lane 0 has the four highest bins
        int own[4], sum = 0;
#pragma unroll
        for (int x = 0; x < 4; ++x) sum += own[x] = bins[BINS - 1 - (4 * lane + x)];
        int before = sum;
#pragma unroll
        for (int x = 1; x < 64; x <<= 1) {
            const int y = __shfl_up(before, x);
            if (lane >= x) before += y;
        }
        before -= sum;
        if (want > before && want <= before + sum) {
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                if (want > before && want <= before + own[x]) {
                    found[0] = BINS - 1 - (4 * lane + x);
                    found[1] = want - before;
                    found[2] = own[x];
                }
                before += own[x];
            }
        }
    }
    __syncthreads();
    want = found[1];
    size = found[2];
    return prefix | (uint32_t)found[0] << shift;
}

// Workgroup = a row.  IN_LDS: the keys stay in LDS, else every pass takes them from the inputs again.
template <bool IN_LDS>
__global__ __launch_bounds__(1024) void evict_select_kernel(Cache c, Evict a, Moves mv) {
    extern __shared__ __align__(16) uint32_t shared[];
    int* hist = (int*)shared;                                // [BINS * COPIES]
    uint32_t* keys = shared + BINS * COPIES;                 // [longest] if IN_LDS
    __shared__ int bins[BINS], found[3], holes[16], movers[16];
    __shared__ uint64_t least[16];
    __shared__ int src[INLINE_MOVES], dst[INLINE_MOVES];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), waves = blockDim.x >> 6;
    const int row = blockIdx.x, b = row / c.kv, h = row % c.kv;
    const int n = min(max(a.lens[b], 0), a.longest), left = min(n, a.budget);
    if (h == 0 && tid == 0) a.lens_out[b] = left;
    const float* score = a.score + (size_t)row * a.ld;
    const int* pos = a.pos + (size_t)row * a.ld;
    float* score_out = a.score_out + (size_t)row * a.ld_out;
    int* pos_out = a.pos_out + (size_t)row * a.ld_out;
    const bool copy_score = a.score_out != a.score, copy_pos = a.pos_out != a.pos;
    const bool listed = mv.count != nullptr;
    if (n == left) {
        for (int t = tid; t < n; t += blockDim.x) {
            if (copy_score) score_out[t] = score[t];
            if (copy_pos) pos_out[t] = pos[t];
        }
        if (listed && tid == 0) mv.count[row] = 0;
        return;
    }
    const int64_t recent = (int64_t)a.seen[b] - a.keep_last;
    auto rank = [&](float s, int p) { return p < a.keep_first || p >= recent ? KEY_INF : key_of(s); };
    // weights and positions of the slots that stay go out as they come; what moves into a freed slot is written over them below
    for (int t = tid; t < n; t += blockDim.x) {
        const float s = score[t];
        const int p = pos[t];
        if (IN_LDS) keys[t] = rank(s, p);
        if (t < left) {
            if (copy_score) score_out[t] = s;
            if (copy_pos) pos_out[t] = p;
        }
    }
    __syncthreads();
    auto key_at = [&](int t) -> uint32_t { return IN_LDS ? keys[t] : rank(score[t], pos[t]); };

    uint32_t border = 0;   // kept: key > border, or key == border in a slot < cut
    int cut = 0;
    const int go = n - left;
    if (left == 0) {
        border = 0xffffffffu;
    } else if (go <= FEW) {
        // the least preferred: the smallest (key, slots from the highest down)
        uint64_t last = 0;
        for (int i = 0; i < go; ++i) {
            uint64_t mine = ~0ull;
            for (int t = tid; t < n; t += blockDim.x) {
                const uint64_t v = (uint64_t)key_at(t) << 32 | (uint32_t)~t;
                if (v < mine && (i == 0 || v > last)) mine = v;
            }
#pragma unroll
            for (int x = 1; x < 64; x <<= 1) {
                const uint64_t o = (uint64_t)__shfl_xor((unsigned long long)mine, x);
                mine = o < mine ? o : mine;
            }
            if (lane == 0) least[wave] = mine;
            __syncthreads();
            for (int w = 0; w < waves; ++w) mine = least[w] < mine ? least[w] : mine;
            __syncthreads();
            last = mine;
        }
        border = (uint32_t)(last >> 32);
        cut = (int)~(uint32_t)last;
    } else {
        int want = left, size = n;
        for (int shift = 24; shift >= 0; shift -= 8)
            border = border_digit(hist, bins, found, border, shift, want, size, [&](auto&& f) {
                for (int t = tid; t < n; t += blockDim.x) f(key_at(t));
            });
        cut = n;   // all of the border's key, or the `want` lowest slots of it: the highest values of ~slot
        if (want < size) {
            uint32_t low = 0;
            for (int shift = 24; shift >= 0; shift -= 8)
                low = border_digit(hist, bins, found, low, shift, want, size, [&](auto&& f) {
                    for (int t = tid; t < n; t += blockDim.x)
                        if (key_at(t) == border) f(~(uint32_t)t);
                });
            cut = (int)~low + 1;
        }
    }

    // freed slots below `left`, kept tokens from `left` on: counted per wave, then written in order.  A wave has a share of whole groups of 64.
    const int share = (n + 64 * waves - 1) / (64 * waves) * 64, from = wave * share, to = min(n, from + share);
    auto kept = [&](int t) {
        const uint32_t k = key_at(t);
        return k > border || (k == border && t < cut);
    };
    int nh = 0, nm = 0;
    for (int t0 = from; t0 < to; t0 += 64) {
        const int t = t0 + lane;
        const bool in = t < to, k = in && kept(t);
        nh += __popcll(__ballot(in && !k && t < left));
        nm += __popcll(__ballot(k && t >= left));
    }
    if (lane == 0) {
        holes[wave] = nh;
        movers[wave] = nm;
    }
    __syncthreads();
    int at_h = 0, at_m = 0, count = 0;
    for (int w = 0; w < waves; ++w) {
        if (w < wave) {
            at_h += holes[w];
            at_m += movers[w];
        }
        count += movers[w];
    }
    int* ls = listed ? mv.src + (size_t)row * mv.cap : src;
    int* ld = listed ? mv.dst + (size_t)row * mv.cap : dst;
    if (nh | nm) {
        for (int t0 = from; t0 < to; t0 += 64) {
            const int t = t0 + lane;
            const bool in = t < to, k = in && kept(t), hole = in && !k && t < left, mover = k && t >= left;
            const uint64_t bh = __ballot(hole), bm = __ballot(mover), below = ((uint64_t)1 << lane) - 1;
            if (hole) ld[at_h + __popcll(bh & below)] = t;
            if (mover) ls[at_m + __popcll(bm & below)] = t;
            at_h += __popcll(bh);
            at_m += __popcll(bm);
        }
    }
    __syncthreads();   // (the lists, and the copies that what follows writes over)
    for (int i = tid; i < count; i += blockDim.x) {
        const int s = ls[i], t = ld[i];
        score_out[t] = score[s];
        pos_out[t] = pos[s];
    }
    if (listed) {
        if (tid == 0) mv.count[row] = count;
    } else {
        move_rows(c, b, h, src, dst, count, tid >> 4, blockDim.x >> 4, tid & 15);
    }
}

constexpr int TILE_MOVES = 64;

// Workgroup = TILE_MOVES moves of a row, 16 lanes a move.
__global__ __launch_bounds__(256) void evict_move_kernel(Cache c, Moves mv, int tiles) {
    const int row = blockIdx.x / tiles, tile = blockIdx.x % tiles;
    const int count = min(mv.count[row] - tile * TILE_MOVES, TILE_MOVES);
    const size_t at = (size_t)row * mv.cap + (size_t)tile * TILE_MOVES;
    move_rows(c, row / c.kv, row % c.kv, mv.src + at, mv.dst + at, count, threadIdx.x >> 4, 16, threadIdx.x & 15);
}

int most_moves(int longest, int budget) { return budget < longest - budget ? budget : longest - budget; }

}  // namespace

size_t evict_workspace(int kv, int64_t seqs, int longest, int budget) {
    const int cap = most_moves(longest, budget);
    if (cap <= INLINE_MOVES) return 0;
    return (size_t)seqs * kv * (1 + 2 * (size_t)cap) * sizeof(int);
}

hipError_t cache_evict(const Cache& c, const Evict& a, hipStream_t s) {
    const int rows = c.seqs * c.kv, cap = most_moves(a.longest, a.budget);
    Moves mv{};
    if (cap > INLINE_MOVES) {
        mv.cap = cap;
        mv.src = (int*)a.ws;
        mv.dst = mv.src + (size_t)rows * cap;
        mv.count = mv.dst + (size_t)rows * cap;
    }
    const int threads = a.longest <= 4096 ? 512 : 1024;
    const bool in_lds = a.longest <= MAX_KEYS;
    const size_t lds = (size_t)BINS * COPIES * 4 + (in_lds ? (size_t)a.longest * 4 : 0);
    static bool raised = false;   // (see qeft.h: the one kind of state)
    if (in_lds && lds > 48 * 1024 && !raised) {
        const hipError_t e = hipFuncSetAttribute((const void*)evict_select_kernel<true>, hipFuncAttributeMaxDynamicSharedMemorySize, (MAX_KEYS + BINS * COPIES) * 4);
        if (e != hipSuccess) return e;
        raised = true;
    }
    if (in_lds) evict_select_kernel<true><<<rows, threads, lds, s>>>(c, a, mv);
    else evict_select_kernel<false><<<rows, threads, lds, s>>>(c, a, mv);
    if (mv.count) {
        const int tiles = (cap + TILE_MOVES - 1) / TILE_MOVES;
        evict_move_kernel<<<(unsigned)((int64_t)rows * tiles), 256, 0, s>>>(c, mv, tiles);
    }
    return hipGetLastError();
}

}  // namespace qeft
