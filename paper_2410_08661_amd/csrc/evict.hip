// Eviction from a paged cache by accumulated attention weight (qeft_cache_evict).
//
// A row is one kv head of one sequence: n tokens with a weight and a position each, of which `budget` stay.  Order of preference: rank (weight as an ordered
// 32-bit key, or the key of +infinity for the first and last positions) from high to low, then slot from low to high.  The kept set is everything before
// one border in that order, (key, slot), which a workgroup finds with its row's keys in registers, 4 to 32 a thread (rows beyond 32768
// tokens: several workgroups a row, a launch a step, or one that reads the row again for each):
//   few to go (a sequence one token over its budget): the least preferred token, so many times;
//   else three digits from the top, 11, 11 and 10 bits (eight would be a float's exponent, and say little), each from a histogram in LDS of the keys that agree with
//   the border above it; fewer digits where a bin's keys all stay.  (Bisection over the key, a comparison, a scalar count and an addition a key and step, takes 1 us a
//   step for 32768 keys, bound by the scalar unit, and some 25 steps.)
//   Where the border cuts through equal keys, they are counted off in slot order.
// What changes is a bit a token: freed slots before the budget, kept tokens behind it.  The i-th of the one takes the i-th of the other in, both counted off in
// slot order.  Where a call has few to move the workgroup does that itself; else the bits go to the workspace and a second launch has a workgroup for every
// 128 tokens behind the budget, which counts the bits before its own.
// Bytes bound it: 16 a token for weights and positions, and 8 head_dim per token that moves.  16 x 32 rows of 2049 tokens, one to go: 5.9 us (latencies of one
// workgroup a row; the bytes alone 3.4); 8 rows, 32768 -> 4096: 24 us for the selection (loads 4, three digits 13, equal keys 1.6, bits 4: eight CUs), 10 for the moves.
#include <algorithm>
#include "qeft_internal.h"
#include "wave.h"

namespace qeft {
namespace {

typedef uint32_t u4 __attribute__((ext_vector_type(4)));
typedef int i4 __attribute__((ext_vector_type(4)));
typedef float f4 __attribute__((ext_vector_type(4)));

constexpr int FEW = 4;                          // tokens to go that are found one by one
constexpr int TILE = 128;                       // tokens behind the budget whose moves one workgroup of the second launch makes; also the most that the first does
constexpr int MAX_IN_REGISTERS = 32 * 1024;     // keys that a workgroup's registers hold, 32 a thread
constexpr uint32_t KEY_INF = 0xff800000u;

// Ordered like the value, or like +infinity for the positions that always stay; never 0.
__device__ __forceinline__ uint32_t key_of(float x, int pos, int first, int recent) {
    const uint32_t u = __builtin_bit_cast(uint32_t, x + 0.f);   // (-0 becomes +0)
    uint32_t k = u ^ ((uint32_t)((int)u >> 31) | 0x80000000u);
    k = x != x ? 0xffffffffu : k;
    return ((pos < first) | (pos >= recent)) ? KEY_INF : k;
}
__device__ __forceinline__ int first_recent(int seen, int keep_last) {
    const int64_t r = (int64_t)seen - keep_last;
    return r < INT32_MIN ? INT32_MIN : (int)r;
}

// A row's arrays.
struct Row {
    int b, h, n, left;
    const float* score;
    const int* pos;
    float* score_out;
    int* pos_out;
};
__device__ __forceinline__ Row row_at(const Cache& c, const Evict& a, int row) {
    Row r;
    r.b = row / c.kv;
    r.h = row % c.kv;
    r.n = min(max(a.lens[r.b], 0), a.longest);
    r.left = min(r.n, a.budget);
    r.score = a.score + (size_t)row * a.ld;
    r.pos = a.pos + (size_t)row * a.ld;
    r.score_out = a.score_out + (size_t)row * a.ld_out;
    r.pos_out = a.pos_out + (size_t)row * a.ld_out;
    return r;
}

// Where token t's row begins, in either pool.  A page out of range is clamped to be read from, and nothing is written to it: OUT gives a place below 0.
template <bool OUT>
__device__ __forceinline__ int64_t slot_at(const Cache& c, int b, int h, int t) {
    const int p = c.by_page.of(t), named = c.table[(size_t)b * c.ld_table + p], page = min(max(named, 0), c.pages - 1);
    const int64_t at = (int64_t)page * c.page_stride + h * c.head_stride + (t - p * c.page_size) * c.token_stride;
    return OUT && named != page ? -1 : at;
}

// What changes in a row: a bit a token, set for freed slots below row.left and for kept tokens behind it, and before every word of 64 the number of bits
// set in the words below.
struct Changes {
    const uint64_t* bits;
    const int* below;
};

struct MoveLists {
    int src[TILE], dst[TILE];
};

// The moves of the kept tokens in [from, to) (TILE at most).  A workgroup; AT_ONCE: moves of 16 lanes that are loaded before the first is stored.
template <int AT_ONCE>
__device__ __forceinline__ void make_moves(const Cache& c, const Row& r, const Changes& ch, int from, int to, MoveLists& l) {
    const int tid = threadIdx.x, T = blockDim.x, lane = tid & 63, wave = tid >> 6, waves = T >> 6;
    const uint64_t under = ((uint64_t)1 << lane) - 1;
    auto low = [](int n) { return ((uint64_t)1 << n) - 1; };   // the n lowest bits, n < 64
    // set bits below row.left (the freed slots) and below `from`: the first mover's rank is the difference, and so for the end
    const int cl = r.left / 64, cf = from / 64, ct = (to - 1) / 64;
    const int holes = ch.below[cl] + __popcll(ch.bits[cl] & low(r.left & 63));
    const int first = ch.below[cf] + __popcll(ch.bits[cf] & low(from & 63)) - holes;
    const int last = ch.below[ct] + __popcll(ch.bits[ct] & (low((to - 1) & 63) | (uint64_t)1 << ((to - 1) & 63))) - holes;
    const int count = last - first;
    if (count == 0) return;
    // the movers, three words at most: a wave a word, a lane a token
    for (int w = cf + wave; w <= ct; w += waves) {
        const uint64_t x = ch.bits[w];
        const int t = 64 * w + lane, rank = ch.below[w] + __popcll(x & under) - holes - first;
        if ((x >> lane & 1) && t >= from && t < to) l.src[rank] = t;
    }
    // the freed slots of ranks first .. last - 1: a wave looks through 64 words at a time for those that hold any, then takes these one by one
    for (int w0 = 64 * wave; w0 <= cl; w0 += 64 * waves) {
        const int w = w0 + lane;
        uint64_t x = 0;
        int at = 0;
        if (w <= cl) {
            x = ch.bits[w];
            at = ch.below[w];
            if (w == cl) x &= low(r.left & 63);
        }
        for (uint64_t hit = __ballot(x != 0 && at < last && at + __popcll(x) > first); hit; hit &= hit - 1) {
            const int o = __builtin_ctzll(hit);
            const uint64_t y = (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(x >> 32), o) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)x, o);
            const int rank = __builtin_amdgcn_readlane(at, o) + __popcll(y & under);
            if ((y >> lane & 1) && rank >= first && rank < last) l.dst[rank - first] = 64 * (w0 + o) + lane;
        }
    }
    __syncthreads();
    if (tid < count) {
        const int s = l.src[tid], t = l.dst[tid];
        r.score_out[t] = r.score[s];
        r.pos_out[t] = r.pos[s];
    }
    // 16 lanes a move, K and V
    const int groups = T >> 4;
    for (int i0 = tid >> 4; i0 < count; i0 += AT_ONCE * groups) {
        int64_t from_at[AT_ONCE], to_at[AT_ONCE];
#pragma unroll
        for (int y = 0; y < AT_ONCE; ++y) {
            const int i = min(i0 + y * groups, count - 1);
            from_at[y] = slot_at<false>(c, r.b, r.h, l.src[i]);
            to_at[y] = slot_at<true>(c, r.b, r.h, l.dst[i]);
        }
        for (int x = 8 * (tid & 15); x < c.d; x += 128) {
            u4 k[AT_ONCE], v[AT_ONCE];
#pragma unroll
            for (int y = 0; y < AT_ONCE; ++y) {
                if (i0 + y * groups >= count) continue;
                k[y] = *reinterpret_cast<const u4*>(c.k + from_at[y] + x);
                v[y] = *reinterpret_cast<const u4*>(c.v + from_at[y] + x);
            }
#pragma unroll
            for (int y = 0; y < AT_ONCE; ++y) {
                if (i0 + y * groups >= count || to_at[y] < 0) continue;
                *reinterpret_cast<u4*>(c.k + to_at[y] + x) = k[y];
                *reinterpret_cast<u4*>(c.v + to_at[y] + x) = v[y];
            }
        }
    }
}

// The border of a row's keys, 4 J a thread: `left` keys stay, all from lo on if exact, else all above lo and `want` of those equal to it.
struct Border {
    uint32_t lo;
    bool exact;
    int want;
};
constexpr int BINS = 1 << 11;
// Counters of a bin side by side, a lane adds to its own: equal weights are common, and one counter takes a wave's 64 additions one after the other.  More of
// them cost more to clear and to read, which a workgroup of few keys notices.
template <int J> constexpr int COPIES = J == 1 ? 2 : J < 8 ? 4 : 8;
struct DigitShared {
    int tally[16], found[3];
};
template <int J>
__device__ __forceinline__ Border find_border(const uint32_t (&key)[J][4], int left, int* hist, DigitShared& sh) {
    constexpr int C = COPIES<J>;
    const int tid = threadIdx.x, T = blockDim.x, lane = tid & 63, wave = tid >> 6;
    Border r{0, false, left};
#pragma unroll 1
    for (int shift = 21; !r.exact; shift = shift == 21 ? 10 : 0) {
        for (int i = 4 * tid; i < BINS * C; i += 4 * T) *reinterpret_cast<i4*>(hist + i) = i4{0, 0, 0, 0};
        __syncthreads();
        const uint32_t mask = shift == 0 ? 1023 : 2047, known = shift == 21 ? 0 : ~0u << (shift == 10 ? 21 : 10);
#pragma unroll
        for (int j = 0; j < J; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const uint32_t k = key[j][e];
                if (k != 0 && ((k ^ r.lo) & known) == 0) atomicAdd(&hist[((k >> shift) & mask) * C + (lane & (C - 1))], 1);
            }
        __syncthreads();
        // runs of 4 bins, the highest first: thread x has runs x, x + T, ... of 512; a sum over runs needs them in order, so threads take neighbouring ones
        const int per = (BINS / 4 + T - 1) / T, first = per * tid;   // runs of this thread: 1 to 4
        int sum = 0;
        for (int x = 0; x < per && first + x < BINS / 4; ++x) {
            const i4* p = reinterpret_cast<const i4*>(hist + (size_t)(BINS - 4 * (first + x + 1)) * C);
#pragma unroll
            for (int y = 0; y < C; ++y) sum += p[y].x + p[y].y + p[y].z + p[y].w;
        }
        const int upto = wave_upto(sum);
        if (lane == 63) sh.tally[wave] = upto;
        __syncthreads();
        int before = upto - sum + waves_reduce(sh.tally, 0, wave, 0, Sum());
        if (r.want > before && r.want <= before + sum) {   // one thread
            for (int bin = BINS - 4 * first - 1;; --bin) {
                int own = 0;
#pragma unroll
                for (int y = 0; y < C; ++y) own += hist[bin * C + y];
                if (r.want <= before + own) {
                    sh.found[0] = bin;
                    sh.found[1] = r.want - before;
                    sh.found[2] = own;
                    break;
                }
                before += own;
            }
        }
        __syncthreads();
        r.lo |= (uint32_t)sh.found[0] << shift;
        r.want = sh.found[1];
        r.exact = sh.found[2] == r.want;
        if (shift == 0) break;
    }
    return r;
}

// The tokens to go are at most FEW: the least preferred one, so many times.  What may move is known beforehand, the last `go` tokens, and was loaded beside
// the keys: 32 threads a token, 16 of them for K's row and 16 for V's.
template <int J>
__device__ __forceinline__ void evict_few(const Cache& c, const Row& r, const uint32_t (&key)[J][4], const u4 (&carried)[2], float carried_score, int carried_pos, uint64_t (*least)[16]) {
    const int tid = threadIdx.x, T = blockDim.x, waves = T >> 6, go = r.n - r.left;
    int gone[FEW];
    uint64_t last = 0;
#pragma unroll
    for (int i = 0; i < FEW; ++i) {
        gone[i] = -1;
        if (i >= go) continue;
        uint64_t x = ~0ull;   // (key, slots from the highest down)
        int t0 = 4 * tid;
        asm volatile("" : "+v"(t0));   // (or the compiler keeps every slot's number for all rounds)
#pragma unroll
        for (int j = 0; j < J; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                uint32_t k = key[j][e];
                asm volatile("" : "+v"(k));   // (or it is kept as the upper half of a pair all the time)
                const uint64_t v = (uint64_t)k << 32 | (uint32_t)~(t0 + 4 * j * T + e);
                if (k != 0 && v < x && v > last) x = v;
            }
        x = wave_reduce(x, Least());
        if ((tid & 63) == 0) least[i & 1][tid >> 6] = x;
        __syncthreads();
        last = waves_reduce(least[i & 1], 0, waves, ~(uint64_t)0, Least());
        gone[i] = (int)~(uint32_t)last;
    }
    const int mine = tid >> 5, token = r.left + mine;
    if (mine >= go) return;
    // the mover's rank among the movers; the freed slot of the same rank
    int rank = 0, to = -1;
#pragma unroll
    for (int t = 0; t < FEW; ++t)
        if (t < mine) {
            bool stays = true;
#pragma unroll
            for (int i = 0; i < FEW; ++i) stays &= gone[i] != r.left + t;
            rank += stays;
        }
#pragma unroll
    for (int i = 0; i < FEW; ++i) {
        if (gone[i] == token) return;
        if (gone[i] < 0 || gone[i] >= r.left) continue;
        int lower = 0;
#pragma unroll
        for (int k = 0; k < FEW; ++k) lower += gone[k] >= 0 && gone[k] < gone[i];
        if (lower == rank) to = gone[i];
    }
    if (to < 0) return;
    if ((tid & 31) == 0) {
        r.score_out[to] = carried_score;
        r.pos_out[to] = carried_pos;
    }
    const int64_t at = slot_at<true>(c, r.b, r.h, to);
    if (at < 0) return;
    __half* p = (tid & 16 ? c.v : c.k) + at + 8 * (tid & 15);
    if (8 * (tid & 15) < c.d) *reinterpret_cast<u4*>(p) = carried[0];
    if (8 * (tid & 15) + 128 < c.d) *reinterpret_cast<u4*>(p + 128) = carried[1];
}

// Workgroup = a row of at most 4 J blockDim.x tokens.  VEC: rows start on 16 bytes.  all_bits: where the bits go, [rows][words], or NULL: no row has more than TILE to go.
template <int J, bool VEC>
__global__ __launch_bounds__(1024, J == 1 ? 8 : 4) void evict_select_kernel(Cache c, Evict a, uint64_t* all_bits, int* all_below, int words) {
    constexpr int WORDS = 4 * J * 1024 / 64;
    __shared__ __align__(16) uint64_t bits[WORDS];
    __shared__ int below[WORDS];
    __shared__ uint64_t least[2][16];
    __shared__ int counts[16 * J];
    __shared__ int cut_at;
    __shared__ MoveLists lists;
    __shared__ DigitShared digit;
    extern __shared__ __align__(16) int hist[];   // [BINS][COPIES<J>]
    const int tid = threadIdx.x, T = blockDim.x, lane = tid & 63, wave = tid >> 6, waves = T >> 6;
    const Row r = row_at(c, a, blockIdx.x);
    const int n = r.n, left = r.left, go = n - left;
    if (r.h == 0 && tid == 0) a.lens_out[r.b] = left;
    const bool copy_score = a.score_out != a.score, copy_pos = a.pos_out != a.pos;
    const int recent = first_recent(a.seen[r.b], a.keep_last);
    const bool few = go > 0 && go <= FEW && left > 0;
    u4 carried[2];
    float carried_score = 0.f;
    int carried_pos = 0;
    if (few && (tid >> 5) < go) {
        const int token = left + (tid >> 5);
        const __half* p = (tid & 16 ? c.v : c.k) + slot_at<false>(c, r.b, r.h, token) + 8 * (tid & 15);
        if (8 * (tid & 15) < c.d) carried[0] = *reinterpret_cast<const u4*>(p);
        if (8 * (tid & 15) + 128 < c.d) carried[1] = *reinterpret_cast<const u4*>(p + 128);
        carried_score = r.score[token];
        carried_pos = r.pos[token];
    }

    // Vector j of an array: a base that all lanes share and one offset for all of a lane's, or the compiler keeps 64 addresses a thread.
    const uint32_t offset = 16u * tid;
    auto vec_of = [&](const void* p, int j) { return (const char*)p + 16 * (size_t)(j * T) + offset; };
    auto vec_to = [&](void* p, int j) { return (char*)p + 16 * (size_t)(j * T) + offset; };
    uint32_t key[J][4];   // token 4 (j T + tid) + e; 0: no token
    constexpr int AT_ONCE = J < 4 ? J : 4;
#pragma unroll
    for (int j0 = 0; j0 < J; j0 += AT_ONCE) {
        f4 s[AT_ONCE];
        i4 p[AT_ONCE];
#pragma unroll
        for (int y = 0; y < AT_ONCE; ++y) {   // loads before the first use
            const int t = 4 * ((j0 + y) * T + tid);
            if (VEC && t + 4 <= n) {
                s[y] = *reinterpret_cast<const f4*>(vec_of(r.score, j0 + y));
                p[y] = *reinterpret_cast<const i4*>(vec_of(r.pos, j0 + y));
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    s[y][e] = t + e < n ? reinterpret_cast<const float*>(vec_of(r.score, j0 + y))[e] : 0.f;
                    p[y][e] = t + e < n ? reinterpret_cast<const int*>(vec_of(r.pos, j0 + y))[e] : 0;
                }
            }
        }
        // weights and positions of the slots that stay go out as they came; what moves into a freed slot is written over them later
#pragma unroll
        for (int y = 0; y < AT_ONCE; ++y) {
            const int t = 4 * ((j0 + y) * T + tid);
            if (VEC && t + 4 <= left) {
                if (copy_score) *reinterpret_cast<f4*>(vec_to(r.score_out, j0 + y)) = s[y];
                if (copy_pos) *reinterpret_cast<i4*>(vec_to(r.pos_out, j0 + y)) = p[y];
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (t + e < left) {
                        if (copy_score) reinterpret_cast<float*>(vec_to(r.score_out, j0 + y))[e] = s[y][e];
                        if (copy_pos) reinterpret_cast<int*>(vec_to(r.pos_out, j0 + y))[e] = p[y][e];
                    }
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const uint32_t k = key_of(s[y][e], p[y][e], a.keep_first, recent);
                key[j0 + y][e] = t + e >= n ? 0u : k;
            }
        }
    }
    // (rows of one call can be of any kind: those whose moves are made here, or that have none, leave no bits)
    const bool moves = go > 0 && !few && left > 0;
    if (moves) {
        const Border border = find_border<J>(key, left, hist, digit);
        const uint32_t lo = border.lo;
        const bool exact = border.exact;
        // equal keys at the border: those in the lowest slots stay, `want` of them
        int cut = n;
        if (!exact) {
            const int want = border.want;
#pragma unroll
            for (int j = 0; j < J; ++j) {
                int all = 0;
#pragma unroll
                for (int e = 0; e < 4; ++e) all += __popcll(__ballot(key[j][e] == lo));
                if (lane == 0) counts[j * waves + wave] = all;
            }
            __syncthreads();
            // sums over the vectors one after the other and the waves within them, the slots' order; up to four counts a lane
            constexpr int PER = (16 * J + 63) / 64;
            int own[PER], sum = 0;
#pragma unroll
            for (int x = 0; x < PER; ++x) {
                const int o = PER * lane + x;
                sum += own[x] = o < J * waves ? counts[o] : 0;
            }
            const int upto = wave_upto(sum), l = __builtin_ctzll(__ballot(upto >= want));   // (there are enough)
            int before = __shfl(upto - sum, l), o = PER * l;
#pragma unroll
            for (int x = 0; x + 1 < PER; ++x) {
                const int y = __shfl(own[x], l);
                if (o == PER * l + x && before + y < want) before += y, ++o;
            }
            if (o % waves == wave) {
#pragma unroll
                for (int j = 0; j < J; ++j) {
                    if (o / waves != j) continue;
                    int rank = before;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const uint64_t x = __ballot(key[j][e] == lo);
                        rank += __builtin_amdgcn_mbcnt_hi((uint32_t)(x >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)x, 0));
                    }
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (key[j][e] == lo && ++rank == want) cut_at = 4 * (j * T + tid) + e + 1;
                }
            }
            __syncthreads();
            cut = cut_at;
        }
        // a bit a token, two threads to a byte: kept from lo on, but for the equal keys from `cut` on; changed below `left` where not kept
        int t0 = 4 * tid;
        asm volatile("" : "+v"(t0));   // (or the compiler keeps every comparison of a slot since the loads, a pair of registers each)
        auto first_of = [](int x) { return (1 << min(max(x, 0), 4)) - 1; };   // as many of four bits
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const int t = t0 + 4 * j * T;
            int f = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) f |= (int)(key[j][e] >= lo) << e;
            if (!exact) {
                int tie = 0;
#pragma unroll
                for (int e = 0; e < 4; ++e) tie |= (int)(key[j][e] == lo) << e;
                f &= ~(tie & ~first_of(cut - t));
            }
            f = (f ^ first_of(left - t)) & first_of(n - t);
            f |= (int)rotated<15>((uint32_t)f) << 4;   // (the next lane's)
            if ((tid & 1) == 0) reinterpret_cast<uint8_t*>(bits)[(j * T + tid) / 2] = (uint8_t)f;
        }
        __syncthreads();
        // the words' bits, summed up to each by the first wave
        const int used = (n + 63) / 64;
        if (wave == 0) {
            int passed = 0;
            for (int w0 = 0; w0 < used; w0 += 64) {
                const uint64_t x = w0 + lane < used ? bits[w0 + lane] : 0;
                const int own = __popcll(x), upto = wave_upto(own);
                if (w0 + lane < used) {
                    below[w0 + lane] = passed + upto - own;
                    if (all_bits) {
                        all_bits[(size_t)blockIdx.x * words + w0 + lane] = x;
                        all_below[(size_t)blockIdx.x * words + w0 + lane] = passed + upto - own;
                    }
                }
                passed += __builtin_amdgcn_readlane(upto, 63);
            }
        }
    }
    if (few) evict_few<J>(c, r, key, carried, carried_score, carried_pos, least);
    if (all_bits) {
        if (!moves)
            for (int w = tid; 64 * w < n; w += T) all_bits[(size_t)blockIdx.x * words + w] = 0, all_below[(size_t)blockIdx.x * words + w] = 0;
    } else if (moves) {
        __syncthreads();
        make_moves<1>(c, r, Changes{bits, below}, left, n, lists);
    }
}

// Rows of any length: the keys taken from the inputs again by each step, the border found digit by digit from histograms, 11, 11 and 10 bits.
constexpr int LONG_COPIES = 4;
__global__ __launch_bounds__(1024) void evict_select_long_kernel(Cache c, Evict a, uint64_t* all_bits, int* all_below, int words) {
    __shared__ __align__(16) int hist[BINS * LONG_COPIES];
    __shared__ int tally[16], found[3], cut_at;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const Row r = row_at(c, a, blockIdx.x);
    const int n = r.n, left = r.left;
    if (r.h == 0 && tid == 0) a.lens_out[r.b] = left;
    for (int t = tid; t < left; t += 1024) {
        if (a.score_out != a.score) r.score_out[t] = r.score[t];
        if (a.pos_out != a.pos) r.pos_out[t] = r.pos[t];
    }
    uint64_t* bits = all_bits + (size_t)blockIdx.x * words;
    int* below = all_below + (size_t)blockIdx.x * words;
    if (n == left || left == 0) {   // (always, where there is no workspace for bits)
        if (all_bits)
            for (int w = tid; 64 * w < n; w += 1024) bits[w] = 0, below[w] = 0;
        return;
    }
    const int recent = first_recent(a.seen[r.b], a.keep_last);
    auto key_from = [&](float s, int p) { return key_of(s, p, a.keep_first, recent); };
    // f(key, slot) for this thread's tokens in [from, to), `step` apart, eight loads at a time
    auto each = [&](int from, int to, int step, auto&& f) {
        for (int t0 = from; t0 < to; t0 += 8 * step) {
            float s[8];
            int p[8];
#pragma unroll
            for (int x = 0; x < 8; ++x) {
                const int t = t0 + x * step;
                s[x] = t < to ? r.score[t] : 0.f;
                p[x] = t < to ? r.pos[t] : 0;
            }
#pragma unroll
            for (int x = 0; x < 8; ++x)
                if (t0 + x * step < to) f(key_from(s[x], p[x]), t0 + x * step);
        }
    };
    uint32_t border = 0;
    int want = left, size = n;
    for (int d = 0; d < 3; ++d) {
        const int shift = d == 0 ? 21 : d == 1 ? 10 : 0, top = d == 0 ? 32 : d == 1 ? 21 : 10;
        const uint32_t mask = d == 2 ? 1023 : 2047;
        for (int i = tid; i < BINS * LONG_COPIES; i += 1024) hist[i] = 0;
        __syncthreads();
        each(tid, n, 1024, [&](uint32_t k, int) {
            if (d == 0 || k >> top == border >> top) atomicAdd(&hist[((k >> shift) & mask) * LONG_COPIES + (lane & (LONG_COPIES - 1))], 1);
        });
        __syncthreads();
        // two bins a thread, thread 0 the highest
        int own[2], sum = 0;
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            const i4 v = *reinterpret_cast<const i4*>(&hist[(BINS - 1 - (2 * tid + x)) * LONG_COPIES]);
            sum += own[x] = v.x + v.y + v.z + v.w;
        }
        const int upto_wave = wave_upto(sum);
        if (lane == 63) tally[wave] = upto_wave;
        __syncthreads();
        int before = upto_wave - sum;
        for (int w = 0; w < wave; ++w) before += tally[w];
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            if (want > before && want <= before + own[x]) {
                found[0] = BINS - 1 - (2 * tid + x);
                found[1] = want - before;
                found[2] = own[x];
            }
            before += own[x];
        }
        __syncthreads();
        border |= (uint32_t)found[0] << shift;
        want = found[1];
        size = found[2];
    }
    // a wave has a share of whole words; equal keys at the border are counted by shares first, `want` of them stay
    const int share = (n + 64 * 16 - 1) / (64 * 16) * 64, from = min(n, wave * share), to = min(n, from + share);
    int cut = n;
    if (want < size) {
        int mine = 0;
        each(from + lane, to, 64, [&](uint32_t k, int) { mine += k == border; });
        mine = wave_reduce(mine, Sum());
        if (lane == 0) tally[wave] = mine;
        __syncthreads();
        int before = 0;
        for (int w = 0; w < wave; ++w) before += tally[w];
        if (before < want && before + mine >= want) {
            for (int t0 = from; t0 < to && before < want; t0 += 64) {
                const int t = t0 + lane;
                const bool tie = t < to && key_from(r.score[t], r.pos[t]) == border;
                const uint64_t x = __ballot(tie);
                if (tie && before + __popcll(x & (((uint64_t)1 << lane) - 1)) + 1 == want) cut_at = t + 1;
                before += __popcll(x);
            }
        }
        __syncthreads();
        cut = cut_at;
    }
    int mine = 0;
    for (int t0 = from; t0 < to; t0 += 8 * 64) {
        float s[8];
        int p[8];
#pragma unroll
        for (int x = 0; x < 8; ++x) {
            const int t = t0 + 64 * x + lane;
            s[x] = t < to ? r.score[t] : 0.f;
            p[x] = t < to ? r.pos[t] : 0;
        }
#pragma unroll
        for (int x = 0; x < 8; ++x) {
            const int t = t0 + 64 * x + lane;
            const uint32_t k = key_from(s[x], p[x]);
            const uint64_t w = __ballot(t < to && (t < left) != (k > border || (k == border && t < cut)));
            if (t0 + 64 * x < to && lane == 0) {
                bits[t0 / 64 + x] = w;
                below[t0 / 64 + x] = mine;
            }
            mine += __popcll(w);
        }
    }
    __syncthreads();   // (tally may still be read)
    if (lane == 0) tally[wave] = mine;
    __syncthreads();
    int before = 0;
    for (int w = 0; w < wave; ++w) before += tally[w];
    for (int w = (from + 63) / 64 + lane; 64 * w < to; w += 64) below[w] += before;   // (a wave without tokens has none of the last word either)
}

// Few rows longer than a workgroup's registers hold: a row by many workgroups, PART tokens each, in five launches, a digit's histograms in each of the first three, then the bits, then their
// sums over the parts.  Every workgroup finds the border of the digit before from the sum of the row's histograms.  28 us for 8 rows of 40000 or of 131001, launches and latencies.
constexpr int PART = 8192;
struct Parts {
    int* hist;     // [3][rows * parts][BINS]
    int2* state;   // [rows][2]: the border after the first and the second digit, and how many of its keys stay
    int* count;    // [rows * parts]: changed tokens
    int parts;
};
template <int STEP>
__global__ __launch_bounds__(1024) void evict_part_kernel(Cache c, Evict a, Parts p, uint64_t* all_bits, int* all_below, int words) {
    __shared__ __align__(16) int hist[STEP < 3 ? BINS * LONG_COPIES : 4];
    __shared__ int tally[16], changes[16], found[3];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int row = blockIdx.x / p.parts, part = blockIdx.x % p.parts;
    const Row r = row_at(c, a, row);
    const int n = r.n, left = r.left, from = PART * part, to = min(n, from + PART);
    if (STEP == 0) {
        if (r.h == 0 && part == 0 && tid == 0) a.lens_out[r.b] = left;
        for (int t = from + tid; t < min(to, left); t += 1024) {
            if (a.score_out != a.score) r.score_out[t] = r.score[t];
            if (a.pos_out != a.pos) r.pos_out[t] = r.pos[t];
        }
    }
    uint64_t* bits = all_bits + (size_t)row * words;
    int* below = all_below + (size_t)row * words;
    if (n == left || left == 0) {
        if (STEP == 3) {
            if (tid == 0) p.count[blockIdx.x] = 0;
            for (int t = from + 64 * tid; t < to; t += 64 * 1024) bits[t / 64] = 0, below[t / 64] = 0;
        }
        return;
    }
    const int recent = first_recent(a.seen[r.b], a.keep_last);
    // a wave's tokens follow each other, 64 at a time
    constexpr int EACH = PART / 1024;
    float s[EACH];
    int ps[EACH];
    const int first = from + 64 * EACH * wave;
#pragma unroll
    for (int x = 0; x < EACH; ++x) {
        const int t = first + 64 * x + lane;
        s[x] = t < to ? r.score[t] : 0.f;
        ps[x] = t < to ? r.pos[t] : 0;
    }
    uint32_t border = 0;
    int want = left;
    if (STEP > 0) {
        if (STEP > 1) {
            const int2 st = p.state[2 * row + STEP - 2];
            border = (uint32_t)st.x;
            want = st.y;
        }
        // two bins a thread, thread 0 the highest
        constexpr int shift = STEP == 1 ? 21 : STEP == 2 ? 10 : 0;
        const int bin = BINS - 2 - 2 * tid;
        const int* h = p.hist + ((size_t)(STEP - 1) * (gridDim.x / p.parts) + row) * p.parts * BINS + bin;
        int own[2] = {0, 0};
        for (int q0 = 0; q0 < p.parts; q0 += 8) {
            int2 v[8];
#pragma unroll
            for (int y = 0; y < 8; ++y) v[y] = q0 + y < p.parts ? *reinterpret_cast<const int2*>(h + (size_t)(q0 + y) * BINS) : int2{0, 0};
#pragma unroll
            for (int y = 0; y < 8; ++y) own[0] += v[y].y, own[1] += v[y].x;
        }
        const int sum = own[0] + own[1], upto = wave_upto(sum);
        if (lane == 63) tally[wave] = upto;
        __syncthreads();
        int before = upto - sum;
        for (int w = 0; w < wave; ++w) before += tally[w];
#pragma unroll
        for (int x = 0; x < 2; ++x) {   // (one thread finds it: there are `want` keys or more)
            if (want > before && want <= before + own[x]) {
                found[0] = bin + 1 - x;
                found[1] = want - before;
            }
            before += own[x];
        }
        __syncthreads();
        border |= (uint32_t)found[0] << shift;
        want = found[1];
        if (STEP < 3 && part == 0 && tid == 0) p.state[2 * row + STEP - 1] = int2{(int)border, want};
    }
    if constexpr (STEP < 3) {
        constexpr int shift = STEP == 0 ? 21 : STEP == 1 ? 10 : 0;
        constexpr uint32_t mask = STEP == 2 ? 1023 : 2047, known = STEP == 0 ? 0u : ~0u << (STEP == 1 ? 21 : 10);
        for (int i = 4 * tid; i < BINS * LONG_COPIES; i += 4 * 1024) *reinterpret_cast<i4*>(hist + i) = i4{0, 0, 0, 0};
        __syncthreads();
#pragma unroll
        for (int x = 0; x < EACH; ++x) {
            const uint32_t k = key_of(s[x], ps[x], a.keep_first, recent);
            if (first + 64 * x + lane < to && ((k ^ border) & known) == 0) atomicAdd(&hist[((k >> shift) & mask) * LONG_COPIES + (lane & (LONG_COPIES - 1))], 1);
        }
        __syncthreads();
        const i4 lo = *reinterpret_cast<const i4*>(&hist[2 * tid * LONG_COPIES]), hi = *reinterpret_cast<const i4*>(&hist[(2 * tid + 1) * LONG_COPIES]);
        int* h = p.hist + ((size_t)STEP * gridDim.x + blockIdx.x) * BINS + 2 * tid;
        *reinterpret_cast<int2*>(h) = int2{lo.x + lo.y + lo.z + lo.w, hi.x + hi.y + hi.z + hi.w};
    } else {
        // equal keys at the border, counted off in slot order: those of the parts and waves before
        const int* h = p.hist + ((size_t)2 * gridDim.x + (size_t)row * p.parts) * BINS + (border & 1023);
        int rank = 0, mine = 0;
        for (int q = lane; q < part; q += 64) rank += h[(size_t)q * BINS];
        rank = wave_reduce(rank, Sum());
        uint32_t k[EACH];
#pragma unroll
        for (int x = 0; x < EACH; ++x) {
            k[x] = key_of(s[x], ps[x], a.keep_first, recent);
            mine += __popcll(__ballot(first + 64 * x + lane < to && k[x] == border));
        }
        __syncthreads();   // (tally may still be read)
        if (lane == 0) tally[wave] = mine;
        __syncthreads();
        for (int w = 0; w < wave; ++w) rank += tally[w];
        const uint64_t under = ((uint64_t)1 << lane) - 1;
        uint64_t word[EACH];
        int changed = 0;
#pragma unroll
        for (int x = 0; x < EACH; ++x) {
            const int t = first + 64 * x + lane;
            const uint64_t ties = __ballot(t < to && k[x] == border);
            const bool stays = k[x] > border || (k[x] == border && rank + __popcll(ties & under) < want);
            rank += __popcll(ties);
            word[x] = __ballot(t < to && (t < left) != stays);
            changed += __popcll(word[x]);
        }
        if (lane == 0) changes[wave] = changed;
        __syncthreads();
        int upto = 0;
        for (int w = 0; w < wave; ++w) upto += changes[w];
#pragma unroll
        for (int x = 0; x < EACH; ++x) {
            const int t = first + 64 * x;
            if (lane == 0 && t < to) {
                bits[t / 64] = word[x];
                below[t / 64] = upto;   // within the part
            }
            upto += __popcll(word[x]);
        }
        if (tid == 1023) p.count[blockIdx.x] = upto;
    }
}
__global__ __launch_bounds__(256) void evict_parts_below_kernel(Cache c, Evict a, Parts p, int* all_below, int words) {
    const int row = blockIdx.x / p.parts, part = blockIdx.x % p.parts, lane = threadIdx.x & 63;
    const int n = row_at(c, a, row).n, w = PART / 64 * part + threadIdx.x;
    int before = 0;
    for (int q = lane; q < part; q += 64) before += p.count[row * p.parts + q];
    before = wave_reduce(before, Sum());
    if (threadIdx.x < PART / 64 && 64 * (int64_t)w < n) all_below[(size_t)row * words + w] += before;
}

// The second launch: workgroup = TILE tokens behind a row's budget.
__global__ __launch_bounds__(256) void evict_move_kernel(Cache c, Evict a, const uint64_t* all_bits, const int* all_below, int words, int tiles) {
    __shared__ MoveLists lists;
    const int row = blockIdx.x / tiles, tile = blockIdx.x % tiles;
    const Row r = row_at(c, a, row);
    const int from = r.left + TILE * tile, to = min(r.n, from + TILE);
    if (from >= to || r.left == 0) return;
    // four at once: 512 rows with 90 moves a workgroup 18.7 us, 19.7 one by one (there are no registers for it beside a row's keys)
    make_moves<4>(c, r, Changes{all_bits + (size_t)row * words, all_below + (size_t)row * words}, from, to, lists);
}

struct Bits {
    uint64_t* bits;
    int* below;
    int words;
};
template <int J, bool VEC>
hipError_t select_rows(const Cache& c, const Evict& a, const Bits& x, int rows, int threads, hipStream_t s) {
    constexpr int HISTOGRAM = BINS * COPIES<J> * sizeof(int);
    const int lds = a.longest - a.budget > FEW ? HISTOGRAM : 0;   // (else no row of this call has more to go)
    const hipError_t e = allow_lds((const void*)evict_select_kernel<J, VEC>, lds, HISTOGRAM);
    if (e == hipSuccess) evict_select_kernel<J, VEC><<<rows, threads, lds, s>>>(c, a, x.bits, x.below, x.words);
    return e;
}
template <int J>
hipError_t select_with(const Cache& c, const Evict& a, const Bits& x, int rows, int threads, bool vec, hipStream_t s) {
    return vec ? select_rows<J, true>(c, a, x, rows, threads, s) : select_rows<J, false>(c, a, x, rows, threads, s);
}

bool second_launch(int longest, int budget) { return longest - budget > TILE || longest > MAX_IN_REGISTERS; }
int words_of(int longest) { return (longest + 63) / 64; }
int parts_of(int longest) { return (longest + PART - 1) / PART; }
// Workgroups that a call of rows longer than MAX_IN_REGISTERS has at most if several take a row (24 KiB of histograms each); with more rows, one a row keeps the CUs busy.  Several against one: 8 rows of
// 40000 -> 30000 44 us against 82, of 131001 -> 32768 88 against 213; 64 rows of 40000 -> 20000 192 against 212; 200 of 40000 -> 39000 132 against 138.
constexpr int MOST_PARTS = 1024;
size_t bits_bytes(int64_t rows, int longest) { return ((size_t)rows * words_of(longest) * (sizeof(uint64_t) + sizeof(int)) + 255) / 256 * 256; }

}  // namespace

size_t evict_workspace(int kv, int64_t seqs, int longest, int budget) {
    if (longest <= budget || !second_launch(longest, budget)) return 0;
    const int64_t rows = seqs * kv, most = rows > 0 ? MOST_PARTS / rows : 0;
    size_t parts = 0;
    // (as much as a shorter bound needs, which a short table can make of a longer one)
    if (longest > MAX_IN_REGISTERS && most >= parts_of(MAX_IN_REGISTERS + 1)) parts = (size_t)rows * std::min<int64_t>(parts_of(longest), most);
    return bits_bytes(rows, longest) + parts * (3 * BINS + 1) * sizeof(int) + (parts ? (size_t)rows * 2 * sizeof(int2) : 0);
}

hipError_t cache_evict(const Cache& c, const Evict& a, hipStream_t s) {
    const int rows = c.seqs * c.kv;
    Bits x{nullptr, nullptr, words_of(a.longest)};
    if (evict_workspace(c.kv, c.seqs, a.longest, a.budget) > 0) {
        x.bits = (uint64_t*)a.ws;
        x.below = (int*)(x.bits + (size_t)rows * x.words);
    }
    const auto on16 = [](const void* p) { return ((uintptr_t)p & 15u) == 0; };
    const bool vec = on16(a.score) && on16(a.pos) && on16(a.score_out) && on16(a.pos_out) && a.ld % 4 == 0 && a.ld_out % 4 == 0;
    // 4 tokens a thread up to 4096, then whole workgroups with 8, 16, 32.  Where histograms are taken, 512 threads at least: their bins are what takes the time (32 heads, 300 tokens -> 200:
    // 13.9 us with 128 threads, 10.0 with 256, 8.7 with 512, 8.9 with 1024; of 32 sequences 100 -> 50: 15.6, 12.5, 12.5, 20.6).
    const int least = a.longest - a.budget > FEW ? 512 : 128;
    hipError_t e = hipSuccess;
    if (a.longest <= 4096) e = select_with<1>(c, a, x, rows, std::max(least, (a.longest + 255) / 256 * 64), vec, s);
    else if (a.longest <= 8192) e = select_with<2>(c, a, x, rows, 1024, vec, s);
    else if (a.longest <= 16384) e = select_with<4>(c, a, x, rows, 1024, vec, s);
    else if (a.longest <= MAX_IN_REGISTERS) e = select_with<8>(c, a, x, rows, 1024, vec, s);
    else if (const int64_t grid = (int64_t)rows * parts_of(a.longest); x.bits && grid <= MOST_PARTS) {
        Parts p;
        p.parts = parts_of(a.longest);
        p.state = (int2*)((char*)a.ws + bits_bytes(rows, a.longest));
        p.hist = (int*)(p.state + 2 * rows);
        p.count = p.hist + 3 * grid * BINS;
        evict_part_kernel<0><<<(unsigned)grid, 1024, 0, s>>>(c, a, p, x.bits, x.below, x.words);
        evict_part_kernel<1><<<(unsigned)grid, 1024, 0, s>>>(c, a, p, x.bits, x.below, x.words);
        evict_part_kernel<2><<<(unsigned)grid, 1024, 0, s>>>(c, a, p, x.bits, x.below, x.words);
        evict_part_kernel<3><<<(unsigned)grid, 1024, 0, s>>>(c, a, p, x.bits, x.below, x.words);
        evict_parts_below_kernel<<<(unsigned)grid, 256, 0, s>>>(c, a, p, x.below, x.words);
    } else evict_select_long_kernel<<<rows, 1024, 0, s>>>(c, a, x.bits, x.below, x.words);
    if (e != hipSuccess) return e;
    if (x.bits) {
        const int tiles = (a.longest - a.budget + TILE - 1) / TILE;
        evict_move_kernel<<<(unsigned)((int64_t)rows * tiles), 256, 0, s>>>(c, a, x.bits, x.below, x.words, tiles);
    }
    return hipGetLastError();
}

}  // namespace qeft
