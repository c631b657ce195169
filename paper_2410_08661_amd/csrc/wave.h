// Sums and extremes over the lanes of a wave and the waves of a workgroup, the same in every lane that asks.
// Within rows of 16 lanes they go by data-parallel moves (a rotation by 8, 4, 2, 1 and an operation each, no trip through LDS), then over rows and halves by
// the lane swaps of gfx950; a workgroup's waves leave one value each in LDS, which every wave reads with one load, a lane per wave, and reduces the same
// way.  (A loop over 16 waves' values waits for LDS sixteen times: 0.7 us.)
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace qeft {

template <int N>   // the value of the lane N places on in the row of 16, around its end
__device__ __forceinline__ uint32_t rotated(uint32_t x) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x120 + N, 0xf, 0xf, false); }

template <int N, class T>
__device__ __forceinline__ T row_rotated(T x) {
    if constexpr (sizeof(T) == 8) {
        const uint64_t u = __builtin_bit_cast(uint64_t, x);
        return __builtin_bit_cast(T, (uint64_t)rotated<N>((uint32_t)(u >> 32)) << 32 | rotated<N>((uint32_t)u));
    } else {
        return __builtin_bit_cast(T, rotated<N>(__builtin_bit_cast(uint32_t, x)));
    }
}
// x of the other half of the wave (HALF), or of the other row of the same half: both as the swap returns them, in one order for all lanes
template <bool HALF, class T, class Op>
__device__ __forceinline__ T across(T x, const Op& op) {
    auto swap = [](uint32_t v) {
        if constexpr (HALF) return __builtin_amdgcn_permlane32_swap(v, v, false, false);
        else return __builtin_amdgcn_permlane16_swap(v, v, false, false);
    };
    if constexpr (sizeof(T) == 8) {
        const uint64_t u = __builtin_bit_cast(uint64_t, x);
        const auto hi = swap((uint32_t)(u >> 32)), lo = swap((uint32_t)u);
        return op(__builtin_bit_cast(T, (uint64_t)hi[0] << 32 | lo[0]), __builtin_bit_cast(T, (uint64_t)hi[1] << 32 | lo[1]));
    } else {
        const auto r = swap(__builtin_bit_cast(uint32_t, x));
        return op(__builtin_bit_cast(T, (uint32_t)r[0]), __builtin_bit_cast(T, (uint32_t)r[1]));
    }
}
template <class T, class Op>
__device__ __forceinline__ T row_reduce(T x, const Op& op) {   // over 16 lanes
    x = op(x, row_rotated<8>(x));
    x = op(x, row_rotated<4>(x));
    x = op(x, row_rotated<2>(x));
    return op(x, row_rotated<1>(x));
}
template <class T, class Op>
__device__ __forceinline__ T wave_reduce(T x, const Op& op) { return across<true>(across<false>(row_reduce(x, op), op), op); }

struct Sum {
    template <class T> __device__ __forceinline__ T operator()(T a, T b) const { return a + b; }
};
struct Least {
    template <class T> __device__ __forceinline__ T operator()(T a, T b) const { return b < a ? b : a; }
};

// Over waves first .. first + waves - 1 of a workgroup (16 at most) from the values they left in slots[]; none: what an absent wave counts for.  The caller has a
// barrier between the writes and this, and one between this and the next writes.
template <class T, class Op>
__device__ __forceinline__ T waves_reduce(const T* slots, int first, int waves, T none, const Op& op) {
    const int w = threadIdx.x & 15;
    const T x = slots[(first + w) & 15];
    return row_reduce(w < waves ? x : none, op);
}

// Sum over the lanes up to and with this one: within rows by shifts, then the last lane of the row before (rows 1 and 3) and of the first half.
__device__ __forceinline__ int wave_upto(int x) {
    x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);   // row_shr 1, 2, 4, 8; lanes without a source add 0
    x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);   // row_bcast 15 into rows 1 and 3
    x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);   // row_bcast 31 into rows 2 and 3
    return x;
}

}  // namespace qeft
