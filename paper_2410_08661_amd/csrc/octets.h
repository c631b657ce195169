// Rows of fp16 or fp32 values by pieces of eight: loads and stores of 16 or 32 bytes a lane, the last piece of a row value by value.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace qeft {

typedef uint32_t u4 __attribute__((ext_vector_type(4)));
typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef float f4 __attribute__((ext_vector_type(4)));

// A row's address, the same in all lanes: kept from the optimiser, which would otherwise add a lane's offset to every array's base outside the loop over
// the rows and hold those sums, two registers each (the gradient has eight arrays), instead of adding in the load.
__device__ __forceinline__ const char* row_of(const void* p, int64_t row, int64_t ld, bool f32) {
    const char* r = (const char*)p + row * ld * (f32 ? 4 : 2);
    asm volatile("" : "+s"(r));
    return r;
}
__device__ __forceinline__ char* row_of(void* p, int64_t row, int64_t ld, bool f32) { return const_cast<char*>(row_of((const void*)p, row, ld, f32)); }

// One load or store; `once`: of data that the caches need not keep
template <class T>
__device__ __forceinline__ T fetch(const char* p, bool once) { return once ? __builtin_nontemporal_load(reinterpret_cast<const T*>(p)) : *reinterpret_cast<const T*>(p); }
template <class T>
__device__ __forceinline__ void place(char* p, T x, bool once) {
    if (once) __builtin_nontemporal_store(x, reinterpret_cast<T*>(p));
    else *reinterpret_cast<T*>(p) = x;
}

// Eight values of a row as loaded.  left: how many of them exist (none from 0 down); a row's last octet may be partial, and is read value by value, the last one
// first.  What does not exist is 0, or the word `none`.
template <bool F32> struct Raw;
template <> struct Raw<false> {
    static constexpr uint32_t NEG_INF = 0xfc00fc00u;   // (a word of values)
    u4 v;
    __device__ __forceinline__ void load(const void* row, uint32_t at, int left, uint32_t none = 0, bool once = false) {
        const char* p = (const char*)row + 2 * at;
        if (left >= 8) {
            v = fetch<u4>(p, once);
            return;
        }
        fill(none);
#pragma unroll 1
        for (int e = left - 1; e >= 0; --e) {
            const uint32_t x = *reinterpret_cast<const uint16_t*>(p + 2 * e);
            v = u4{v.x << 16 | x, v.y << 16 | v.x >> 16, v.z << 16 | v.y >> 16, v.w << 16 | v.z >> 16};
        }
    }
    __device__ __forceinline__ float operator[](int e) const { return (float)__builtin_bit_cast(h8, v)[e]; }
    __device__ __forceinline__ void fill(uint32_t word) { v = u4{word, word, word, word}; }
    __device__ __forceinline__ void clear() { fill(0); }
    // Eight values stay four registers: without this the compiler converts once and keeps eight (across a loop for a row of weights).
    __device__ __forceinline__ void pin() { asm volatile("" : "+v"(v)); }
    __device__ __forceinline__ void hold() { pin(); }   // (the same for fp32, where nothing is converted but what is made of the values could be kept as well)
};
template <> struct Raw<true> {
    static constexpr uint32_t NEG_INF = 0xff800000u;
    f4 a, b;
    __device__ __forceinline__ void load(const void* row, uint32_t at, int left, uint32_t none = 0, bool once = false) {
        const char* p = (const char*)row + 4 * at;
        if (left >= 8) {
            a = fetch<f4>(p, once);
            b = fetch<f4>(p + 16, once);
            return;
        }
        fill(none);
#pragma unroll 1
        for (int e = left - 1; e >= 0; --e) {
            b = f4{a.w, b.x, b.y, b.z};
            a = f4{*reinterpret_cast<const float*>(p + 4 * e), a.x, a.y, a.z};
        }
    }
    __device__ __forceinline__ float operator[](int e) const { return e < 4 ? a[e & 3] : b[e & 3]; }
    __device__ __forceinline__ void fill(uint32_t word) {
        const float x = __builtin_bit_cast(float, word);
        a = b = f4{x, x, x, x};
    }
    __device__ __forceinline__ void clear() { fill(0); }
    __device__ __forceinline__ void pin() {}
    __device__ __forceinline__ void hold() { asm volatile("" : "+v"(a), "+v"(b)); }
};
typedef Raw<false> Half8;

__device__ __forceinline__ void store_halves(void* row, uint32_t at, int left, u4 v, bool once = false) {
    char* p = (char*)row + 2 * at;
    if (left >= 8) {
        place(p, v, once);
        return;
    }
#pragma unroll 1
    for (int e = 0; e < left; ++e) {
        *reinterpret_cast<uint16_t*>(p + 2 * e) = (uint16_t)v.x;
        v = u4{v.x >> 16 | v.y << 16, v.y >> 16 | v.z << 16, v.z >> 16 | v.w << 16, v.w >> 16};
    }
}
// x goes to the row, rounded to its type (which x then is too)
template <bool F32>
__device__ __forceinline__ void store(void* row, uint32_t at, int left, float (&x)[8], bool once = false) {
    if (F32) {
        char* p = (char*)row + 4 * at;
        f4 a = {x[0], x[1], x[2], x[3]}, b = {x[4], x[5], x[6], x[7]};
        if (left >= 8) {
            place(p, a, once);
            place(p + 16, b, once);
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
    store_halves(row, at, left, __builtin_bit_cast(u4, h), once);
}

}  // namespace qeft
