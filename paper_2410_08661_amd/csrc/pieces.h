// Pieces of 1, 2, 4 or 8 fp16 values: one load, one store.
#pragma once

#include <hip/hip_runtime.h>
#include <hip/hip_fp16.h>
#include <stdint.h>

namespace qeft {

template <int VW> struct Piece { typedef uint32_t type __attribute__((ext_vector_type(VW / 2))); };
template <> struct Piece<2> { typedef uint32_t type; };
template <> struct Piece<1> { typedef uint16_t type; };

// one piece of VW values: read, write
template <int VW>
__device__ __forceinline__ void get(const __half* p, _Float16 (&x)[VW]) {
    const auto v = *reinterpret_cast<const typename Piece<VW>::type*>(p);
    __builtin_memcpy(x, &v, sizeof x);
}
template <int VW>
__device__ __forceinline__ void put(__half* p, const _Float16 (&x)[VW]) {
    typename Piece<VW>::type v;
    __builtin_memcpy(&v, x, sizeof x);
    *reinterpret_cast<typename Piece<VW>::type*>(p) = v;
}

}  // namespace qeft
