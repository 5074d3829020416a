// Element types of the caller's tensors: conversions, and groups of four elements as one access.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "legend.h"

namespace legend {

typedef __bf16 bf16_t;
typedef _Float16 half_t;

// Four consecutive elements at any address that is aligned to one element: global memory takes 8- and 16-byte accesses
// at such addresses.
template <class T>
struct Quad {
    typedef T type __attribute__((ext_vector_type(4), aligned(sizeof(T))));
};
template <bool STREAM = false, class T>
__device__ inline void store_quad(T* p, const float* in) {
    typename Quad<T>::type v;
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = (T)in[j];
    if (STREAM) __builtin_nontemporal_store(v, reinterpret_cast<typename Quad<T>::type*>(p));
    else *reinterpret_cast<typename Quad<T>::type*>(p) = v;
}

// one element of a tensor whose type is known at run time only
__device__ inline float load_as(const void* p, int64_t i, int type) {
    if (type == LEGEND_TYPE_FLOAT) return static_cast<const float*>(p)[i];
    if (type == LEGEND_TYPE_BFLOAT) return (float)static_cast<const bf16_t*>(p)[i];
    return (float)static_cast<const half_t*>(p)[i];
}
__device__ inline void store_as(void* p, int64_t i, int type, float v) {
    if (type == LEGEND_TYPE_FLOAT) static_cast<float*>(p)[i] = v;
    else if (type == LEGEND_TYPE_BFLOAT) static_cast<bf16_t*>(p)[i] = (bf16_t)v;
    else static_cast<half_t*>(p)[i] = (half_t)v;
}

}  // namespace legend
