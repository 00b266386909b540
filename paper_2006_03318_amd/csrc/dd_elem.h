// Elements of training tensors: types, loads and stores of several at a time,
// rounding, and reductions over a wave or a workgroup (wave64 / CDNA4).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "dd.h"

namespace dd {

typedef __bf16 bf16_t;
typedef _Float16 f16_t;

// Global memory, said so: an address read from a table would otherwise be
// taken for any address space, whose loads also wait on LDS.
template <class T>
using gptr = __attribute__((address_space(1))) T *;
template <class T>
__device__ __forceinline__ gptr<T> global(T *p) {
    return (gptr<T>)(p);
}

// N consecutive elements of E as floats.  The address is aligned to E and no
// more (tensors start anywhere in a buffer, rows have any stride): CDNA4 loads
// 16 bytes from any address.
template <class E, int N>
struct Pack {
    typedef E vec __attribute__((ext_vector_type(N)));
    typedef float fvec __attribute__((ext_vector_type(N)));
};
template <class E, int N>
__device__ __forceinline__ void load_n(const E *p, float (&x)[N]) {
    typedef typename Pack<E, N>::vec V;
    typedef V __attribute__((aligned(alignof(E)))) U;
    const V v = *(gptr<const U>)(p);
#pragma unroll
    for (int i = 0; i < N; i++) x[i] = (float)v[i];
}
// (round to nearest even)
template <class E, int N>
__device__ __forceinline__ void store_n(E *p, const float (&x)[N]) {
    typedef typename Pack<E, N>::vec V;
    typedef V __attribute__((aligned(alignof(E)))) U;
    typename Pack<E, N>::fvec f;
#pragma unroll
    for (int i = 0; i < N; i++) f[i] = x[i];
    *(gptr<U>)(p) = __builtin_convertvector(f, V);
}
// the first `have` (0 to N) of them; the rest reads as zero and is not written
template <class E, int N>
__device__ __forceinline__ void load_some(const E *p, float (&x)[N], int have) {
#pragma unroll
    for (int i = 0; i < N; i++) x[i] = i < have ? (float)global(p)[i] : 0.0f;
}
template <class E, int N>
__device__ __forceinline__ void store_some(E *p, const float (&x)[N], int have) {
#pragma unroll
    for (int i = 0; i < N; i++)
        if (i < have) global(p)[i] = (E)x[i];
}

template <class T>
__device__ __forceinline__ T lane_xor(T x, int d) {
    return __shfl_xor(x, d, 64);
}
// over aligned groups of W lanes (a power of two); every lane has the result,
// the same bits in each (the order of the sums does not depend on the lane)
template <int W, class T>
__device__ __forceinline__ T lanes_sum(T x) {
#pragma unroll
    for (int o = W / 2; o > 0; o >>= 1) x += lane_xor(x, o);
    return x;
}
template <int W>
__device__ __forceinline__ uint32_t lanes_max(uint32_t x) {
#pragma unroll
    for (int o = W / 2; o > 0; o >>= 1) {
        const uint32_t y = lane_xor(x, o);
        x = y > x ? y : x;
    }
    return x;
}

inline int32_t elem_size(int32_t type) {
    return type == DD_F32 ? 4 : type == DD_BF16 || type == DD_F16 ? 2 : type == DD_E4M3 || type == DD_I8 ? 1 : 0;
}

}  // namespace dd
