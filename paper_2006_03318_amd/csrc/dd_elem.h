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

// N consecutive elements of E.  The address is aligned to E and no more
// (tensors start anywhere in a buffer, rows have any stride): CDNA4 loads 16
// bytes from any address.  Loading and converting are separate steps, so that
// a kernel has all its loads under way before it waits for the first.
template <class E, int N>
struct Pack {
    typedef E vec __attribute__((ext_vector_type(N)));
    typedef float fvec __attribute__((ext_vector_type(N)));
    typedef vec __attribute__((aligned(alignof(E)))) any;
    vec v;
    __device__ __forceinline__ void load(const E *p) { v = *(gptr<const any>)(p); }
    __device__ __forceinline__ void store(E *p) const { *(gptr<any>)(p) = v; }
    // the first `have` of them, any number; the others read as zero, and are not written
    __device__ __forceinline__ void load(const E *p, int have) {
        if (have >= N) {
            load(p);
        } else {
#pragma unroll
            for (int i = 0; i < N; i++) v[i] = i < have ? global(p)[i] : (E)0.0f;
        }
    }
    __device__ __forceinline__ void store(E *p, int have) const {
        if (have >= N) {
            store(p);
        } else {
#pragma unroll
            for (int i = 0; i < N; i++)
                if (i < have) global(p)[i] = v[i];
        }
    }
    __device__ __forceinline__ void to(float (&x)[N]) const {
#pragma unroll
        for (int i = 0; i < N; i++) x[i] = (float)v[i];
    }
    // What was computed from the pack before is not kept beyond this point: it
    // is cheaper to convert again than to hold twice the registers.
    __device__ __forceinline__ void forget() {
        typedef uint32_t words __attribute__((ext_vector_type(N * sizeof(E) / 4)));
        words w = __builtin_bit_cast(words, v);
#pragma unroll
        for (unsigned i = 0; i < N * sizeof(E) / 4; i++) {
            uint32_t x = w[i];
            asm volatile("" : "+v"(x));
            w[i] = x;
        }
        v = __builtin_bit_cast(vec, w);
    }
    // (rounds to nearest even)
    __device__ __forceinline__ void from(const float (&x)[N]) {
        fvec f;
#pragma unroll
        for (int i = 0; i < N; i++) f[i] = x[i];
        v = __builtin_convertvector(f, vec);
    }
};

// Sums and maxima over aligned groups of W lanes (4, 8, 16 or 64); every lane
// has the result, the same bits in each.  Steps inside 16 lanes are DPP moves
// (once the four lanes of a quad agree, mirroring eight lanes pairs the quads;
// so on for sixteen), the four sixteens are read as scalars: no trips to LDS.
template <int CTRL>
__device__ __forceinline__ uint32_t dpp(uint32_t x) {
    return (uint32_t)__builtin_amdgcn_mov_dpp((int)x, CTRL, 0xf, 0xf, true);
}
constexpr int kDppXor1 = 0xb1, kDppXor2 = 0x4e, kDppHalfMirror = 0x141, kDppMirror = 0x140;

template <int W, class T, class F>
__device__ __forceinline__ T lanes_fold(T x, const F &f) {
    static_assert(sizeof(T) == 4 && (W == 4 || W == 8 || W == 16 || W == 64), "lanes");
    auto from = [](uint32_t b) { T y; __builtin_memcpy(&y, &b, 4); return y; };
    auto bits = [](T y) { uint32_t b; __builtin_memcpy(&b, &y, 4); return b; };
    x = f(x, from(dpp<kDppXor1>(bits(x))));
    x = f(x, from(dpp<kDppXor2>(bits(x))));
    if (W >= 8) x = f(x, from(dpp<kDppHalfMirror>(bits(x))));
    if (W >= 16) x = f(x, from(dpp<kDppMirror>(bits(x))));
    if (W == 64) {
        const T a = from(__builtin_amdgcn_readlane((int)bits(x), 0)), b = from(__builtin_amdgcn_readlane((int)bits(x), 16));
        const T c = from(__builtin_amdgcn_readlane((int)bits(x), 32)), d = from(__builtin_amdgcn_readlane((int)bits(x), 48));
        x = f(f(a, b), f(c, d));
    }
    return x;
}
template <int W>
__device__ __forceinline__ float lanes_sum(float x) {
    return lanes_fold<W>(x, [](float a, float b) { return a + b; });
}
template <int W>
__device__ __forceinline__ uint32_t lanes_max(uint32_t x) {
    return lanes_fold<W>(x, [](uint32_t a, uint32_t b) { return a > b ? a : b; });
}
__device__ __forceinline__ double wave_sum(double x) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) x += __shfl_xor(x, o, 64);
    return x;
}

__host__ __device__ inline int32_t elem_size(int32_t type) {
    return type == DD_F32 ? 4 : type == DD_BF16 || type == DD_F16 ? 2 : type == DD_E4M3 || type == DD_I8 ? 1 : 0;
}

}  // namespace dd
