// What becomes of a product's sums: the activations and the epilogue.
#pragma once

#include <type_traits>

#include "dd_elem.h"
#include "dd_layers.h"

namespace dd {

// --- activations --------------------------------------------------------------
// Phi(-|x|) and exp(-x^2 / 2), from Abramowitz and Stegun 7.1.26 (off by 1.5e-7
// at most).  Few instructions count: each takes 3.4 us of 16,384 x 2,048 -> 8,192, where
// the matrix units wait: GELU 510 us, SiLU 479, none 477.
__device__ __forceinline__ void normal(float x, float &below, float &e) {
    const float u = x * 0.84932180f;        // sqrt(log2(e) / 2)
    const float t = __builtin_amdgcn_rcpf(fmaf(0.27273748f, fabsf(u), 1.0f));       // 0.3275911 |x| / sqrt(2)
    e = __builtin_amdgcn_exp2f(-(u * u));
    below = t * fmaf(t, fmaf(t, fmaf(t, fmaf(t, 0.5f * 1.061405429f, 0.5f * -1.453152027f), 0.5f * 1.421413741f),
                             0.5f * -0.284496736f), 0.5f * 0.254829592f) * e;
}
__device__ __forceinline__ float sigmoid(float x) {
    return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(x * -1.44269504f));
}
template <int ACT>
__device__ __forceinline__ float act_of(float z) {
    if (ACT == DD_ACT_RELU) return z > 0.0f || z != z ? z : 0.0f;
    if (ACT == DD_ACT_GELU) {
        float below, e;
        normal(z, below, e);
        return fmaf(-fminf(fabsf(z), 1e30f), below, fmaxf(z, 0.0f));      // z Phi(z), also of infinities
    }
    if (ACT == DD_ACT_GELU_TANH) return z * sigmoid(z * fmaf(2.0f * 0.7978845608f * 0.044715f, z * z, 2.0f * 0.7978845608f));
    if (ACT == DD_ACT_SILU) return z * sigmoid(z);
    return z;
}
// z where its factor is 0 from far below 200 on: that of an infinity stays 0 (a NaN's factor is one itself)
__device__ __forceinline__ float reined(float z) { return __builtin_amdgcn_fmed3f(z, -200.0f, 200.0f); }
// The derivative; at infinities, which a z of 16 bits holds for sums beyond its range, its limit.  dx of 16,384 x 2,048 ->
// 8,192 bf16 through GELU 529 us, SiLU 512, none 458.
template <int ACT>
__device__ __forceinline__ float slope_of(float z) {
    if (ACT == DD_ACT_RELU) return z > 0.0f ? 1.0f : 0.0f;
    if (ACT == DD_ACT_GELU) {
        float below, e;
        normal(z, below, e);
        return fmaf(reined(z) * e, 0.3989422804f, z < 0.0f ? below : 1.0f - below);
    }
    if (ACT == DD_ACT_GELU_TANH) {
        const float x = z > 20.0f ? 20.0f : z < -20.0f ? -20.0f : z;     // (x^2 in range; the slope is 0 or 1 there)
        const float s = sigmoid(x * fmaf(2.0f * 0.7978845608f * 0.044715f, x * x, 2.0f * 0.7978845608f));
        return fmaf(x * s * (1.0f - s), fmaf(6.0f * 0.7978845608f * 0.044715f, x * x, 2.0f * 0.7978845608f), s);
    }
    if (ACT == DD_ACT_SILU) {
        const float s = sigmoid(z);
        return s * fmaf(reined(z), 1.0f - s, 1.0f);
    }
    return 1.0f;
}
// f<ACT>() of the eight values, chosen once for all
template <class F>
__device__ __forceinline__ void by_act(int32_t act, const F &f) {
    if (act == DD_ACT_RELU) f(std::integral_constant<int, DD_ACT_RELU>{});
    else if (act == DD_ACT_GELU) f(std::integral_constant<int, DD_ACT_GELU>{});
    else if (act == DD_ACT_GELU_TANH) f(std::integral_constant<int, DD_ACT_GELU_TANH>{});
    else if (act == DD_ACT_SILU) f(std::integral_constant<int, DD_ACT_SILU>{});
}

// What eight sums of a row need beside them, loaded ahead: the residual's or in_z's (an
// epilogue has one of them at most).
template <class T>
__device__ __forceinline__ void load_side(const Epilogue &e, int64_t i, int64_t j, int have, Pack<T, 8> &side) {
    const T *p = static_cast<const T *>(e.residual ? e.residual : e.in_z);
    if (p) side.load(p + i * e.side_stride + j, have);
}
template <class T>
__device__ __forceinline__ void load_bias(const Epilogue &e, int64_t j, int have, float (&x)[8]) {
    if (!e.bias) {
#pragma unroll
        for (int c = 0; c < 8; c++) x[c] = 0.0f;
    } else if (e.bias_type == DD_F32) {
        Pack<float, 8> b;
        b.load(static_cast<const float *>(e.bias) + j, have);
        b.to(x);
    } else {
        Pack<T, 8> b;
        b.load(static_cast<const T *>(e.bias) + j, have);
        b.to(x);
    }
}
// Eight sums of row i from column j on, of which `have` are in the output.
template <class T>
__device__ __forceinline__ void finish(const Epilogue &e, int64_t i, int64_t j, int have, float (&v)[8], const float (&bias)[8], const Pack<T, 8> &side) {
    Pack<T, 8> p;
    float x[8];
#pragma unroll
    for (int c = 0; c < 8; c++) v[c] += bias[c];
    if (e.z) {
        p.from(v);
        p.store(static_cast<T *>(e.z) + i * e.z_stride + j, have);
    }
    by_act(e.act, [&](auto act) {
#pragma unroll
        for (int c = 0; c < 8; c++) v[c] = act_of<decltype(act)::value>(v[c]);
    });
    if (e.residual) {
        side.to(x);
#pragma unroll
        for (int c = 0; c < 8; c++) v[c] += x[c];
    } else if (e.in_z) {
        side.to(x);
        by_act(e.in_act, [&](auto act) {
#pragma unroll
            for (int c = 0; c < 8; c++) v[c] *= slope_of<decltype(act)::value>(x[c]);
        });
    }
    p.from(v);
    p.store(static_cast<T *>(e.out) + i * e.out_stride + j, have);
}

}  // namespace dd
