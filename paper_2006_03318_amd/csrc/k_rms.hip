// The residual's addition and the root-mean-square norm over rows, with an
// output in the inputs' type or in 8 bits, and its gradient.
//
//   s = x + residual,  rstd = 1 / sqrt(mean(s^2) + eps),  y = s * rstd * weight
//   8 bits: per group of columns, scale = max(|y|, 2^-100) / most, q = y / scale
//
//   xh = h * rstd,  c = mean(weight * dy * xh)
//   dx = (weight * dy - xh * c) * rstd + dh,  dweight = sum over rows of dy * xh
//
// Everything is computed in 32 bits and rounded once, where it is stored.
#include "dd_elem.h"
#include "dd_internal.h"

namespace dd {

namespace {

constexpr int kBlock = 256;

__device__ float block_sum(float x) {
    __shared__ float part[kBlock / 64];
    x = lanes_sum<64>(x);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = x;
    __syncthreads();
    float t = 0.0f;
#pragma unroll
    for (int w = 0; w < kBlock / 64; w++) t += part[w];
    __syncthreads();
    return t;
}
__device__ uint32_t block_max(uint32_t x) {
    __shared__ uint32_t part[kBlock / 64];
    x = lanes_max<64>(x);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = x;
    __syncthreads();
    uint32_t t = 0;
#pragma unroll
    for (int w = 0; w < kBlock / 64; w++) t = part[w] > t ? part[w] : t;
    __syncthreads();
    return t;
}

__device__ __forceinline__ float weight_at(const RmsArgs &a, int64_t c) {
    if (!a.weight) return 1.0f;
    if (a.weight_type == DD_F32) return global(static_cast<const float *>(a.weight))[c];
    if (a.weight_type == DD_BF16) return (float)global(static_cast<const bf16_t *>(a.weight))[c];
    return (float)global(static_cast<const f16_t *>(a.weight))[c];
}

__device__ __forceinline__ float most_of(int32_t out_type) { return out_type == DD_E4M3 ? 448.0f : 127.0f; }

// The largest |y| is taken over its bits: those of a NaN are above infinity's,
// so a group that holds one has a NaN for its scale.
__device__ __forceinline__ float scale_of(uint32_t amax, float most) {
    const float a = __uint_as_float(amax);
    return (a > 0x1p-100f || a != a ? a : 0x1p-100f) / most;
}

__device__ __forceinline__ uint8_t to_8_bits(float x, int32_t out_type) {
    if (out_type == DD_E4M3) return (uint8_t)__builtin_amdgcn_cvt_pk_fp8_f32(x, x, 0, false);
    const float r = rintf(x);
    return (uint8_t)(int8_t)(r < -127.0f ? -127 : r > 127.0f ? 127 : r != r ? 0 : (int)r);
}

// One workgroup per row, any width: the row is read once for each of its sums.
template <class T>
__global__ void __launch_bounds__(kBlock) k_rms_loop(RmsArgs a) {
    const int64_t row = blockIdx.x + (int64_t)blockIdx.y * gridDim.x;
    if (row >= a.rows) return;
    const T *x = static_cast<const T *>(a.x) + row * a.x_stride;
    const T *r = a.residual ? static_cast<const T *>(a.residual) + row * a.residual_stride : nullptr;
    T *h = a.h ? static_cast<T *>(a.h) + row * a.h_stride : nullptr;
    auto at = [&](int64_t c) { return (float)global(x)[c] + (r ? (float)global(r)[c] : 0.0f); };
    float q = 0.0f;
    for (int64_t c = threadIdx.x; c < a.cols; c += kBlock) {
        const float s = at(c);
        q = fmaf(s, s, q);
    }
    const float rstd = 1.0f / sqrtf(block_sum(q) / (float)a.cols + a.eps);
    if (a.rstd && threadIdx.x == 0) a.rstd[row] = rstd;
    if (a.out_type == DD_E4M3 || a.out_type == DD_I8) {
        uint8_t *out = static_cast<uint8_t *>(a.out) + row * a.out_stride;
        const int64_t group = a.group ? a.group : a.cols;
        const int64_t groups = (a.cols + group - 1) / group;
        for (int64_t k = 0; k < groups; k++) {
            const int64_t c0 = k * group, c1 = c0 + group < a.cols ? c0 + group : a.cols;
            uint32_t m = 0;
            for (int64_t c = c0 + threadIdx.x; c < c1; c += kBlock) {
                const uint32_t b = __float_as_uint(at(c) * rstd * weight_at(a, c)) & 0x7fffffffu;
                m = b > m ? b : m;
            }
            const float scale = scale_of(block_max(m), most_of(a.out_type));
            const float inv = 1.0f / scale;
            if (threadIdx.x == 0) a.scales[row * groups + k] = scale;
            for (int64_t c = c0 + threadIdx.x; c < c1; c += kBlock) {
                const float s = at(c);
                if (h) global(h)[c] = (T)s;
                out[c] = to_8_bits(s * rstd * weight_at(a, c) * inv, a.out_type);
            }
        }
        return;
    }
    T *out = static_cast<T *>(a.out) + row * a.out_stride;
    for (int64_t c = threadIdx.x; c < a.cols; c += kBlock) {
        const float s = at(c);
        if (h) global(h)[c] = (T)s;
        global(out)[c] = (T)(s * rstd * weight_at(a, c));
    }
}

__device__ __forceinline__ float weight_at(const RmsGradArgs &a, int64_t c) {
    if (!a.weight) return 1.0f;
    if (a.weight_type == DD_F32) return global(static_cast<const float *>(a.weight))[c];
    if (a.weight_type == DD_BF16) return (float)global(static_cast<const bf16_t *>(a.weight))[c];
    return (float)global(static_cast<const f16_t *>(a.weight))[c];
}

template <class T>
__global__ void __launch_bounds__(kBlock) k_rms_dx_loop(RmsGradArgs a) {
    const int64_t row = blockIdx.x + (int64_t)blockIdx.y * gridDim.x;
    if (row >= a.rows) return;
    const T *dy = static_cast<const T *>(a.dy) + row * a.dy_stride;
    const T *h = static_cast<const T *>(a.h) + row * a.h_stride;
    const T *dh = a.dh ? static_cast<const T *>(a.dh) + row * a.dh_stride : nullptr;
    T *dx = static_cast<T *>(a.dx) + row * a.dx_stride;
    const float rstd = a.rstd[row];
    float q = 0.0f;
    for (int64_t c = threadIdx.x; c < a.cols; c += kBlock)
        q = fmaf((float)global(dy)[c] * weight_at(a, c), (float)global(h)[c] * rstd, q);
    const float m = block_sum(q) / (float)a.cols;
    for (int64_t c = threadIdx.x; c < a.cols; c += kBlock) {
        const float g = (float)global(dy)[c] * weight_at(a, c) - (float)global(h)[c] * rstd * m;
        global(dx)[c] = (T)(g * rstd + (dh ? (float)global(dh)[c] : 0.0f));
    }
}

// Partial sums of dweight: workgroup (i, j) has 64 columns and the j-th of
// gridDim.y runs of rows.
template <class T>
__global__ void __launch_bounds__(kBlock) k_rms_dw_loop(RmsGradArgs a, float *part) {
    __shared__ float lds[kBlock];
    const int64_t c = (int64_t)blockIdx.x * 64 + (threadIdx.x & 63);
    const int64_t run = (a.rows + gridDim.y - 1) / gridDim.y;
    const int64_t r0 = blockIdx.y * run, r1 = r0 + run < a.rows ? r0 + run : a.rows;
    float s = 0.0f;
    if (c < a.cols)
        for (int64_t r = r0 + (threadIdx.x >> 6); r < r1; r += kBlock / 64)
            s = fmaf((float)global(static_cast<const T *>(a.dy))[r * a.dy_stride + c],
                     (float)global(static_cast<const T *>(a.h))[r * a.h_stride + c] * a.rstd[r], s);
    lds[threadIdx.x] = s;
    __syncthreads();
    if (threadIdx.x < 64 && c < a.cols) {
        for (int w = 1; w < kBlock / 64; w++) s += lds[threadIdx.x + 64 * w];
        part[blockIdx.y * a.cols + c] = s;
    }
}

__global__ void __launch_bounds__(kBlock) k_rms_dw_join(RmsGradArgs a, const float *part, int n) {
    const int64_t c = (int64_t)blockIdx.x * kBlock + threadIdx.x;
    if (c >= a.cols) return;
    float s = 0.0f;
    for (int i = 0; i < n; i++) s += part[i * a.cols + c];
    if (a.weight_type == DD_F32) static_cast<float *>(a.dw)[c] = s;
    else if (a.weight_type == DD_BF16) static_cast<bf16_t *>(a.dw)[c] = (bf16_t)s;
    else static_cast<f16_t *>(a.dw)[c] = (f16_t)s;
}

dim3 grid_of_rows(int64_t rows) {
    const int64_t x = rows < (1 << 20) ? rows : (1 << 20);
    return dim3((unsigned)x, (unsigned)((rows + x - 1) / x));
}

int dw_runs(int64_t rows) {
    const int64_t r = (rows + 255) / 256;
    return r < 1 ? 1 : r > kRmsParts ? kRmsParts : (int)r;
}

}  // namespace

size_t rms_grad_work(int64_t rows, int64_t cols) { return (size_t)dw_runs(rows) * (size_t)cols * sizeof(float); }

hipError_t launch_rms_norm(const RmsArgs &a, hipStream_t s) {
    const dim3 g = grid_of_rows(a.rows);
    if (a.type == DD_F32) k_rms_loop<float><<<g, kBlock, 0, s>>>(a);
    else if (a.type == DD_BF16) k_rms_loop<bf16_t><<<g, kBlock, 0, s>>>(a);
    else k_rms_loop<f16_t><<<g, kBlock, 0, s>>>(a);
    return hipGetLastError();
}

template <class T>
static void rms_grad(const RmsGradArgs &a, float *work, hipStream_t s) {
    if (a.dw) {       // first: dx may overwrite what it reads
        const int n = dw_runs(a.rows);
        k_rms_dw_loop<T><<<dim3((unsigned)((a.cols + 63) / 64), n), kBlock, 0, s>>>(a, work);
        k_rms_dw_join<<<(unsigned)((a.cols + kBlock - 1) / kBlock), kBlock, 0, s>>>(a, work, n);
    }
    if (a.rows > 0) k_rms_dx_loop<T><<<grid_of_rows(a.rows), kBlock, 0, s>>>(a);
}

hipError_t launch_rms_norm_grad(const RmsGradArgs &a, float *work, hipStream_t s) {
    if (a.type == DD_F32) rms_grad<float>(a, work, s);
    else if (a.type == DD_BF16) rms_grad<bf16_t>(a, work, s);
    else rms_grad<f16_t>(a, work, s);
    return hipGetLastError();
}

}  // namespace dd
