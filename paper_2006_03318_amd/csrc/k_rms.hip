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
#include "dd_train.h"

namespace dd {

namespace {

__device__ __forceinline__ float most_of(int32_t out_type) { return out_type == DD_E4M3 ? 448.0f : 127.0f; }

// The largest |y| is taken over its bits: those of a NaN are above infinity's,
// so a group that holds one has a NaN for its scale.
__device__ __forceinline__ float scale_of(uint32_t amax, float most) {
    const float a = __uint_as_float(amax);
    return (a > 0x1p-100f || a != a ? a : 0x1p-100f) / most;
}

// x / scale rounded once, for many x: what the division gives, bit for bit.  The
// product in 64 bits is off by 2^-52 of the quotient, and a quotient of two
// numbers of 24 bits lies at least 2^-49 of it from any tie of 32 bits: a tie is
// an odd M of 25 bits, and Y 2^k - S M of whole numbers is not 0 (M would divide
// Y, which is smaller).  A product with a rounded 32-bit 1 / scale sends values
// near a tie of 8 bits to the other neighbour.  8,192 x 4,096 bf16 to e4m3 by
// 128 columns: 50.0 us, 51.2 with a division for each value (48.2 with the product in
// 32 bits).
struct Quotient {
    const double inv;
    __device__ __forceinline__ explicit Quotient(float scale) : inv(1.0 / (double)scale) {}
    __device__ __forceinline__ float operator()(float x) const { return (float)((double)x * inv); }
};

__device__ __forceinline__ uint8_t to_i8(float x) {
    const float r = rintf(x);
    return (uint8_t)(int8_t)(r < -127.0f ? -127 : r > 127.0f ? 127 : r != r ? 0 : (int)r);
}

// --- rows held in registers -------------------------------------------------
// A row is taken by LANES lanes, each with NV packs of 8 consecutive columns
// (lane l has packs l, l + LANES, ...), so x and residual are read once and
// a group of 32, 64 or 128 columns is 4, 8 or 16 neighbouring lanes.  Up to 64
// lanes need no barrier; several waves exchange one number through LDS.
//
// Bound: HBM, at the rate of a large copy (4.9 TB/s) or above it; a few rows,
// the launch.  8,192 x 4,096 bf16 with a residual to e4m3 by 128 columns 50 us
// (4.7 TB/s), 65,536 x 2,048 bf16 184 us (5.8), 4,099 x 1,237 f32 16.5 us
// (4.9), 4 x 4,096 4.3 us.
template <int LANES>
struct RowSum {
    static constexpr int kWaves = LANES / 64 > 1 ? LANES / 64 : 1;
    // slot: another one for each exchange of a row, by turns between rows
    static __device__ __forceinline__ float sum(float x, float *slot) {
        x = lanes_sum<(LANES < 64 ? LANES : 64)>(x);
        if (LANES <= 64) return x;
        if ((threadIdx.x & 63) == 0) slot[threadIdx.x >> 6] = x;
        __syncthreads();
        float t = 0.0f;
#pragma unroll
        for (int w = 0; w < kWaves; w++) t += slot[w];
        return t;
    }
    static __device__ __forceinline__ uint32_t max(uint32_t x, float *slot) {
        x = lanes_max<(LANES < 64 ? LANES : 64)>(x);
        if (LANES <= 64) return x;
        if ((threadIdx.x & 63) == 0) slot[threadIdx.x >> 6] = __uint_as_float(x);
        __syncthreads();
        uint32_t t = 0;
#pragma unroll
        for (int w = 0; w < kWaves; w++) {
            const uint32_t y = __float_as_uint(slot[w]);
            t = y > t ? y : t;
        }
        return t;
    }
};

__device__ __forceinline__ void store_pack_8(uint8_t *p, const float (&x)[8], int have, int32_t out_type) {
    typedef uint32_t u2 __attribute__((ext_vector_type(2)));
    typedef u2 __attribute__((aligned(1))) U;
    u2 b;
    if (out_type == DD_E4M3) {
#pragma unroll
        for (int i = 0; i < 2; i++) {
            int w = __builtin_amdgcn_cvt_pk_fp8_f32(x[4 * i], x[4 * i + 1], 0, false);
            b[i] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x[4 * i + 2], x[4 * i + 3], w, true);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 2; i++)
            b[i] = (uint32_t)to_i8(x[4 * i]) | (uint32_t)to_i8(x[4 * i + 1]) << 8 | (uint32_t)to_i8(x[4 * i + 2]) << 16 |
                   (uint32_t)to_i8(x[4 * i + 3]) << 24;
    }
    if (have >= 8) {
        *(gptr<U>)(p) = b;
    } else {
        for (int i = 0; i < have; i++) global(p)[i] = (uint8_t)(b[i >> 2] >> (8 * (i & 3)));
    }
}

// bits of the largest magnitude
__device__ __forceinline__ uint32_t largest(const float (&v)[8]) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; i++) {
        const uint32_t b = __float_as_uint(v[i]) & 0x7fffffffu;
        m = b > m ? b : m;
    }
    return m;
}

// eight weights, held as they were loaded
template <class T>
struct Weights {
    Pack<float, 8> f;
    Pack<T, 8> t;
    __device__ __forceinline__ void load(const void *w, int32_t type, int64_t c, int have) {
        if (!w) return;
        if (type == DD_F32) f.load(static_cast<const float *>(w) + c, have);
        else t.load(static_cast<const T *>(w) + c, have);
    }
    __device__ __forceinline__ void to(const void *w, int32_t type, float (&x)[8]) const {
        if (!w) {
#pragma unroll
            for (int i = 0; i < 8; i++) x[i] = 1.0f;
        } else if (type == DD_F32) {
            f.to(x);
        } else {
            t.to(x);
        }
    }
};

// (rows that share a workgroup do not share a wave, and need no barrier)
constexpr int row_threads(int lanes) { return lanes <= 64 ? 256 : lanes; }

// (the same for a whole wave, and said so, where a row has one)
template <int LANES>
__device__ __forceinline__ int row_of_thread() {
    const int r = threadIdx.x / LANES;
    return LANES >= 64 ? __builtin_amdgcn_readfirstlane(r) : r;
}

template <class T, int LANES, int NV>
__global__ void __launch_bounds__(row_threads(LANES)) k_rms_row(RmsArgs a) {
    constexpr int kThreads = row_threads(LANES), kRows = kThreads / LANES;
    __shared__ float slots[4][16];
    const int lane = threadIdx.x % LANES;
    const int cols = (int)a.cols;
    const bool narrow = a.out_type == DD_E4M3 || a.out_type == DD_I8;
    const float most = most_of(a.out_type);
    int turn = 0;
    for (int64_t row = (int64_t)blockIdx.x * kRows + row_of_thread<LANES>(); row < a.rows;
         row += (int64_t)gridDim.x * kRows, turn ^= 1) {
        const T *x = static_cast<const T *>(a.x) + row * a.x_stride;
        const T *r = static_cast<const T *>(a.residual) + row * a.residual_stride;
        float v[NV][8];
        {
            Pack<T, 8> px[NV], pr[NV];
#pragma unroll
            for (int k = 0; k < NV; k++) px[k].load(x + 8 * (lane + k * LANES), cols - 8 * (lane + k * LANES));
            if (a.residual) {
#pragma unroll
                for (int k = 0; k < NV; k++) pr[k].load(r + 8 * (lane + k * LANES), cols - 8 * (lane + k * LANES));
            }
#pragma unroll
            for (int k = 0; k < NV; k++) px[k].to(v[k]);
            if (a.residual) {
#pragma unroll
                for (int k = 0; k < NV; k++) {
                    float y[8];
                    pr[k].to(y);
#pragma unroll
                    for (int i = 0; i < 8; i++) v[k][i] += y[i];
                }
            }
        }
        float q = 0.0f;
#pragma unroll
        for (int k = 0; k < NV; k++)
#pragma unroll
            for (int i = 0; i < 8; i++) q = fmaf(v[k][i], v[k][i], q);
        const float rstd = 1.0f / sqrtf(RowSum<LANES>::sum(q, slots[turn]) / (float)cols + a.eps);
        if (a.rstd && lane == 0) a.rstd[row] = rstd;
        if (a.h) {
            T *h = static_cast<T *>(a.h) + row * a.h_stride;
#pragma unroll
            for (int k = 0; k < NV; k++) {
                Pack<T, 8> p;
                p.from(v[k]);
                p.store(h + 8 * (lane + k * LANES), cols - 8 * (lane + k * LANES));
            }
        }
#pragma unroll
        for (int k = 0; k < NV; k++) {
            const int c = 8 * (lane + k * LANES);
            Weights<T> p;
            float w[8];
            p.load(a.weight, a.weight_type, c, cols - c);
            p.to(a.weight, a.weight_type, w);
#pragma unroll
            for (int i = 0; i < 8; i++) v[k][i] = v[k][i] * rstd * w[i];
        }
        if (!narrow) {
            T *out = static_cast<T *>(a.out) + row * a.out_stride;
#pragma unroll
            for (int k = 0; k < NV; k++) {
                Pack<T, 8> p;
                p.from(v[k]);
                p.store(out + 8 * (lane + k * LANES), cols - 8 * (lane + k * LANES));
            }
            continue;
        }
        uint32_t m[NV];
#pragma unroll
        for (int k = 0; k < NV; k++) m[k] = largest(v[k]);
        if (a.group == 0) {
#pragma unroll
            for (int k = 1; k < NV; k++) m[0] = m[k] > m[0] ? m[k] : m[0];
            const uint32_t t = RowSum<LANES>::max(m[0], slots[2 + turn]);
#pragma unroll
            for (int k = 0; k < NV; k++) m[k] = t;
        } else {
#pragma unroll
            for (int k = 0; k < NV; k++)
                m[k] = a.group == 128 ? lanes_max<16>(m[k]) : a.group == 64 ? lanes_max<8>(m[k]) : lanes_max<4>(m[k]);
        }
        const int group = a.group ? a.group : cols, groups = (cols + group - 1) / group;
        uint8_t *out = static_cast<uint8_t *>(a.out) + row * a.out_stride;
#pragma unroll
        for (int k = 0; k < NV; k++) {
            const int c = 8 * (lane + k * LANES);
            const float scale = scale_of(m[k], most);
            const Quotient by(scale);
            if (a.group ? c < cols && c % group == 0 : c == 0) a.scales[row * groups + c / group] = scale;
            float y[8];
#pragma unroll
            for (int i = 0; i < 8; i++) y[i] = by(v[k][i]);
            store_pack_8(out + c, y, cols - c, a.out_type);
        }
    }
}

// --- rows of any width --------------------------------------------------------
// A workgroup of 1,024 threads goes over the row in packs, again for each of
// its sums (a row of x and residual mostly stays in the L2).
constexpr int kLoopLanes = 1024;

// columns of the pack at c that the row has: 0 to 8
__device__ __forceinline__ int have_of(int64_t cols, int64_t c) {
    const int64_t n = cols - c;
    return n < 0 ? 0 : n < 8 ? (int)n : 8;
}

template <class T>
struct LoopRow {
    const T *x, *r;
    int64_t cols;
    __device__ __forceinline__ void sum_at(int64_t c, int have, float (&v)[8]) const {
        Pack<T, 8> px, pr;
        px.load(x + c, have);
        if (r) pr.load(r + c, have);
        px.to(v);
        if (r) {
            float y[8];
            pr.to(y);
#pragma unroll
            for (int i = 0; i < 8; i++) v[i] += y[i];
        }
    }
};
template <class T, class Args>
__device__ __forceinline__ void weights_at(const Args &a, int64_t c, int have, float (&w)[8]) {
    Weights<T> p;
    p.load(a.weight, a.weight_type, c, have);
    p.to(a.weight, a.weight_type, w);
}
// Wider than 32,768 columns: bound by HBM and what the L2 does not keep.
// 4,000 x 40,000 bf16 with a residual 289 us (4.4 TB/s of what has to move), to
// 8 bits by 128 columns 269 us (column by column 641 and 1,463).
template <class T>
__global__ void __launch_bounds__(kLoopLanes) k_rms_loop(RmsArgs a) {
    __shared__ float slots[2][16];
    const int64_t row = blockIdx.x + (int64_t)blockIdx.y * gridDim.x;
    if (row >= a.rows) return;
    const LoopRow<T> in{static_cast<const T *>(a.x) + row * a.x_stride,
                        a.residual ? static_cast<const T *>(a.residual) + row * a.residual_stride : nullptr, a.cols};
    const bool narrow = a.out_type == DD_E4M3 || a.out_type == DD_I8;
    const float most = most_of(a.out_type);
    float q = 0.0f;
    for (int64_t c = 8 * threadIdx.x; c < a.cols; c += 8 * kLoopLanes) {
        float v[8];
        in.sum_at(c, have_of(a.cols, c), v);
#pragma unroll
        for (int i = 0; i < 8; i++) q = fmaf(v[i], v[i], q);
    }
    const float rstd = 1.0f / sqrtf(RowSum<kLoopLanes>::sum(q, slots[0]) / (float)a.cols + a.eps);
    if (a.rstd && threadIdx.x == 0) a.rstd[row] = rstd;
    uint32_t all = 0;
    if (narrow && a.group == 0) {
        for (int64_t c = 8 * threadIdx.x; c < a.cols; c += 8 * kLoopLanes) {
            float v[8], w[8];
            in.sum_at(c, have_of(a.cols, c), v);
            weights_at<T>(a, c, have_of(a.cols, c), w);
#pragma unroll
            for (int i = 0; i < 8; i++) v[i] = v[i] * rstd * w[i];
            const uint32_t m = largest(v);
            all = m > all ? m : all;
        }
        all = RowSum<kLoopLanes>::max(all, slots[1]);
        if (threadIdx.x == 0) a.scales[row] = scale_of(all, most);
    }
    const int64_t groups = a.group ? (a.cols + a.group - 1) / a.group : 1;
    // (every lane goes round as often as the first: groups are exchanged)
    for (int64_t first = 0; first < a.cols; first += 8 * kLoopLanes) {
        const int64_t c = first + 8 * threadIdx.x;
        const int have = have_of(a.cols, c);
        float v[8], w[8];
        in.sum_at(c, have, v);
        weights_at<T>(a, c, have, w);
        if (a.h) {
            Pack<T, 8> p;
            p.from(v);
            p.store(static_cast<T *>(a.h) + row * a.h_stride + c, have);
        }
#pragma unroll
        for (int i = 0; i < 8; i++) v[i] = v[i] * rstd * w[i];
        if (!narrow) {
            Pack<T, 8> p;
            p.from(v);
            p.store(static_cast<T *>(a.out) + row * a.out_stride + c, have);
            continue;
        }
        uint32_t m = all;
        if (a.group) {
            m = largest(v);
            m = a.group == 128 ? lanes_max<16>(m) : a.group == 64 ? lanes_max<8>(m) : lanes_max<4>(m);
        }
        const float scale = scale_of(m, most);
        const Quotient by(scale);
        if (a.group && c < a.cols && c % a.group == 0) a.scales[row * groups + c / a.group] = scale;
#pragma unroll
        for (int i = 0; i < 8; i++) v[i] = by(v[i]);
        store_pack_8(static_cast<uint8_t *>(a.out) + row * a.out_stride + c, v, have, a.out_type);
    }
}

// The gradient of rows held in registers, as k_rms_row holds them.  A workgroup
// goes over rows (b, b + grid, ...) and keeps its sums of dy * xh per column in
// registers; at the end rows of one workgroup are joined through LDS, and the
// workgroup writes one partial sum per column, which k_rms_dw_join adds up in
// order (no atomics: the same bits on every call).
//
// Bound: HBM.  32,768 x 8,192 bf16 with dh 369 us (5.8 TB/s); 16,384 x 1,024
// 28.6 us (4.7) and 4.2 for the join, of which a launch alone is 2.8.
constexpr int grad_threads(int lanes) { return lanes <= 64 ? 1024 : lanes; }

template <class T, int LANES, int NV>
__global__ void __launch_bounds__(grad_threads(LANES)) k_rms_grad_row(RmsGradArgs a, float *part) {
    constexpr int kThreads = grad_threads(LANES), kRows = kThreads / LANES;
    __shared__ float slots[2][16];
    const int lane = threadIdx.x % LANES;
    const int cols = (int)a.cols;
    float sum[NV][8] = {};
    float w[NV][8];
#pragma unroll
    for (int k = 0; k < NV; k++) {
        Weights<T> p;
        p.load(a.weight, a.weight_type, 8 * (lane + k * LANES), cols - 8 * (lane + k * LANES));
        p.to(a.weight, a.weight_type, w[k]);
    }
    int turn = 0;
    for (int64_t row = (int64_t)blockIdx.x * kRows + row_of_thread<LANES>(); row < a.rows;
         row += (int64_t)gridDim.x * kRows, turn ^= 1) {
        const T *dy = static_cast<const T *>(a.dy) + row * a.dy_stride;
        const T *h = static_cast<const T *>(a.h) + row * a.h_stride;
        const T *dh = static_cast<const T *>(a.dh) + row * a.dh_stride;
        T *dx = static_cast<T *>(a.dx) + row * a.dx_stride;
        Pack<T, 8> pd[NV], ph[NV], pe[NV];
#pragma unroll
        for (int k = 0; k < NV; k++) pd[k].load(dy + 8 * (lane + k * LANES), cols - 8 * (lane + k * LANES));
#pragma unroll
        for (int k = 0; k < NV; k++) ph[k].load(h + 8 * (lane + k * LANES), cols - 8 * (lane + k * LANES));
        if (a.dh) {
#pragma unroll
            for (int k = 0; k < NV; k++) pe[k].load(dh + 8 * (lane + k * LANES), cols - 8 * (lane + k * LANES));
        }
        const float rstd = a.rstd[row];
        float q = 0.0f;
#pragma unroll
        for (int k = 0; k < NV; k++) {
            float d[8], x[8];
            pd[k].to(d);
            ph[k].to(x);
#pragma unroll
            for (int i = 0; i < 8; i++) {
                const float t = d[i] * (x[i] * rstd);
                sum[k][i] += t;
                q = fmaf(w[k][i], t, q);
            }
        }
        const float c = RowSum<LANES>::sum(q, slots[turn]) / (float)cols;
#pragma unroll
        for (int k = 0; k < NV; k++) {
            float d[8], x[8], y[8];
            if (LANES <= 16 || LANES == 1024) {     // (their registers would spill)
                pd[k].forget();
                ph[k].forget();
            }
            pd[k].to(d);
            ph[k].to(x);
#pragma unroll
            for (int i = 0; i < 8; i++) y[i] = 0.0f;
            if (a.dh) pe[k].to(y);
            Pack<T, 8> p;
#pragma unroll
            for (int i = 0; i < 8; i++) y[i] = fmaf(d[i] * w[k][i] - x[i] * rstd * c, rstd, y[i]);
            p.from(y);
            p.store(dx + 8 * (lane + k * LANES), cols - 8 * (lane + k * LANES));
        }
    }
    if (!a.dw) return;
    // one workgroup has all rows: its sums are the result
    if (gridDim.x > 1) part += (int64_t)blockIdx.x * cols;
    auto put = [&](int c, const float (&x)[8]) {
        if (gridDim.x > 1) {
            Pack<float, 8> p;
            p.from(x);
            p.store(part + c, cols - c);
        } else if (a.weight_type == DD_F32) {
            Pack<float, 8> p;
            p.from(x);
            p.store(static_cast<float *>(a.dw) + c, cols - c);
        } else {
            Pack<T, 8> p;
            p.from(x);
            p.store(static_cast<T *>(a.dw) + c, cols - c);
        }
    };
    if (kRows == 1) {
#pragma unroll
        for (int k = 0; k < NV; k++) put(8 * (lane + k * LANES), sum[k]);
        return;
    }
    // rows that share the workgroup, joined in order, LANES packs at a time
    __shared__ float all[kRows * LANES * 8];
#pragma unroll
    for (int k = 0; k < NV; k++) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 8; i++) all[threadIdx.x * 8 + i] = sum[k][i];
        __syncthreads();
        if (threadIdx.x < LANES) {
            float t[8] = {};
            for (int r = 0; r < kRows; r++)
#pragma unroll
                for (int i = 0; i < 8; i++) t[i] += all[(r * LANES + threadIdx.x) * 8 + i];
            put(8 * (threadIdx.x + k * LANES), t);
        }
    }
}

// Wider than 16,384 columns: dweight first (dx may overwrite what it reads),
// then dx, in passes over the rows: dy and h are read three times.  4,000 x
// 40,000 bf16 with dh 410 us (column by column 940).
template <class T>
__global__ void __launch_bounds__(kLoopLanes) k_rms_dx_loop(RmsGradArgs a) {
    __shared__ float slot[16];
    const int64_t row = blockIdx.x + (int64_t)blockIdx.y * gridDim.x;
    if (row >= a.rows) return;
    const T *dy = static_cast<const T *>(a.dy) + row * a.dy_stride;
    const T *h = static_cast<const T *>(a.h) + row * a.h_stride;
    const T *dh = a.dh ? static_cast<const T *>(a.dh) + row * a.dh_stride : nullptr;
    T *dx = static_cast<T *>(a.dx) + row * a.dx_stride;
    const float rstd = a.rstd[row];
    // weight * dy, and xh
    auto terms = [&](int64_t c, int have, float (&g)[8], float (&x)[8]) {
        Pack<T, 8> pd, ph;
        float w[8];
        pd.load(dy + c, have);
        ph.load(h + c, have);
        weights_at<T>(a, c, have, w);
        pd.to(g);
        ph.to(x);
#pragma unroll
        for (int i = 0; i < 8; i++) {
            g[i] *= w[i];
            x[i] *= rstd;
        }
    };
    float q = 0.0f;
    for (int64_t c = 8 * threadIdx.x; c < a.cols; c += 8 * kLoopLanes) {
        float g[8], x[8];
        terms(c, have_of(a.cols, c), g, x);
#pragma unroll
        for (int i = 0; i < 8; i++) q = fmaf(g[i], x[i], q);
    }
    const float m = RowSum<kLoopLanes>::sum(q, slot) / (float)a.cols;
    for (int64_t c = 8 * threadIdx.x; c < a.cols; c += 8 * kLoopLanes) {
        const int have = have_of(a.cols, c);
        float g[8], x[8], y[8] = {};
        Pack<T, 8> p;
        if (dh) {
            p.load(dh + c, have);
            p.to(y);
        }
        terms(c, have, g, x);
#pragma unroll
        for (int i = 0; i < 8; i++) y[i] = fmaf(g[i] - x[i] * m, rstd, y[i]);
        p.from(y);
        p.store(dx + c, have);
    }
}

// Partial sums of dweight: workgroup (i, j) has 256 columns and the j-th of
// gridDim.y runs of rows, eight rows at a time.
constexpr int kDwCols = 256, kDwRows = 8;
template <class T>
__global__ void __launch_bounds__(kDwCols) k_rms_dw_loop(RmsGradArgs a, float *part) {
    __shared__ float lds[kDwRows][kDwCols];
    const int x = threadIdx.x % (kDwCols / 8), y = threadIdx.x / (kDwCols / 8);
    const int64_t c = (int64_t)blockIdx.x * kDwCols + 8 * x;
    const int have = have_of(a.cols, c);
    const int64_t run = (a.rows + gridDim.y - 1) / gridDim.y;
    const int64_t r0 = blockIdx.y * run, r1 = r0 + run < a.rows ? r0 + run : a.rows;
    float s[8] = {};
    for (int64_t r = r0 + y; r < r1; r += kDwRows) {
        Pack<T, 8> pd, ph;
        float d[8], v[8];
        pd.load(static_cast<const T *>(a.dy) + r * a.dy_stride + c, have);
        ph.load(static_cast<const T *>(a.h) + r * a.h_stride + c, have);
        const float rstd = a.rstd[r];
        pd.to(d);
        ph.to(v);
#pragma unroll
        for (int i = 0; i < 8; i++) s[i] = fmaf(d[i], v[i] * rstd, s[i]);
    }
#pragma unroll
    for (int i = 0; i < 8; i++) lds[y][8 * x + i] = s[i];
    __syncthreads();
    const int64_t mine = (int64_t)blockIdx.x * kDwCols + threadIdx.x;
    if (mine >= a.cols) return;
    float t = 0.0f;
#pragma unroll
    for (int i = 0; i < kDwRows; i++) t += lds[i][threadIdx.x];
    part[blockIdx.y * a.cols + mine] = t;
}

// A workgroup has 32 columns; 32 threads share a column, each with up to 16
// loads under way (512 partial sums, all of them).
__global__ void __launch_bounds__(1024) k_rms_dw_join(RmsGradArgs a, const float *part, int n) {
    __shared__ float lds[32][33];
    const int x = threadIdx.x & 31, y = threadIdx.x >> 5;
    const int64_t c = (int64_t)blockIdx.x * 32 + x;
    float s = 0.0f;
    if (c < a.cols) {
        float t[kRmsParts / 32];
#pragma unroll
        for (int i = 0; i < kRmsParts / 32; i++) t[i] = y + 32 * i < n ? part[(y + 32 * i) * a.cols + c] : 0.0f;
#pragma unroll
        for (int i = 0; i < kRmsParts / 32; i++) s += t[i];
    }
    lds[y][x] = s;
    __syncthreads();
    if (y || c >= a.cols) return;
    s = 0.0f;
#pragma unroll
    for (int i = 0; i < 32; i++) s += lds[i][x];
    if (a.weight_type == DD_F32) static_cast<float *>(a.dw)[c] = s;
    else if (a.weight_type == DD_BF16) static_cast<bf16_t *>(a.dw)[c] = (bf16_t)s;
    else static_cast<f16_t *>(a.dw)[c] = (f16_t)s;
}

dim3 grid_of_rows(int64_t rows) {       // (a launch takes fewer than 2^32 threads a dimension)
    const int64_t x = rows < (1 << 20) ? rows : (1 << 20);
    return dim3((unsigned)x, (unsigned)((rows + x - 1) / x));
}

int dw_runs(int64_t rows) {
    const int64_t r = (rows + 255) / 256;
    return r < 1 ? 1 : r > kRmsParts ? kRmsParts : (int)r;
}

// Lanes per row and packs per lane.  Two packs of each input are enough loads
// under way, and more cost registers, so the fewest lanes that hold the row
// with two packs (four at the widest), a whole wave or more past 256 columns
// so that no lanes idle.  Measured on bf16 with a residual, TB/s (to 8 bits with
// the quotients in 32, which takes 3 to 6 % less): 8,192 x 4,096 to 8 bits 4.8
// with 256 lanes x 2 (128 x 4: 4.2, 64 x 8: 3.6, 1,024 x 1: 2.7); 16,384 x 1,024
// 5.0 with 64 x 2 (256 x 1: 4.3); 65,536 x 2,048 5.8 with 256 x 1 (64 x 4: 5.7);
// 65,536 x 128 to 8 bits 3.6 with 16 x 1 (64 x 1: 1.5); 65,536 x 64 3.5 with 8 x 1 (16 x 1: 2.7).  Few rows take the
// same: 4 to 512 rows of 4,096 are as fast with any of these shapes, the launch
// bounds them.
struct Shape {
    int lanes, packs;      // 0: k_rms_loop
};
Shape row_shape(int64_t cols) {
    const int64_t n = (cols + 7) / 8;
    if (n <= 8) return {8, 1};
    if (n <= 32) return {16, n <= 16 ? 1 : 2};
    if (n <= 128) return {64, n <= 64 ? 1 : 2};
    if (n <= 512) return {256, n <= 256 ? 1 : 2};
    if (n <= 1024) return {512, 2};
    if (n <= 4096) return {1024, n <= 2048 ? 2 : 4};
    return {0, 0};
}

constexpr int kRowBlocks = 1 << 20;    // workgroups of a launch at most; rows beyond go round

template <class T, int LANES, int NV>
void run_rows(const RmsArgs &a, hipStream_t s) {
    constexpr int kThreads = row_threads(LANES), kRows = kThreads / LANES;
    const int64_t need = (a.rows + kRows - 1) / kRows;
    k_rms_row<T, LANES, NV><<<(unsigned)(need < kRowBlocks ? need : kRowBlocks), kThreads, 0, s>>>(a);
}
template <class T>
void rms_norm(const RmsArgs &a, hipStream_t s) {
    const Shape p = row_shape(a.cols);
    if (p.lanes == 8) return run_rows<T, 8, 1>(a, s);
    if (p.lanes == 16 && p.packs == 1) return run_rows<T, 16, 1>(a, s);
    if (p.lanes == 16 && p.packs == 2) return run_rows<T, 16, 2>(a, s);
    if (p.lanes == 64 && p.packs == 1) return run_rows<T, 64, 1>(a, s);
    if (p.lanes == 64 && p.packs == 2) return run_rows<T, 64, 2>(a, s);
    if (p.lanes == 256 && p.packs == 1) return run_rows<T, 256, 1>(a, s);
    if (p.lanes == 256 && p.packs == 2) return run_rows<T, 256, 2>(a, s);
    if (p.lanes == 512 && p.packs == 2) return run_rows<T, 512, 2>(a, s);
    if (p.lanes == 1024 && p.packs == 2) return run_rows<T, 1024, 2>(a, s);
    if (p.lanes == 1024 && p.packs == 4) return run_rows<T, 1024, 4>(a, s);
    k_rms_loop<T><<<grid_of_rows(a.rows), kLoopLanes, 0, s>>>(a);
}

// The gradient holds three times as much per column: four packs do not fit.
Shape grad_shape(int64_t cols) {
    const Shape p = row_shape(cols);
    return p.packs > 2 ? Shape{0, 0} : p;
}

// Workgroups of the gradient: as many as run at once, each with rows to go
// over: two to a compute unit where they are of four waves and hold less than
// 16 KiB of a row (65,536 x 2,048 bf16: 196 us, one to each 306; 16,384 x 4,096
// f32: 204, one to each 188; 32,768 x 8,192 bf16: 404 and 369).
int grad_parts(int64_t rows, int64_t cols, int elem) {
    const Shape p = grad_shape(cols);
    if (!p.lanes) return dw_runs(rows);
    const int per = grad_threads(p.lanes) / p.lanes;
    const int64_t need = (rows + per - 1) / per, most = p.lanes == 256 && p.lanes * p.packs * 8 * elem < 16384 ? 512 : 256;
    return (int)(need < 1 ? 1 : need < most ? need : most);
}

template <class T, int LANES, int NV>
void run_grad(const RmsGradArgs &a, float *work, int parts, hipStream_t s) {
    k_rms_grad_row<T, LANES, NV><<<parts, grad_threads(LANES), 0, s>>>(a, work);
}
template <class T>
void rms_grad(const RmsGradArgs &a, float *work, hipStream_t s) {
    const Shape p = grad_shape(a.cols);
    const int n = grad_parts(a.rows, a.cols, sizeof(T));
    auto join = [&] { k_rms_dw_join<<<(unsigned)((a.cols + 31) / 32), 1024, 0, s>>>(a, work, n); };
    if (!p.lanes) {
        if (a.dw) {
            k_rms_dw_loop<T><<<dim3((unsigned)((a.cols + kDwCols - 1) / kDwCols), n), kDwCols, 0, s>>>(a, work);
            join();
        }
        if (a.rows > 0) k_rms_dx_loop<T><<<grid_of_rows(a.rows), kLoopLanes, 0, s>>>(a);
        return;
    }
    if (p.lanes == 8) run_grad<T, 8, 1>(a, work, n, s);
    else if (p.lanes == 16 && p.packs == 1) run_grad<T, 16, 1>(a, work, n, s);
    else if (p.lanes == 16) run_grad<T, 16, 2>(a, work, n, s);
    else if (p.lanes == 64 && p.packs == 1) run_grad<T, 64, 1>(a, work, n, s);
    else if (p.lanes == 64) run_grad<T, 64, 2>(a, work, n, s);
    else if (p.lanes == 256 && p.packs == 1) run_grad<T, 256, 1>(a, work, n, s);
    else if (p.lanes == 256) run_grad<T, 256, 2>(a, work, n, s);
    else if (p.lanes == 512) run_grad<T, 512, 2>(a, work, n, s);
    else run_grad<T, 1024, 2>(a, work, n, s);
    if (a.dw && n > 1) join();
}

}  // namespace

size_t rms_grad_work(int64_t rows, int64_t cols) {
    return (size_t)grad_parts(rows, cols, 2) * (size_t)cols * sizeof(float);    // (the most of any type)
}

hipError_t launch_rms_norm(const RmsArgs &args, hipStream_t s) {
    RmsArgs a = args;
    if (a.group >= a.cols) a.group = 0;     // (a row narrower than a group may have fewer lanes than one)
    if (a.type == DD_F32) rms_norm<float>(a, s);
    else if (a.type == DD_BF16) rms_norm<bf16_t>(a, s);
    else rms_norm<f16_t>(a, s);
    return hipGetLastError();
}

hipError_t launch_rms_norm_grad(const RmsGradArgs &a, float *work, hipStream_t s) {
    if (a.type == DD_F32) rms_grad<float>(a, work, s);
    else if (a.type == DD_BF16) rms_grad<bf16_t>(a, work, s);
    else rms_grad<f16_t>(a, work, s);
    return hipGetLastError();
}

}  // namespace dd
