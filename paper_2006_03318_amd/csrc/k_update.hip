// The weight update over many tensors: global gradient norm, clipping, Adam.
//
// A handle cuts its tensors into chunks of one length (the last of a tensor
// shorter) and holds one record per chunk with the chunk's own addresses, so
// one launch takes any number of tensors and a workgroup finds its work with
// one read.  All three passes move each element once and compute little:
// they are bound by memory, small lists by the launch.
#include "dd_elem.h"
#include "dd_internal.h"

namespace dd {

namespace {

constexpr int kBlock = 256;


// Squares in 64 bits: one of an f32 (or bf16) gradient leaves the 32-bit range
// above 1.8e19 and below 1e-19, and a sum over 10^9 elements keeps its digits.
template <class G>
__device__ double chunk_squares(const G *g, int n) {
    double s = 0.0;
    for (int i = threadIdx.x; i < n; i += kBlock) {
        const double x = (double)(float)global(g)[i];
        s = fma(x, x, s);
    }
    return s;
}

__device__ double block_sum(double x) {
    __shared__ double part[kBlock / 64];
    x = wave_sum(x);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = x;
    __syncthreads();
    double t = 0.0;
#pragma unroll
    for (int w = 0; w < kBlock / 64; w++) t += part[w];
    __syncthreads();
    return t;
}

// Each workgroup sums its chunks (a fixed set: chunk b, b + grid, ...) into
// its own partial; a second launch joins them in order.  No atomics: the
// result is the same on every call.
__global__ void __launch_bounds__(kBlock) k_grad_squares(const TensorChunk *ck, int n_chunks, double *part) {
    double s = 0.0;
    for (int c = blockIdx.x; c < n_chunks; c += gridDim.x) {
        const TensorChunk k = ck[c];
        if (k.grad_type == DD_F32) s += chunk_squares(static_cast<const float *>(k.grad), k.n);
        else if (k.grad_type == DD_BF16) s += chunk_squares(static_cast<const bf16_t *>(k.grad), k.n);
        else s += chunk_squares(static_cast<const f16_t *>(k.grad), k.n);
    }
    s = block_sum(s);
    if (threadIdx.x == 0) part[blockIdx.x] = s;
}

__device__ void write_stats(double s, double max_norm, const float *inv_scale, float *stats) {
    const double u = inv_scale ? (double)*inv_scale : 1.0;
    const double norm = sqrt(s) * u;
    const bool finite = isfinite(s);
    double f = u;
    if (max_norm > 0.0 && norm > max_norm) f = u * (max_norm / norm);
    stats[0] = (float)norm;
    stats[1] = finite ? (float)f : 0.0f;
    stats[2] = finite ? 0.0f : 1.0f;
}

__global__ void __launch_bounds__(kBlock) k_grad_join(const double *part, int n, double max_norm, const float *inv_scale,
                                                      float *stats) {
    double s = 0.0;
    for (int i = threadIdx.x; i < n; i += kBlock) s += part[i];
    s = block_sum(s);
    if (threadIdx.x == 0) write_stats(s, max_norm, inv_scale, stats);
}

template <class G, class D>
__device__ void chunk_clip(const G *g, D *d, int n, float f) {
    for (int i = threadIdx.x; i < n; i += kBlock) {
        const float x = (float)global(g)[i];
        global(d)[i] = (D)(f == 0.0f ? 0.0f : x * f);
    }
}

template <class G>
__device__ void chunk_clip_to(const G *g, const TensorChunk &d, int n, float f) {
    if (d.grad_type == DD_F32) chunk_clip(g, static_cast<float *>(d.grad), n, f);
    else if (d.grad_type == DD_BF16) chunk_clip(g, static_cast<bf16_t *>(d.grad), n, f);
    else chunk_clip(g, static_cast<f16_t *>(d.grad), n, f);
}

// Chunks of both lists are alike (equal sizes, one rule for the chunk length).
__global__ void __launch_bounds__(kBlock) k_grad_clip(const TensorChunk *src, const TensorChunk *dst, int n_chunks,
                                                      const float *stats) {
    const float f = stats[1];
    for (int c = blockIdx.x; c < n_chunks; c += gridDim.x) {
        const TensorChunk a = src[c], b = dst[c];
        if (a.grad_type == DD_F32) chunk_clip_to(static_cast<const float *>(a.grad), b, a.n, f);
        else if (a.grad_type == DD_BF16) chunk_clip_to(static_cast<const bf16_t *>(a.grad), b, a.n, f);
        else chunk_clip_to(static_cast<const f16_t *>(a.grad), b, a.n, f);
    }
}

// beta^t by squaring: t < 2^63 in at most 126 multiplications, each of
// relative error 2^-53
__device__ double power(double b, int64_t t) {
    double r = 1.0;
    for (; t > 0; t >>= 1, b *= b)
        if (t & 1) r *= b;
    return r;
}

struct AdamFactors {      // of one call, rounded once from 64 bits
    float f;              // factor of the gradients
    float b1, c1, b2, c2; // beta1, 1 - beta1, beta2, 1 - beta2
    float l2, keep;       // added weight * l2, or kept share of the weight
    float lr, rv, eps;    // lr / (1 - beta1^t), 1 / sqrt(1 - beta2^t)
};

__device__ __forceinline__ void adam_one(const AdamFactors &a, bool decay, float g, float &w, float &m, float &v) {
    g *= a.f;
    if (decay) g = fmaf(a.l2, w, g);
    m = fmaf(a.b1, m, a.c1 * g);
    v = fmaf(a.b2, v, a.c2 * (g * g));
    if (decay) w *= a.keep;
    w -= a.lr * (m / fmaf(sqrtf(v), a.rv, a.eps));
}

template <class G>
__device__ void chunk_adam(const TensorChunk &k, const AdamFactors &a) {
    const G *g = static_cast<const G *>(k.grad);
    const bool low = k.param_type != DD_F32;
    for (int i = threadIdx.x; i < k.n; i += kBlock) {
        float w = global(k.w)[i], m = global(k.m)[i], v = global(k.v)[i];
        adam_one(a, k.decay, (float)global(g)[i], w, m, v);
        global(k.w)[i] = w;
        global(k.m)[i] = m;
        global(k.v)[i] = v;
        if (low) {
            if (k.param_type == DD_BF16) global(static_cast<bf16_t *>(k.param))[i] = (bf16_t)w;
            else global(static_cast<f16_t *>(k.param))[i] = (f16_t)w;
        }
    }
}

__global__ void __launch_bounds__(kBlock) k_adam(const TensorChunk *ck, int n_chunks, const int64_t *step, const float *stats,
                                                 AdamParams p) {
    if (stats && stats[2] != 0.0f) return;
    const int64_t t = *step + 1;
    AdamFactors a;
    a.f = stats ? stats[1] : 1.0f;
    a.b1 = (float)p.beta1;
    a.c1 = (float)(1.0 - p.beta1);
    a.b2 = (float)p.beta2;
    a.c2 = (float)(1.0 - p.beta2);
    a.l2 = p.decoupled ? 0.0f : (float)p.weight_decay;
    a.keep = p.decoupled ? (float)(1.0 - p.lr * p.weight_decay) : 1.0f;
    a.lr = (float)(p.lr / (1.0 - power(p.beta1, t)));
    a.rv = (float)(1.0 / sqrt(1.0 - power(p.beta2, t)));
    a.eps = (float)p.eps;
    for (int c = blockIdx.x; c < n_chunks; c += gridDim.x) {
        const TensorChunk k = ck[c];
        if (k.grad_type == DD_F32) chunk_adam<float>(k, a);
        else if (k.grad_type == DD_BF16) chunk_adam<bf16_t>(k, a);
        else chunk_adam<f16_t>(k, a);
    }
}

__global__ void k_adam_step(int64_t *step, const float *stats) {
    if (!(stats && stats[2] != 0.0f)) *step += 1;
}

int grid_of(int n_chunks) { return n_chunks < kNormParts ? (n_chunks < 1 ? 1 : n_chunks) : kNormParts; }

}  // namespace

hipError_t launch_grad_norm(const dd_tensors *t, double max_norm, const float *inv_scale, float *stats, hipStream_t s) {
    const int g = grid_of(t->n_chunks);
    k_grad_squares<<<g, kBlock, 0, s>>>(t->chunks, t->n_chunks, t->part);
    k_grad_join<<<1, kBlock, 0, s>>>(t->part, g, max_norm, inv_scale, stats);
    return hipGetLastError();
}

hipError_t launch_grad_clip(const dd_tensors *src, const dd_tensors *dst, const float *stats, hipStream_t s) {
    if (src->n_chunks == 0) return hipSuccess;
    k_grad_clip<<<grid_of(src->n_chunks), kBlock, 0, s>>>(src->chunks, dst->chunks, src->n_chunks, stats);
    return hipGetLastError();
}

hipError_t launch_adam(const dd_tensors *t, int64_t *step, const float *stats, const AdamParams &p, hipStream_t s) {
    if (t->n_chunks) k_adam<<<grid_of(t->n_chunks), kBlock, 0, s>>>(t->chunks, t->n_chunks, step, stats, p);
    k_adam_step<<<1, 1, 0, s>>>(step, stats);
    return hipGetLastError();
}

}  // namespace dd
