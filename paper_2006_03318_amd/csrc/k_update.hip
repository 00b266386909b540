// The weight update over many tensors: global gradient norm, clipping, Adam.
//
// A handle cuts its tensors into chunks of kChunkLen elements (the last of a
// tensor shorter) and holds one record per chunk with the chunk's own
// addresses, so one launch takes any number of tensors and a workgroup finds
// its work with one read.  All three passes move each element once and compute
// little: they are bound by memory, small lists by the launch.
//
// The norm only reads: 1,024 workgroups go over all chunks, four loads of 16
// bytes or more under way in every lane (302 M bf16 gradients 102 us, 5.9 TB/s,
// after other norms, and 129 after a pass that wrote, of which up to 256 MB go
// to memory meanwhile; a workgroup per chunk 140).  Clipping and Adam write as much as they read, and
// go fastest with a workgroup for each kPartLen elements that does nothing else
// (Adam on the same list 5.3 TB/s, 5.1 with 8,192 elements to a workgroup, 5.0
// with 2,048 workgroups that go round).
#include <type_traits>

#include "dd_elem.h"
#include "dd_train.h"

namespace dd {

namespace {

constexpr int kBlock = 256;

// One thread per chunk finds its tensor (the last that starts at or before it).
__global__ void __launch_bounds__(kBlock) k_tensor_chunks(const TensorPlace *p, int count, TensorChunk *ck, int n_chunks,
                                                          uint32_t *ticket) {
    const int64_t c = (int64_t)blockIdx.x * kBlock + threadIdx.x;
    if (c == 0) *ticket = 0;
    if (c >= n_chunks) return;
    int lo = 0, hi = count - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) / 2;
        if (p[mid].first <= c) lo = mid;
        else hi = mid - 1;
    }
    TensorChunk k = p[lo].whole;
    const int64_t o = (c - p[lo].first) * kChunkLen, left = p[lo].n - o;
    k.grad = static_cast<char *>(k.grad) + o * elem_size(k.grad_type);
    if (k.param) {
        k.param = static_cast<char *>(k.param) + o * elem_size(k.param_type);
        k.w += o;
        k.m += o;
        k.v += o;
    }
    k.n = (int)(left < kChunkLen ? left : kChunkLen);
    ck[c] = k;
}

// Elements per thread and load.
constexpr int kWide = 8, kTurn = kBlock * kWide, kAhead = kChunkLen / kTurn;
static_assert(kChunkLen == kAhead * kTurn, "a chunk is whole turns of a workgroup");
constexpr int kPartLen = 2048, kPartsOf = kChunkLen / kPartLen;
static_assert(kPartLen == kTurn, "clipping: a pack for each thread");

// Adam: 1, 2 or 4 workgroups share a chunk (`split` is the logarithm), each
// taking every so many-th part of it: four, a part each, but of many chunks
// (past kSmallShares) no more than the mean chunk fills, as workgroups that
// find no part only cost (1,000 tensors of 3,000 elements or fewer: 9.0 us with
// one to a chunk, 12.6 with four; 30 tensors of 5,000 or fewer 6.3 and 5.3).
// Clipping always takes four: with a loop over parts it ran 5 % longer on large
// lists.
//
// Up to kSmallShares the tickets of k_adam_small (12 ns each) cost less than a
// launch more: 50 shares 5.4 us against 7.4, 300 shares 6.5 against 7.4, 480
// shares 8.5 against 7.3.
constexpr int64_t kSmallShares = 320;
int split_of(const dd_tensors *t) {
    const int64_t mean = t->total / (t->n_chunks ? t->n_chunks : 1);
    int split = 2;
    while (split > 0 && (int64_t)t->n_chunks << split > kSmallShares && mean <= kPartLen << (split - 1)) split--;
    return split;
}

// Squares in 64 bits: one of an f32 (or bf16) gradient leaves the 32-bit range
// above 1.8e19 and below 1e-19, and a sum over 10^9 elements keeps its digits.
__device__ __forceinline__ double squares(const float (&x)[kWide], double s) {
#pragma unroll
    for (int i = 0; i < kWide; i++) s = fma((double)x[i], (double)x[i], s);
    return s;
}
template <class G>
__device__ __forceinline__ double chunk_squares(const G *g, int n) {
    double s[2] = {0.0, 0.0};
    float x[kWide];
    int i = threadIdx.x * kWide;
    if (n == kChunkLen) {
        Pack<G, kWide> p[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; u++) p[u].load(g + i + u * kTurn);
#pragma unroll
        for (int u = 0; u < kAhead; u++) {
            p[u].to(x);
            s[u & 1] = squares(x, s[u & 1]);
        }
        return s[0] + s[1];
    }
    for (; i < n; i += kTurn) {
        Pack<G, kWide> p;
        p.load(g + i, n - i);
        p.to(x);
        s[0] = squares(x, s[0]);
    }
    return s[0];
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

__device__ void write_stats(double s, double max_norm, const float *inv_scale, float *stats) {
    const double u = inv_scale ? (double)*inv_scale : 1.0;
    const double norm = sqrt(s) * u;
    const bool finite = isfinite(norm);
    double f = u;
    if (max_norm > 0.0 && norm > max_norm) f = u * (max_norm / norm);
    stats[0] = (float)norm;
    stats[1] = finite ? (float)f : 0.0f;
    stats[2] = finite ? 0.0f : 1.0f;
}

// How the workgroups of a launch find out which of them is the last: each takes
// a ticket when it is done.  What they hand to the last one are atomic stores
// and loads of the device's scope, which pass the caches of the eight XCDs, so
// all that is needed is that a store has arrived before its ticket is taken:
// the wait.  (An acquire-release ticket writes back and invalidates an L2 each
// time: 302 M bf16 gradients by 1,024 workgroups 140 us instead of 102.)
__device__ __forceinline__ bool last_ticket(uint32_t *ticket) {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    return __hip_atomic_fetch_add(ticket, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == gridDim.x - 1;
}

// Each workgroup sums its chunks (a fixed set: chunk b, b + grid, ...) into its
// own partial; the one that finishes last adds the partials in their order, so
// the result is the same bits on every call.
__global__ void __launch_bounds__(kBlock) k_grad_norm(const TensorChunk *ck, int n_chunks, double *part, uint32_t *ticket,
                                                      double max_norm, const float *inv_scale, float *stats) {
    double s = 0.0;
    for (int c = blockIdx.x; c < n_chunks; c += gridDim.x) {
        const TensorChunk k = ck[c];
        if (k.grad_type == DD_F32) s += chunk_squares(static_cast<const float *>(k.grad), k.n);
        else if (k.grad_type == DD_BF16) s += chunk_squares(static_cast<const bf16_t *>(k.grad), k.n);
        else s += chunk_squares(static_cast<const f16_t *>(k.grad), k.n);
    }
    s = block_sum(s);
    __shared__ bool last;
    if (threadIdx.x == 0) {
        __hip_atomic_store(&part[blockIdx.x], s, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        last = last_ticket(ticket);
    }
    __syncthreads();
    if (!last) return;
    s = 0.0;
    for (int i = threadIdx.x; i < (int)gridDim.x; i += kBlock)
        s += __hip_atomic_load(&part[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    s = block_sum(s);
    if (threadIdx.x == 0) {
        write_stats(s, max_norm, inv_scale, stats);
        *ticket = 0;
    }
}

template <class G, class D>
__device__ __forceinline__ void part_clip(const G *g, D *d, int n, float f) {
    const int i = threadIdx.x * kWide;
    if (i >= n) return;
    Pack<G, kWide> p;
    Pack<D, kWide> q;
    float x[kWide];
    p.load(g + i, n - i);
    p.to(x);
#pragma unroll
    for (int j = 0; j < kWide; j++) x[j] = f == 0.0f ? 0.0f : x[j] * f;   // (an infinity too)
    q.from(x);
    q.store(d + i, n - i);
}

template <class G>
__device__ __forceinline__ void part_clip_to(const G *g, const TensorChunk &d, int o, int n, float f) {
    if (d.grad_type == DD_F32) part_clip(g + o, static_cast<float *>(d.grad) + o, n, f);
    else if (d.grad_type == DD_BF16) part_clip(g + o, static_cast<bf16_t *>(d.grad) + o, n, f);
    else part_clip(g + o, static_cast<f16_t *>(d.grad) + o, n, f);
}

// Chunks of both lists are alike (equal sizes).
__global__ void __launch_bounds__(kBlock) k_grad_clip(const TensorChunk *src, const TensorChunk *dst, int64_t n_parts,
                                                      const float *stats) {
    const float f = stats[1];
    if (src == dst && f == 1.0f) return;     // in place, within the bound: nothing changes
    for (int64_t b = blockIdx.x; b < n_parts; b += gridDim.x) {
        const TensorChunk a = src[b / kPartsOf], d = dst[b / kPartsOf];
        const int o = (int)(b % kPartsOf) * kPartLen, n = a.n - o < kPartLen ? a.n - o : kPartLen;
        if (a.grad_type == DD_F32) part_clip_to(static_cast<const float *>(a.grad), d, o, n, f);
        else if (a.grad_type == DD_BF16) part_clip_to(static_cast<const bf16_t *>(a.grad), d, o, n, f);
        else part_clip_to(static_cast<const f16_t *>(a.grad), d, o, n, f);
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

// What one call multiplies with, each rounded once from 64 bits.
__device__ AdamFactors adam_factors(const AdamParams &p, int64_t t, const float *stats) {
    AdamFactors a;
    a.f = stats ? stats[1] : 1.0f;
    a.b1 = (float)p.beta1;
    a.c1 = (float)(1.0 - p.beta1);
    a.b2 = (float)p.beta2;
    a.c2 = (float)(1.0 - p.beta2);
    a.l2 = p.decoupled ? 0.0f : (float)p.weight_decay;
    a.shrink = p.decoupled ? (float)(p.lr * p.weight_decay) : 0.0f;
    a.lr = (float)(p.lr / (1.0 - power(p.beta1, t)));
    a.rv = (float)(1.0 / sqrt(1.0 - power(p.beta2, t)));
    a.eps = (float)p.eps;
    if (p.eps > 0.0 && a.eps == 0.0f) a.eps = 0x1p-149f;      // (0 / 0 where both moments are 0)
    a.skip = 0;
    return a;
}

// The weight changes by one number, decay and update together, so what is small
// beside the weight is rounded once and not away on its own; and the decay is
// held as lr * weight_decay, as 1 - lr * weight_decay has 2^-24 for a grid (at
// 1e-7 that would be 19 % off, every step).
__device__ __forceinline__ void adam_one(const AdamFactors &a, bool decay, float g, float &w, float &m, float &v) {
    g *= a.f;
    if (decay) g = fmaf(a.l2, w, g);
    m = fmaf(a.b1, m, a.c1 * g);
    v = fmaf(a.b2, v, (a.c2 * g) * g);      // (g * g alone leaves the range from 1.8e19 on)
    float change = a.lr * (m / fmaf(sqrtf(v), a.rv, a.eps));
    if (decay) change = fmaf(a.shrink, w, change);
    w -= change;
}

// Four elements per thread and load, two loads of each array at a time.
constexpr int kAdamWide = 4, kAdamTurn = kBlock * kAdamWide, kAdamAhead = kPartLen / kAdamTurn;
static_assert(kPartLen == kAdamAhead * kAdamTurn, "a part is whole turns of a workgroup");

template <class G, class P>
struct AdamPack {
    Pack<G, kAdamWide> g;
    Pack<float, kAdamWide> w, m, v;
    template <class... Have>
    __device__ __forceinline__ void load(const TensorChunk &k, int i, Have... have) {
        g.load(static_cast<const G *>(k.grad) + i, have...);
        w.load(k.w + i, have...);
        m.load(k.m + i, have...);
        v.load(k.v + i, have...);
    }
    template <class... Have>
    __device__ __forceinline__ void step(const TensorChunk &k, const AdamFactors &a, int i, Have... have) {
        float xg[kAdamWide], xw[kAdamWide], xm[kAdamWide], xv[kAdamWide];
        g.to(xg);
        w.to(xw);
        m.to(xm);
        v.to(xv);
#pragma unroll
        for (int j = 0; j < kAdamWide; j++) adam_one(a, k.decay, xg[j], xw[j], xm[j], xv[j]);
        w.from(xw);
        m.from(xm);
        v.from(xv);
        w.store(k.w + i, have...);
        m.store(k.m + i, have...);
        v.store(k.v + i, have...);
        if (!std::is_same<P, float>::value) {
            Pack<P, kAdamWide> p;
            p.from(xw);
            p.store(static_cast<P *>(k.param) + i, have...);
        }
    }
};

template <class G, class P>
__device__ __forceinline__ void part_adam(const TensorChunk &k, const AdamFactors &a, int o, int n) {
    int i = o + threadIdx.x * kAdamWide;
    if (n - o >= kPartLen) {
        AdamPack<G, P> p[kAdamAhead];
#pragma unroll
        for (int u = 0; u < kAdamAhead; u++) p[u].load(k, i + u * kAdamTurn);
#pragma unroll
        for (int u = 0; u < kAdamAhead; u++) p[u].step(k, a, i + u * kAdamTurn);
        return;
    }
    for (; i < n; i += kAdamTurn) {
        AdamPack<G, P> p;
        p.load(k, i, n - i);
        p.step(k, a, i, n - i);
    }
}
template <class G>
__device__ __forceinline__ void part_adam(const TensorChunk &k, const AdamFactors &a, int o, int n) {
    if (k.param_type == DD_F32) part_adam<G, float>(k, a, o, n);
    else if (k.param_type == DD_BF16) part_adam<G, bf16_t>(k, a, o, n);
    else part_adam<G, f16_t>(k, a, o, n);
}

__device__ __forceinline__ void adam_share(const TensorChunk *ck, int64_t b, int split, const AdamFactors &a) {
    const TensorChunk k = ck[b >> split];
    for (int o = (int)(b & ((1 << split) - 1)) * kPartLen; o < k.n; o += kPartLen << split) {
        const int n = k.n < o + kPartLen ? k.n : o + kPartLen;
        if (k.grad_type == DD_F32) part_adam<float>(k, a, o, n);
        else if (k.grad_type == DD_BF16) part_adam<bf16_t>(k, a, o, n);
        else part_adam<f16_t>(k, a, o, n);
    }
}

// The factors of a step, once for all workgroups, and the step's number.
__global__ void k_adam_begin(int64_t *step, const float *stats, AdamParams p, AdamFactors *out) {
    AdamFactors a = {};
    a.skip = stats && stats[2] != 0.0f;
    if (!a.skip) a = adam_factors(p, *step += 1, stats);
    *out = a;
}
__global__ void __launch_bounds__(kBlock) k_adam(const TensorChunk *ck, int64_t n_shares, int split,
                                                 const AdamFactors *factors) {
    const AdamFactors a = *factors;
    if (a.skip) return;
    for (int64_t b = blockIdx.x; b < n_shares; b += gridDim.x) adam_share(ck, b, split, a);
}

// Small lists: one launch, in which every workgroup finds the factors itself,
// and the one that finishes last counts the step.  By then all others have
// read its number: each takes its ticket after it has used the number, and
// only the last ticket is followed by the write.
__global__ void __launch_bounds__(kBlock) k_adam_small(const TensorChunk *ck, int64_t n_shares, int split, int64_t *step,
                                                       const float *stats, AdamParams p, uint32_t *ticket) {
    if (stats && stats[2] != 0.0f) return;
    const int64_t t = __hip_atomic_load(step, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) + 1;
    const AdamFactors a = adam_factors(p, t, stats);
    if (blockIdx.x < n_shares) adam_share(ck, blockIdx.x, split, a);
    __syncthreads();
    if (threadIdx.x == 0 && last_ticket(ticket)) {
        *step = t;
        *ticket = 0;
    }
}

constexpr int64_t kMaxGrid = 1 << 22;     // workgroups of a launch; shares beyond go round

// Workgroups of the norm: four chunks each, at least 256 (one per compute
// unit), at most kNormParts: each ticket is 12 ns, one after the other (1,000
// tensors of 300 elements or fewer: 7.5 us with 256, 15.6 with 1,024).
int norm_grid(int n_chunks) {
    const int g = n_chunks / 4 < 256 ? 256 : n_chunks / 4 < kNormParts ? n_chunks / 4 : kNormParts;
    return n_chunks < 1 ? 1 : n_chunks < g ? n_chunks : g;
}
unsigned grid_of(int64_t shares) { return (unsigned)(shares < kMaxGrid ? shares : kMaxGrid); }

}  // namespace

hipError_t launch_tensor_chunks(const TensorPlace *p, int count, const dd_tensors *t, hipStream_t s) {
    const int64_t grid = ((int64_t)t->n_chunks + kBlock - 1) / kBlock;
    k_tensor_chunks<<<grid < 1 ? 1 : (unsigned)grid, kBlock, 0, s>>>(p, count, t->chunks, t->n_chunks, &t->work->ticket);
    return hipGetLastError();
}

hipError_t launch_grad_norm(const dd_tensors *t, double max_norm, const float *inv_scale, float *stats, hipStream_t s) {
    k_grad_norm<<<norm_grid(t->n_chunks), kBlock, 0, s>>>(t->chunks, t->n_chunks, t->work->part, &t->work->ticket, max_norm, inv_scale, stats);
    return hipGetLastError();
}

hipError_t launch_grad_clip(const dd_tensors *src, const dd_tensors *dst, const float *stats, hipStream_t s) {
    const int64_t parts = (int64_t)src->n_chunks * kPartsOf;
    if (parts == 0) return hipSuccess;
    k_grad_clip<<<grid_of(parts), kBlock, 0, s>>>(src->chunks, dst->chunks, parts, stats);
    return hipGetLastError();
}

hipError_t launch_adam(const dd_tensors *t, int64_t *step, const float *stats, const AdamParams &p, hipStream_t s) {
    const int split = split_of(t);
    const int64_t shares = (int64_t)t->n_chunks << split;
    if (shares <= kSmallShares) {
        k_adam_small<<<shares < 1 ? 1 : (unsigned)shares, kBlock, 0, s>>>(t->chunks, shares, split, step, stats, p, &t->work->ticket);
    } else {
        k_adam_begin<<<1, 1, 0, s>>>(step, stats, p, &t->work->factors);
        k_adam<<<grid_of(shares), kBlock, 0, s>>>(t->chunks, shares, split, &t->work->factors);
    }
    return hipGetLastError();
}

}  // namespace dd
