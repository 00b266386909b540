// Products of matrices of 16 bits with 32-bit sums and what follows them fused
// into their epilogue (dd_linear), the products of its gradient, sums over rows
// and the derivative of an activation.
//
//   z = x w + bias,  y = act(z) + residual
//   dx = (dy w^T) * act'(in_z),  dw = x^T dy,  db = sum over rows of dy
//
// All three products are out(i, j) = sum over l of p(i, l) q(l, j), with operands that
// lie by their rows (l is consecutive) or by their sums (i or j is).
#include "dd_product.h"

namespace dd {

namespace {

// The parts of a product whose sums were cut, joined in order.  Bound: the last cache, which holds the parts that were
// just written (4 of 2,048 x 2,048, written and read: 17 us, launch included), or latency.
template <class T>
__global__ void __launch_bounds__(256) k_product_join(Product a, const float *part, int splits) {
    const int64_t packs = (a.n + 7) / 8, total = packs * a.m;
    for (int64_t t = blockIdx.x * (int64_t)256 + threadIdx.x; t < total; t += (int64_t)gridDim.x * 256) {
        const int64_t i = t / packs, j = (t - i * packs) * 8;
        const int have = a.n - j >= 8 ? 8 : (int)(a.n - j);
        const float *p = part + i * a.n + j;
        float v[8] = {}, bias[8];
        Pack<T, 8> side;
        load_bias<T>(a.e, j, have, bias);
        load_side<T>(a.e, i, j, have, side);
        for (int s = 0; s < splits; s += 8) {       // (eight loads at a time)
            Pack<float, 8> b[8];
#pragma unroll
            for (int u = 0; u < 8; u++) b[u].load(p + (s + u) * a.m * a.n, s + u < splits ? have : 0);
#pragma unroll
            for (int u = 0; u < 8; u++) {
                float x[8];
                b[u].to(x);
#pragma unroll
                for (int c = 0; c < 8; c++) v[c] += x[c];
            }
        }
        finish<T>(a.e, i, j, have, v, bias, side);
    }
}

// --- which tiles, and how sums are cut -------------------------------------------
int64_t tiles_of(int64_t x, int64_t n) { return (x + n - 1) / n; }
constexpr int64_t kMostApart = int64_t(1) << 22;        // a workgroup of 512 threads each: a launch has fewer than 2^32

// Tile and parts that are expected to take least (us).  A step of 64 sums of a tile takes 1.44 with 256 x 256
// and 0.53 with 128 x 128 where all compute units have one, and down to 1.0 and 0.4 where few do (1.05 with operands of
// any alignment); what comes after, the epilogue, 11 and 3.4.  Measured, from x k to 8,192 x 8,192 bf16, in us a round of 256
// tiles: 256 x 256 k 64 12.5, 512 23.2, 1,024 34.0; 128 x 128 4.6, 7.6, 11.2.  Where waves share
// the sums of 64 x 64, a wave's step takes 0.75 of four waves and the end 3 (k 64 3.8, 1,024 6.1; of
// any alignment 2.5 of eight waves, and 5.5).  Joining parts takes another launch, and their bytes come from the
// caches (4 parts of 2,048 x 2,048 17, 16 of 1,024 x 1,024 15).
Plan plan_of(int64_t m, int64_t n, int64_t k, bool p_rows, bool direct) {
    Plan p{0, 0, 0, 1, 0, 0.0};
    const int64_t steps = tiles_of(k, 64) > 0 ? tiles_of(k, 64) : 1;
    for (int tile : {256, 128, 64, 16}) {
        if ((tile == 256 && !direct) || (tile == 16 && (m > 16 || !p_rows))) continue;
        const int64_t tm = tiles_of(m, tile), tn = tiles_of(n, tile <= 64 ? 64 : tile);
        const int64_t waves = tile == 16 ? 8 : tile == 64 ? (direct ? kApart<true> : kApart<false>) : 1;
        const int64_t turns = tiles_of(steps, waves);
        for (int64_t s = 1; s <= turns && (s == 1 || tm * tn * s < 4 * kUnits); s += s < 8 ? 1 : s / 4) {
            const int64_t each = tiles_of(turns, s) * waves, parts = tiles_of(steps, each), tiles = tm * tn * parts;
            if (tile <= 64 && tiles >= kMostApart) break;
            const int64_t rounds = tiles_of(tiles, kUnits);
            const double busy = tiles < kUnits ? (double)tiles / kUnits : 1.0;
            double us = tile == 256 ? each * (1.0 + 0.44 * busy) + 11.0 : tile == 128 ? each * (direct ? 0.4 + 0.13 * busy : 1.05) + 3.4
                      : each / waves * (direct ? 0.75 : 2.5) + (direct ? 3.0 : 5.5);
            us *= (double)rounds;
            if (parts > 1) us += 4.0 + (0.1 + 0.8e-6 * (double)m * (double)n) * (double)parts;
            if (p.tile && us >= p.us) continue;
            p = Plan{tile, (int)tm, (int)tn, (int)parts, each * 64, us};
        }
    }
    return p;
}

size_t plan_work(const Plan &p, int64_t m, int64_t n) { return p.splits > 1 ? (size_t)p.splits * (size_t)m * (size_t)n * sizeof(float) : 0; }

// An operand that loads go to LDS directly from: 16 bytes in a row lie aligned, all of
// one row (or one l), and a tile spans less than 2 GiB, the reach of a load's offset.
constexpr int64_t kReach = int64_t(1) << 22;        // of strides, in elements
bool aligned_operand(const void *p, int64_t stride, bool by_rows, int64_t count, int64_t k, bool padded) {
    return reinterpret_cast<uintptr_t>(p) % 16 == 0 && stride % 8 == 0 && (padded || (by_rows ? k : count) % 8 == 0) && stride < kReach;
}
// so is a copy, of rows of that length
bool copy_reaches(int64_t cols) { return tiles_of(cols, 8) * 8 < kReach; }

// --- sums over few rows -----------------------------------------------------------
__device__ __forceinline__ void store_as(void *p, int32_t type, int64_t i, float x) {
    if (type == DD_F32) static_cast<float *>(p)[i] = x;
    else if (type == DD_BF16) static_cast<bf16_t *>(p)[i] = (bf16_t)x;
    else static_cast<f16_t *>(p)[i] = (f16_t)x;
}

// Up to 4,096 rows in one launch: a workgroup has 64 columns, 128 rows at a time.  Bound: latency.  1,021 x 1,237
// f16 6 us; with parts two launches, 9.
constexpr int kFewRows = 4096;
typedef float FewRoom[128][65];
template <class T>
__device__ __forceinline__ void sum_few(const FewSums &a, int64_t block, FewRoom &lds) {
    const T *x = static_cast<const T *>(a.x);
    const int64_t stride = a.stride, cols = a.cols;
    const int rows = a.rows;
    const int cx = threadIdx.x % 8, cy = threadIdx.x / 8;
    const int64_t c = block * 64 + 8 * cx;
    const int have = cols - c >= 8 ? 8 : cols - c < 0 ? 0 : (int)(cols - c);
    float s[8] = {};
    for (int r = cy; r < rows; r += 512) {
        Pack<T, 8> p[4];
#pragma unroll
        for (int i = 0; i < 4; i++) p[i].load(x + (r + i * 128) * stride + c, r + i * 128 < rows ? have : 0);
#pragma unroll
        for (int i = 0; i < 4; i++) {
            float v[8];
            p[i].to(v);
#pragma unroll
            for (int j = 0; j < 8; j++) s[j] += v[j];
        }
    }
#pragma unroll
    for (int j = 0; j < 8; j++) lds[cy][8 * cx + j] = s[j];
    __syncthreads();
    const int y = threadIdx.x / 64, mine = threadIdx.x % 64;
    float t = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; i++) t += lds[y * 8 + i][mine];
    __syncthreads();
    lds[y][mine] = t;
    __syncthreads();
    if (y || block * 64 + mine >= cols) return;
    t = 0.0f;
#pragma unroll
    for (int i = 0; i < 16; i++) t += lds[i][mine];
    store_as(a.out, a.out_type, block * 64 + mine, t);
}
__device__ __forceinline__ void sum_few(const FewSums &a, int64_t block, FewRoom &lds) {
    if (a.type == DD_BF16) sum_few<bf16_t>(a, block, lds);
    else sum_few<f16_t>(a, block, lds);
}
__global__ void __launch_bounds__(1024) k_column_sum_few(FewSums a) {
    __shared__ FewRoom lds;
    sum_few(a, blockIdx.x, lds);
}

// --- operands of odd sizes --------------------------------------------------------
// Rows that are not multiples of 16 bytes cannot be loaded to LDS directly, which makes a step half as fast and
// more.  So operands are copied first, rows padded with zeros to 16 bytes, if that is expected to take less than it
// gains (4,099 x 1,237 -> 777 f16 29 us, of which the copies 8; 32 without.  A weight of
// 15,219 x 3,471 bf16 is not copied for 139 rows: 45 us).  Sums over few rows are taken by workgroups of the same
// launch (1,021 rows of 777 x 1,237 f16, all gradients: 5 us less than with a launch of their own).
__global__ void __launch_bounds__(1024) k_pad_rows(PadRows x, PadRows y, PadRows z, FewSums sums) {
    __shared__ FewRoom lds;
    const int which = (int)blockIdx.y - (sums.cols ? 1 : 0);
    if (which < 0) {        // (first: they take longest)
        if ((int64_t)blockIdx.x * 64 < sums.cols) sum_few(sums, blockIdx.x, lds);
        return;
    }
    const PadRows &r = which == 0 ? x : which == 1 ? y : z;
    const int64_t packs = (r.cols + 7) / 8, total = packs * r.rows;
    const bf16_t *from = static_cast<const bf16_t *>(r.from);       // (16 bits, whatever they mean)
    for (int64_t t = blockIdx.x * (int64_t)1024 + threadIdx.x; t < total; t += (int64_t)gridDim.x * 1024) {
        const int64_t i = (uint64_t)total >> 32 ? t / packs : (int64_t)((uint32_t)t / (uint32_t)packs), j = (t - i * packs) * 8;
        Pack<bf16_t, 8> v;
        v.load(from + i * r.stride + j, r.cols - j >= 8 ? 8 : (int)(r.cols - j));
        v.store(static_cast<bf16_t *>(r.to) + t * 8);
    }
}
// Whether operands may be copied: always for odd sizes; where only strides or addresses are in the way, which the size of
// the working memory does not know, up to kMostCopied bytes (249 rows of 14,400 x 1,136 bf16 at odd strides, all
// gradients: 56 us, 62 through registers).
constexpr int64_t kMostCopied = int64_t(64) << 20;
bool pads(int64_t m, int64_t n, int64_t k) {
    if (m <= 64 || n <= 64) return false;
    return m % 8 || n % 8 || k % 8 || (double)(m + n) * (double)k * 2.0 <= (double)kMostCopied;
}
double copy_us(size_t bytes) { return (double)bytes * (2.0 / 4.5e6); }
constexpr double kLaunch = 2.5;
size_t pad_work(int64_t m, int64_t n, int64_t k) {       // (of either layout)
    auto most = [&](int64_t i) {
        const int64_t by_rows = copy_reaches(k) ? i * tiles_of(k, 8) : 0, by_sums = copy_reaches(i) ? k * tiles_of(i, 8) : 0;
        return by_rows > by_sums ? by_rows : by_sums;
    };
    return pads(m, n, k) ? (size_t)(most(m) + most(n)) * 16 : 0;
}

// How a product runs: which operands are copied, and the plan.
struct Way {
    bool copy_p, copy_q, direct;
    Plan plan;
};
double apart_us(int64_t k) { return (double)tiles_of(tiles_of(k, 64), kApart<true>) * 0.75 + 3.0; }
Way way_of(const Product &a) {
    const bool ap = aligned_operand(a.p, a.p_stride, a.p_by_rows, a.m, a.k, a.padded & 1);
    const bool aq = aligned_operand(a.q, a.q_stride, a.q_by_rows, a.n, a.k, a.padded & 2);
    Plan direct = plan_of(a.m, a.n, a.k, a.p_by_rows, true);
    if (a.small) {
        const int64_t tm = tiles_of(a.m, 64), tn = tiles_of(a.n, 64);
        direct = Plan{64, (int)tm, (int)tn, 1, tiles_of(a.k, 64) * 64, (double)tiles_of(tm * tn, kUnits) * apart_us(a.k)};
    }
    if ((ap && aq) || a.k == 0) return Way{false, false, true, direct};     // (no sums: nothing is loaded)
    const Plan any = plan_of(a.m, a.n, a.k, a.p_by_rows, false);
    const size_t bytes = (size_t)((ap ? 0 : a.m) + (aq ? 0 : a.n)) * (size_t)a.k * 2;
    const bool reach = (ap || copy_reaches(a.p_by_rows ? a.k : a.m)) && (aq || copy_reaches(a.q_by_rows ? a.k : a.n));
    if (reach && pads(a.m, a.n, a.k) && direct.us + kLaunch + copy_us(bytes) < any.us) return Way{!ap, !aq, true, direct};
    return Way{false, false, false, any};
}
size_t up16(size_t x) { return (x + 15) / 16 * 16; }

template <class T>
hipError_t product(const Product &args, char *work, hipStream_t s) {
    Product a = args;
    const Way way = way_of(a);
    const Plan &p = way.plan;
    float *part = reinterpret_cast<float *>(work);
    if (way.copy_p || way.copy_q) {
        char *to = work + up16(plan_work(p, a.m, a.n));
        PadRows x{}, y{};
        if (way.copy_p) to += pad_rows(a.p, a.p_stride, a.p_by_rows ? a.m : a.k, a.p_by_rows ? a.k : a.m, to, &x);
        if (way.copy_q) pad_rows(a.q, a.q_stride, a.q_by_rows ? a.n : a.k, a.q_by_rows ? a.k : a.n, to, way.copy_p ? &y : &x);
        const hipError_t e = launch_pad_rows(x, y, PadRows{}, FewSums{}, s);
        if (e != hipSuccess) return e;
    }
    if (way.direct) launch_tiles<T, true>(a, p, part, s);
    else launch_tiles<T, false>(a, p, part, s);
    if (p.splits > 1) {
        const int64_t need = tiles_of(a.m * tiles_of(a.n, 8), 256);
        k_product_join<T><<<(unsigned)(need < 8 * kUnits ? need : 8 * kUnits), 256, 0, s>>>(a, part, p.splits);
    }
    return hipGetLastError();
}

// --- sums over rows, and an activation's derivative -------------------------------
// Workgroup (i, j) has 256 columns and the j-th run of rows, eight rows at a time,
// and writes its sums to part j (a single one: to the output); then 32 threads a
// column join the parts in order.  Bound: HBM.  16,384 x 2,048 bf16 13 us, 5.1 TB/s, and 3 to 5 for the join.
constexpr int kSumParts = 256, kSumCols = 256, kSumRows = 8;

template <class T>
__global__ void __launch_bounds__(kSumCols) k_column_sum(const T *x, int64_t stride, int64_t rows, int64_t cols, int64_t run, void *out, int32_t out_type,
                                                        float *part) {
    __shared__ float lds[kSumRows][kSumCols];
    const int cx = threadIdx.x % (kSumCols / 8), cy = threadIdx.x / (kSumCols / 8);
    const int64_t c = (int64_t)blockIdx.x * kSumCols + 8 * cx;
    const int have = cols - c >= 8 ? 8 : cols - c < 0 ? 0 : (int)(cols - c);
    const int64_t r1 = (blockIdx.y + 1) * run < rows ? (blockIdx.y + 1) * run : rows;
    float s[8] = {};
    int64_t r = blockIdx.y * run + cy;
    for (; r + 3 * kSumRows < r1; r += 4 * kSumRows) {
        Pack<T, 8> p[4];
#pragma unroll
        for (int i = 0; i < 4; i++) p[i].load(x + (r + i * kSumRows) * stride + c, have);
#pragma unroll
        for (int i = 0; i < 4; i++) {
            float v[8];
            p[i].to(v);
#pragma unroll
            for (int j = 0; j < 8; j++) s[j] += v[j];
        }
    }
    for (; r < r1; r += kSumRows) {
        Pack<T, 8> p;
        float v[8];
        p.load(x + r * stride + c, have);
        p.to(v);
#pragma unroll
        for (int j = 0; j < 8; j++) s[j] += v[j];
    }
#pragma unroll
    for (int j = 0; j < 8; j++) lds[cy][8 * cx + j] = s[j];
    __syncthreads();
    const int64_t mine = (int64_t)blockIdx.x * kSumCols + threadIdx.x;
    if (mine >= cols) return;
    float t = 0.0f;
#pragma unroll
    for (int i = 0; i < kSumRows; i++) t += lds[i][threadIdx.x];
    if (gridDim.y > 1) part[blockIdx.y * cols + mine] = t;
    else store_as(out, out_type, mine, t);
}

__global__ void __launch_bounds__(1024) k_column_join(const float *part, int n, int64_t cols, void *out, int32_t out_type) {
    __shared__ float lds[32][33];
    const int x = threadIdx.x & 31, y = threadIdx.x >> 5;
    const int64_t c = (int64_t)blockIdx.x * 32 + x;
    float s = 0.0f;
    if (c < cols) {
        float t[kSumParts / 32];
#pragma unroll
        for (int i = 0; i < kSumParts / 32; i++) t[i] = y + 32 * i < n ? part[(y + 32 * i) * cols + c] : 0.0f;
#pragma unroll
        for (int i = 0; i < kSumParts / 32; i++) s += t[i];
    }
    lds[y][x] = s;
    __syncthreads();
    if (y || c >= cols) return;
    s = 0.0f;
#pragma unroll
    for (int i = 0; i < 32; i++) s += lds[i][x];
    store_as(out, out_type, c, s);
}

// parts of the rows: enough workgroups to fill the card, of 32 rows at least
int sum_parts(int64_t rows, int64_t cols) {
    if (few_rows(rows, cols)) return 1;
    const int64_t blocks = tiles_of(cols, kSumCols);
    int64_t n = tiles_of(4 * kUnits, blocks), most = rows / 32;
    if (n > most) n = most;
    if (n > kSumParts) n = kSumParts;
    return n < 1 ? 1 : (int)n;
}

// Bound: HBM.  16,384 x 8,192 bf16 138 us (ReLU) and 140 (GELU), 5.8 TB/s.
template <class T>
__global__ void __launch_bounds__(256) k_act_grad(dd_act_grad_args a) {
    const int64_t packs = (a.cols + 7) / 8, total = packs * a.rows;
    for (int64_t t = blockIdx.x * (int64_t)256 + threadIdx.x; t < total; t += (int64_t)gridDim.x * 256) {
        const int64_t i = t / packs, j = (t - i * packs) * 8;
        const int have = a.cols - j >= 8 ? 8 : (int)(a.cols - j);
        Pack<T, 8> pd, pz;
        float d[8], z[8];
        pd.load(static_cast<const T *>(a.dy) + i * a.dy_stride + j, have);
        pz.load(static_cast<const T *>(a.z) + i * a.z_stride + j, have);
        pd.to(d);
        pz.to(z);
        by_act(a.act, [&](auto act) {
#pragma unroll
            for (int c = 0; c < 8; c++) d[c] *= slope_of<decltype(act)::value>(z[c]);
        });
        pd.from(d);
        pd.store(static_cast<T *>(a.dz) + i * a.dz_stride + j, have);
    }
}

}  // namespace

size_t pad_rows(const void *&x, int64_t &stride, int64_t rows, int64_t cols, void *to, PadRows *r) {
    *r = PadRows{x, to, stride, rows, cols};
    x = to;
    stride = tiles_of(cols, 8) * 8;
    return padded_size(rows, cols);
}

bool loads_directly(const void *p, int64_t stride, bool by_rows, int64_t count, int64_t k) { return aligned_operand(p, stride, by_rows, count, k, false); }

GradCopies grad_copies(int64_t rows, int64_t k, int64_t n, bool turned, const GradCopies &needed) {
    if (!needed.dy || !grad_copies_work(rows, k, n)) return GradCopies{};
    if ((needed.x && !copy_reaches(k)) || (needed.w && !copy_reaches(turned ? k : n))) return GradCopies{};
    auto us = [&](bool of_dw, bool direct) {
        return of_dw ? plan_of(turned ? n : k, turned ? k : n, rows, false, direct).us : plan_of(rows, k, n, true, direct).us;
    };
    const size_t dy = (size_t)rows * (size_t)n * 2, x = needed.x ? (size_t)rows * (size_t)k * 2 : 0, w = needed.w ? (size_t)k * (size_t)n * 2 : 0;
    auto alone = [&](bool of_dw, size_t bytes) {
        const double any = us(of_dw, false), copied = us(of_dw, true) + kLaunch + copy_us(bytes);
        return any < copied ? any : copied;
    };
    const double apart = alone(true, dy + x) + alone(false, dy + w), both = us(true, true) + kLaunch + copy_us(dy + x);
    const double with_w = both + copy_us(w) + us(false, true), without = both + us(false, !needed.w);
    if (apart <= with_w && apart <= without) return GradCopies{};
    return GradCopies{true, needed.x, needed.w && with_w < without};
}

size_t grad_copies_work(int64_t rows, int64_t k, int64_t n) {
    if (rows <= 64 || k <= 64 || n <= 64 || !copy_reaches(n)) return 0;
    const size_t w = padded_size(k, n), turned = padded_size(n, k), all = padded_size(rows, n) + padded_size(rows, k) + (w > turned ? w : turned);
    return n % 8 || all <= (size_t)kMostCopied ? all : 0;
}

size_t padded_size(int64_t rows, int64_t cols) { return (size_t)rows * (size_t)tiles_of(cols, 8) * 16; }

bool few_rows(int64_t rows, int64_t cols) { return rows <= kFewRows && cols < (int64_t(1) << 27); }     // (16 threads a column)

hipError_t launch_pad_rows(const PadRows &x, const PadRows &y, const PadRows &z, const FewSums &sums, hipStream_t s) {
    int64_t most = 1;
    for (const PadRows *r : {&x, &y, &z}) most = tiles_of(tiles_of(r->cols, 8) * r->rows, 1024) > most ? tiles_of(tiles_of(r->cols, 8) * r->rows, 1024) : most;
    most = most < 2 * kUnits ? most : 2 * kUnits;
    if (tiles_of(sums.cols, 64) > most) most = tiles_of(sums.cols, 64);
    k_pad_rows<<<dim3((unsigned)most, (z.rows ? 3 : y.rows ? 2 : 1) + (sums.cols ? 1 : 0)), 1024, 0, s>>>(x, y, z, sums);
    return hipGetLastError();
}

size_t product_work(int64_t m, int64_t n, int64_t k, bool p_rows) {
    const size_t a = up16(plan_work(plan_of(m, n, k, p_rows, true), m, n)) + pad_work(m, n, k), b = plan_work(plan_of(m, n, k, p_rows, false), m, n);
    return a > b ? a : b;
}

size_t product_need(const Product &a) {
    const Way way = way_of(a);
    const size_t parts = plan_work(way.plan, a.m, a.n);
    if (!way.copy_p && !way.copy_q) return parts;
    return up16(parts) + (way.copy_p ? padded_size(a.p_by_rows ? a.m : a.k, a.p_by_rows ? a.k : a.m) : 0) +
           (way.copy_q ? padded_size(a.q_by_rows ? a.n : a.k, a.q_by_rows ? a.k : a.n) : 0);
}

bool product_fits(int64_t m, int64_t n, int64_t k, bool p_rows) {
    for (bool direct : {true, false}) {       // (tiles are counted in 32 bits)
        const Plan p = plan_of(m, n, k, p_rows, direct);
        if ((int64_t)p.tm * p.tn * p.splits >= (int64_t(1) << 30)) return false;
    }
    return true;
}

// (the longer of the two decides how long a round of workgroups takes, and a launch is saved)
bool small_gradients(int64_t rows, int64_t k, int64_t n, bool turned) {
    const int64_t wr = turned ? n : k, wc = turned ? k : n, tiles = tiles_of(wr, 64) * tiles_of(wc, 64) + tiles_of(rows, 64) * tiles_of(k, 64);
    return tiles < 4 * kUnits && (double)tiles_of(tiles, kUnits) * apart_us(rows > n ? rows : n) < plan_of(wr, wc, rows, false, true).us + plan_of(rows, k, n, true, true).us + kLaunch;
}

bool goes_together(const Product &dw, const Product &dx) {
    const Way w = way_of(dw), x = way_of(dx);
    return dw.small && dx.small && w.direct && x.direct && !w.copy_p && !w.copy_q && !x.copy_p && !x.copy_q;
}

hipError_t launch_together(const Product &dw, const Product &dx, hipStream_t s) {
    if (dw.type == DD_BF16) launch_two<bf16_t>(dw, dx, s);
    else launch_two<f16_t>(dw, dx, s);
    return hipGetLastError();
}

hipError_t launch_product(const Product &p, void *work, hipStream_t s) {
    return p.type == DD_BF16 ? product<bf16_t>(p, static_cast<char *>(work), s) : product<f16_t>(p, static_cast<char *>(work), s);
}

size_t column_sum_work(int64_t rows, int64_t cols) {
    const int n = sum_parts(rows, cols);
    return n > 1 ? (size_t)n * (size_t)cols * sizeof(float) : 0;
}

hipError_t launch_column_sum(const void *x, int64_t stride, int64_t rows, int64_t cols, int32_t type, void *out, int32_t out_type, void *work,
                             hipStream_t s) {
    if (few_rows(rows, cols)) {
        k_column_sum_few<<<(unsigned)tiles_of(cols, 64), 1024, 0, s>>>(FewSums{x, out, stride, cols, (int32_t)rows, type, out_type});
        return hipGetLastError();
    }
    const int n = sum_parts(rows, cols);
    const int64_t run = tiles_of(rows, n);
    float *part = static_cast<float *>(work);
    const dim3 grid((unsigned)tiles_of(cols, kSumCols), (unsigned)n);
    if (type == DD_BF16) k_column_sum<bf16_t><<<grid, kSumCols, 0, s>>>(static_cast<const bf16_t *>(x), stride, rows, cols, run, out, out_type, part);
    else k_column_sum<f16_t><<<grid, kSumCols, 0, s>>>(static_cast<const f16_t *>(x), stride, rows, cols, run, out, out_type, part);
    if (n > 1) k_column_join<<<(unsigned)tiles_of(cols, 32), 1024, 0, s>>>(part, n, cols, out, out_type);
    return hipGetLastError();
}

hipError_t launch_act_grad(const dd_act_grad_args &a, hipStream_t s) {
    const int64_t need = tiles_of(a.rows * tiles_of(a.cols, 8), 256);
    const unsigned grid = (unsigned)(need < (1 << 16) ? need : (1 << 16));
    if (a.type == DD_F32) k_act_grad<float><<<grid, 256, 0, s>>>(a);
    else if (a.type == DD_BF16) k_act_grad<bf16_t><<<grid, 256, 0, s>>>(a);
    else k_act_grad<f16_t><<<grid, 256, 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace dd
