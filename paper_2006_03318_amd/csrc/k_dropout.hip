// Dropout from a counter-based generator: the mask is made where it is used,
// forward and backward, and never stored.
//
//   out = residual + (kept(i) ? x / (1 - q) : 0),  q = a number of 65,536ths
//
// Eight elements share one call of Philox 4x32-10 (J. Salmon, M. Moraes, R. Dror,
// D. Shaw: Parallel random numbers: as easy as 1, 2, 3; SC 2011): its four words
// are eight numbers of 16 bits.
#include "dd_elem.h"
#include "dd_layers.h"

namespace dd {

namespace {

struct Words {
    uint32_t w[4];
    __device__ __forceinline__ uint32_t half(int i) const { return i & 1 ? w[i >> 1] >> 16 : w[i >> 1] & 0xffff; }
};

__device__ __forceinline__ Words philox(uint64_t i, uint64_t c, uint64_t key) {
    uint32_t c0 = (uint32_t)i, c1 = (uint32_t)(i >> 32), c2 = (uint32_t)c, c3 = (uint32_t)(c >> 32);
    uint32_t k0 = (uint32_t)key, k1 = (uint32_t)(key >> 32);
#pragma unroll
    for (int r = 0; r < 10; r++) {
        const uint64_t a = (uint64_t)c0 * 0xD2511F53u, b = (uint64_t)c2 * 0xCD9E8D57u;
        c0 = (uint32_t)(b >> 32) ^ c1 ^ k0;
        c1 = (uint32_t)b;
        c2 = (uint32_t)(a >> 32) ^ c3 ^ k1;
        c3 = (uint32_t)a;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return {{c0, c1, c2, c3}};
}

// Where the eight elements from number 8 i on lie: in a row (FLAT: all of the array
// is one), in one row of several (ROWS: cols is a multiple of 8), or (ANY) at the end of one row and the
// beginning of others too.
enum { FLAT, ROWS, ANY };

template <int WHERE>
struct At {
    int64_t first, row, col;
    const dd_dropout_args &a;
    __device__ __forceinline__ At(const dd_dropout_args &args, int64_t i) : first(8 * i), row(0), col(8 * i), a(args) {
        if (WHERE != FLAT) {
            row = (uint64_t)first >> 32 || (uint64_t)a.cols >> 32 ? first / a.cols : (int64_t)((uint32_t)first / (uint32_t)a.cols);
            col = first - row * a.cols;
        }
    }
    template <class T>
    __device__ __forceinline__ void load(const T *p, int64_t stride, int have, Pack<T, 8> &v) const {
        if (WHERE != ANY || col + have <= a.cols) {
            v.load(p + row * stride + col, have);
            return;
        }
        int64_t r = row, c = col;
#pragma unroll
        for (int i = 0; i < 8; i++) {
            v.v[i] = i < have ? global(p)[r * stride + c] : (T)0.0f;
            if (++c == a.cols) {
                c = 0;
                r++;
            }
        }
    }
    template <class T>
    __device__ __forceinline__ void store(T *p, int64_t stride, int have, const Pack<T, 8> &v) const {
        if (WHERE != ANY || col + have <= a.cols) {
            v.store(p + row * stride + col, have);
            return;
        }
        int64_t r = row, c = col;
#pragma unroll
        for (int i = 0; i < 8; i++) {
            if (i < have) global(p)[r * stride + c] = v.v[i];
            if (++c == a.cols) {
                c = 0;
                r++;
            }
        }
    }
};

// Bound: HBM; ten rounds of two products each cost less than the bytes.  16,384 x 2,048 bf16 into a residual
// 37.5 us, 5.4 TB/s; 4,099 x 1,237 f32 of strided rows 9.2, 4.4 TB/s (20 with every element on its own).
template <class T, int WHERE>
__global__ void __launch_bounds__(256) k_dropout(dd_dropout_args a, uint32_t gone, float scale) {
    const uint64_t key = a.d_state[0], c = a.d_state[1] + a.call;
    if (a.d_used && blockIdx.x == 0 && threadIdx.x == 0) {
        a.d_used[0] = key;
        a.d_used[1] = c;
    }
    const int64_t n = a.rows * a.cols, packs = (n + 7) / 8;
    for (int64_t i = blockIdx.x * (int64_t)256 + threadIdx.x; i < packs; i += (int64_t)gridDim.x * 256) {
        const int have = n - 8 * i >= 8 ? 8 : (int)(n - 8 * i);
        const At<WHERE> at(a, i);
        Pack<T, 8> px, pr;
        at.load(static_cast<const T *>(a.x), a.x_stride, have, px);
        if (a.residual) at.load(static_cast<const T *>(a.residual), a.residual_stride, have, pr);
        const Words w = philox((uint64_t)i, c, key);
        float x[8], r[8] = {};
        px.to(x);
        if (a.residual) pr.to(r);
#pragma unroll
        for (int j = 0; j < 8; j++) r[j] += w.half(j) >= gone ? x[j] * scale : 0.0f;
        px.from(r);
        at.store(static_cast<T *>(a.out), a.out_stride, have, px);
    }
}

template <class T>
void dropout(const dd_dropout_args &a, hipStream_t s) {
    const uint32_t gone = (uint32_t)rint(a.p * 65536.0);        // (65,536: no half is that large)
    const float scale = gone < 65536 ? 65536.0f / (float)(65536 - gone) : 0.0f;
    const int64_t packs = (a.rows * a.cols + 7) / 8, need = (packs + 255) / 256;
    const unsigned grid = (unsigned)(need < 1 ? 1 : need < (1 << 16) ? need : (1 << 16));      // (no rows: d_used)
    const bool flat = a.rows == 1 || (a.x_stride == a.cols && a.out_stride == a.cols && (!a.residual || a.residual_stride == a.cols));
    if (flat) k_dropout<T, FLAT><<<grid, 256, 0, s>>>(a, gone, scale);
    else if (a.cols % 8 == 0) k_dropout<T, ROWS><<<grid, 256, 0, s>>>(a, gone, scale);
    else k_dropout<T, ANY><<<grid, 256, 0, s>>>(a, gone, scale);
}

}  // namespace

hipError_t launch_dropout(const dd_dropout_args &a, hipStream_t s) {
    if (a.type == DD_F32) dropout<float>(a, s);
    else if (a.type == DD_BF16) dropout<bf16_t>(a, s);
    else dropout<f16_t>(a, s);
    return hipGetLastError();
}

}  // namespace dd
