// Products of matrices of 16 bits with 32-bit sums and what follows them fused
// into their epilogue (dd_linear), the products of its gradient, sums over rows
// and the derivative of an activation.
//
//   z = x w + bias,  y = act(z) + residual
//   dx = (dy w^T) * act'(in_z),  dw = x^T dy,  db = sum over rows of dy
//
// All three products are out(i, j) = sum over l of p(i, l) q(l, j), with operands that
// lie by their rows (l is consecutive) or by their sums (i or j is).
#include <type_traits>

#include "dd_elem.h"
#include "dd_layers.h"

namespace dd {

namespace {

typedef float f4 __attribute__((ext_vector_type(4)));
typedef int i4 __attribute__((ext_vector_type(4)));
typedef short s4 __attribute__((ext_vector_type(4)));
typedef short s8 __attribute__((ext_vector_type(8)));
typedef bf16_t bf16x8 __attribute__((ext_vector_type(8)));
typedef f16_t f16x8 __attribute__((ext_vector_type(8)));

template <class V>
using lptr = __attribute__((address_space(3))) V *;

__device__ __forceinline__ f4 mfma(bf16_t, s8 a, s8 b, f4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
__device__ __forceinline__ f4 mfma(f16_t, s8 a, s8 b, f4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

// --- activations --------------------------------------------------------------
// Phi(x) and exp(-x^2 / 2), from Abramowitz and Stegun 7.1.26 (off by 1.5e-7
// at most).
__device__ __forceinline__ void normal(float x, float &phi, float &e) {
    const float a = fabsf(x) * 0.70710678f;
    const float t = __builtin_amdgcn_rcpf(fmaf(0.3275911f, a, 1.0f));
    e = __builtin_amdgcn_exp2f(a * a * -1.44269504f);
    const float s = t * fmaf(t, fmaf(t, fmaf(t, fmaf(t, 0.5f * 1.061405429f, 0.5f * -1.453152027f), 0.5f * 1.421413741f),
                                     0.5f * -0.284496736f), 0.5f * 0.254829592f) * e;
    phi = x < 0.0f ? s : 1.0f - s;
}
__device__ __forceinline__ float sigmoid(float x) {
    return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(x * -1.44269504f));
}
template <int ACT>
__device__ __forceinline__ float act_of(float z) {
    if (ACT == DD_ACT_RELU) return z > 0.0f || z != z ? z : 0.0f;
    if (ACT == DD_ACT_GELU) {
        float phi, e;
        normal(z, phi, e);
        return z * phi;
    }
    if (ACT == DD_ACT_GELU_TANH) return z * sigmoid(z * fmaf(2.0f * 0.7978845608f * 0.044715f, z * z, 2.0f * 0.7978845608f));
    if (ACT == DD_ACT_SILU) return z * sigmoid(z);
    return z;
}
template <int ACT>
__device__ __forceinline__ float slope_of(float z) {
    if (ACT == DD_ACT_RELU) return z > 0.0f ? 1.0f : 0.0f;
    if (ACT == DD_ACT_GELU) {
        float phi, e;
        normal(z, phi, e);
        return fmaf(z * e, 0.3989422804f, phi);
    }
    if (ACT == DD_ACT_GELU_TANH) {
        const float x = z > 20.0f ? 20.0f : z < -20.0f ? -20.0f : z;     // (x^2 in range; the slope is 0 or 1 there)
        const float s = sigmoid(x * fmaf(2.0f * 0.7978845608f * 0.044715f, x * x, 2.0f * 0.7978845608f));
        return fmaf(x * s * (1.0f - s), fmaf(6.0f * 0.7978845608f * 0.044715f, x * x, 2.0f * 0.7978845608f), s);
    }
    if (ACT == DD_ACT_SILU) {
        const float s = sigmoid(z);
        return s * fmaf(z, 1.0f - s, 1.0f);
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

// --- tiles in LDS -----------------------------------------------------------------
// N rows (or columns) of BK sums each, as lines of 16-byte chunks: by rows, a
// line is a row (BK / 8 chunks); by sums, a line is one l (N / 8 chunks).  Loads
// to LDS write 1,024 bytes in a row, so a chunk's place within its line is
// permuted by choosing which lane loads it: place = chunk ^ turn(line), so that
// the sixteen rows a wave reads at once lie in different banks.
//   The rows of q are taken in another order (TURN): of 32 rows the matrix
// instructions s = 0, 1 have 8 a + 4 s + b as their row 4 a + b, so that a lane's
// sums are eight consecutive columns.
template <bool ROWS, bool TURN, int N, int BK>
struct Tile {
    static constexpr int kLine = ROWS ? BK / 8 : N / 8;         // chunks
    static constexpr int kBytes = N * BK * 2, kLoads = kBytes / 1024;
    static_assert(kBytes % 1024 == 0 && kLine <= 64, "tile");
    static __device__ __forceinline__ int turn(int line) {
        if (ROWS && BK == 64) return TURN ? (line >> 1 & 1) | (line >> 3 & 3) << 1 : line >> 1 & 7;
        if (ROWS) return TURN ? line >> 3 & 3 : line >> 2 & 3;
        if (TURN) return ((line & 3) | (line >> 3 & 1) << 2) << 2 & (kLine - 1);
        return ((line & 3) | (line >> 3 & 3) << 2) << 1 & (kLine - 1);
    }
    // row and first sum of the chunk that a lane loads in load number i
    static __device__ __forceinline__ void source(int i, int lane, int &row, int &l) {
        const int line = i * (64 / kLine) + lane / kLine, c = lane % kLine ^ turn(line);
        row = ROWS ? line : 8 * c;
        l = ROWS ? 8 * c : line;
    }
    // Fragments: 16 rows (TURN: matrix instruction s of 32) of sums 32 h to 32 h + 31; a lane gets row lane %
    // 16, sums 8 (lane / 16) and on.  They are numbered from the wave's first row on, which is a
    // multiple of all their rows; base() is the lane's place in the first.  A later one's place differs by a
    // constant or, where chunks are permuted by more than the line, in a few bits.
    static __device__ __forceinline__ uint32_t base(int lane, int first) {
        const int r = lane & 15, g = lane >> 4;
        if (ROWS) {
            const int line = first + (TURN ? (r >> 2) * 8 + (r & 3) : r);
            return line * (BK * 2) + (g ^ turn(line)) * 16;
        }
        // read and transposed: lane 4 a + b of sixteen gives four rows' values of one sum, and
        // gets those of four sums for its row
        const int line = 8 * g + (r >> 2), row = first + (TURN ? 8 : 4) * (r & 3);
        return line * (N * 2) + ((row >> 3) ^ turn(line)) * 16 + (row & 7) * 2;
    }
    static __device__ __forceinline__ s8 fragment(uint32_t at, int i, int s, int h) {
        if (ROWS) {
            const uint32_t p = (at ^ h * 64) + (TURN ? i * 32 + s * 4 : i * 16) * (BK * 2);
            return *(lptr<const s8>)(uintptr_t)(p);
        }
        const uint32_t p = (at ^ i * (TURN ? 64 : 32)) + h * 32 * (N * 2) + s * 8;
        const s4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lptr<s4>)(uintptr_t)(p));
        const s4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lptr<s4>)(uintptr_t)(p + 4 * (N * 2)));
        return s8{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
    }
};

// x, about which the compiler forgets what it knows: what is made of it is not kept
// in registers from before a loop.
__device__ __forceinline__ int fresh(int x) {
    asm volatile("" : "+v"(x));
    return x;
}

// A wave's loads of one operand's tiles.  DIRECT: to LDS, without registers; the
// operand is aligned to 16 bytes, and rows beyond its end and sums beyond l are read at
// an offset that the buffer does not have, which gives zeros.  Else in registers,
// of any alignment, and from there to LDS.
template <class T, class TILE, bool ROWS, int WAVES, bool DIRECT>
struct Loads {
    static constexpr int kCount = (TILE::kLoads + WAVES - 1) / WAVES;      // (some twice, where they do not go round)
    uint32_t off[DIRECT ? kCount : 1];
    Pack<T, 8> v[DIRECT ? 1 : kCount];
    const T *base;               // of the tile's first row, at l = 0
    int64_t stride;
    int rows, lane, wave;        // rows: that the operand has from the tile's first on

    static __device__ __forceinline__ int number(int wave, int j) {
        return kCount * WAVES == TILE::kLoads ? wave * kCount + j : (wave * kCount + j) % TILE::kLoads;
    }
    __device__ __forceinline__ void init(const T *p, int64_t ld, int64_t first, int64_t count) {
        lane = threadIdx.x & 63;
        wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        stride = ld;
        base = p + (ROWS ? first * ld : first);
        rows = count - first < (1 << 20) ? (int)(count - first) : 1 << 20;
        if (DIRECT) {
            const int mine = fresh(lane);
#pragma unroll
            for (int j = 0; j < kCount; j++) {
                int row, l;
                TILE::source(number(wave, j), mine, row, l);
                off[j] = row < rows ? (uint32_t)((ROWS ? row * ld + l : l * ld + row) * 2) : 0x80000000u;
            }
        }
    }
    // the last tile has fewer sums: those beyond them read as zeros
    __device__ __forceinline__ void cut(int64_t left) {
        const int mine = fresh(lane);
#pragma unroll
        for (int j = 0; j < kCount; j++) {
            int row, l;
            TILE::source(number(wave, j), mine, row, l);
            if (l >= left) off[j] = 0x80000000u;
        }
    }
    __device__ __forceinline__ uint64_t from(int64_t l0) const { return (uint64_t)(uintptr_t)(base + (ROWS ? l0 : l0 * stride)); }
    // load j of the tile that begins at `from`, to LDS at `to`
    __device__ __forceinline__ void direct(uint64_t from, uint32_t to, int j) const {
        const i4 buffer = {__builtin_amdgcn_readfirstlane((int)(uint32_t)from), __builtin_amdgcn_readfirstlane((int)(uint32_t)(from >> 32)),
                           (int)0x80000000u, 0x00020000};
        // (m0 is the place in LDS, which nothing else here uses; one wait state before the load that does)
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(to + number(wave, j) * 1024),
                     "v"(off[j]), "s"(buffer));
    }
    __device__ __forceinline__ void load(int64_t l0, int64_t left) {
#pragma unroll
        for (int j = 0; j < kCount; j++) {
            int row, l;
            TILE::source(number(wave, j), lane, row, l);
            const int64_t most = ROWS ? left - l : rows - row;
            const bool in = ROWS ? row < rows : l < left;
            v[j].load(base + (ROWS ? row * stride + l0 + l : (l0 + l) * stride + row), !in || most <= 0 ? 0 : most < 8 ? (int)most : 8);
        }
    }
    __device__ __forceinline__ void store(uint32_t to) const {
#pragma unroll
        for (int j = 0; j < kCount; j++)
            *(lptr<typename Pack<T, 8>::vec>)(uintptr_t)(to + number(wave, j) * 1024 + lane * 16) = v[j].v;
    }
};

// Tile of workgroup b: workgroups go round the eight XCDs, so each gets a run of tiles
// that share rows and columns in its L2: eight tiles down, then the next column.
struct Place {
    int m, n, split;
};
__device__ __forceinline__ Place place_of(int b, int tm, int tn, int splits) {
    const int total = tm * tn * splits, q = total / 8, r = total % 8, xcd = b % 8;
    int t = xcd * q + (xcd < r ? xcd : r) + b / 8;
    const int split = t / (tm * tn);
    t -= split * tm * tn;
    constexpr int kDown = 8;
    const int group = t / (kDown * tn), first = group * kDown, down = tm - first < kDown ? tm - first : kDown;
    t -= group * kDown * tn;
    return {first + t % down, t / down, split};
}

// A workgroup has tile blockIdx.x and every gridDim.x-th after it.  Their steps, of BK sums each,
// are one sequence: while a step's fragments are multiplied, the next one's are read from LDS and a
// later one's tiles are loaded to it, across the end of a tile too, whose epilogue runs while the
// next one's loads are under way and the stores of the last go out.
template <class T, bool PROWS, bool QROWS, int BM, int BN, int WM, int WN, int STAGES, int PER_CU, bool DIRECT>
__global__ void __launch_bounds__(64 * WM * WN, PER_CU * WM * WN / 4)
    k_product(Product a, float *part, int tm, int tn, int splits, int64_t k_part) {
    constexpr int BK = 64, kWaves = WM * WN, WTM = BM / WM, WTN = BN / WN, MT = WTM / 16, NT = WTN / 32;
    typedef Tile<PROWS, false, BM, BK> PTile;
    typedef Tile<QROWS, true, BN, BK> QTile;
    typedef Loads<T, PTile, PROWS, kWaves, DIRECT> PLoads;
    typedef Loads<T, QTile, QROWS, kWaves, DIRECT> QLoads;
    constexpr int kStage = PTile::kBytes + QTile::kBytes, kOut = 16 * WTN * 4;
    constexpr int kLoads = PLoads::kCount + QLoads::kCount;
    static_assert(DIRECT || STAGES == 2, "stages");
    __shared__ __attribute__((aligned(1024))) char lds[STAGES * kStage + kWaves * kOut];
    const uint32_t lds0 = (uint32_t)(uintptr_t)(lptr<char>)(lds);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave / WN, wn = wave % WN;
    const int tiles = tm * tn * splits;
    auto sums_of = [&](const Place &at, int64_t &k0, int64_t &k1) __attribute__((always_inline)) {
        k0 = at.split * k_part;
        k1 = k0 + k_part < a.k ? k0 + k_part : a.k;
        return k1 - k0 > BK ? (int)((k1 - k0 + BK - 1) / BK) : 1;     // steps (one, if there are no sums)
    };

    // The step whose loads come next: what is left of its tile, and where its operands lie.  Behind the last
    // tile's last step, zeros are loaded, without a trip to memory.
    PLoads lp;
    QLoads lq;
    uint64_t from_p = 0, from_q = 0;
    int load_tile = blockIdx.x, load_left = 0;
    int64_t load_l = 0, load_end = 0;
    const int64_t by_p = PROWS ? BK * 2 : a.p_stride * (BK * 2), by_q = QROWS ? BK * 2 : a.q_stride * (BK * 2);
    auto next_load = [&]() __attribute__((always_inline)) {
        load_left--;
        load_l += BK;
        if (DIRECT) {
            from_p += (uint64_t)by_p;
            from_q += (uint64_t)by_q;
        }
        if (load_left <= 1) {
            if (load_left <= 0 && load_tile < tiles) {
                const Place at = place_of(load_tile, tm, tn, splits);
                load_left = sums_of(at, load_l, load_end);
                lp.init(static_cast<const T *>(a.p), a.p_stride, (int64_t)at.m * BM, a.m);
                lq.init(static_cast<const T *>(a.q), a.q_stride, (int64_t)at.n * BN, a.n);
                load_tile += gridDim.x;
                if (DIRECT) {
                    from_p = lp.from(load_l);
                    from_q = lq.from(load_l);
                }
            }
            if (DIRECT && load_left <= 1) {
                lp.cut(load_left == 1 ? load_end - load_l : 0);
                lq.cut(load_left == 1 ? load_end - load_l : 0);
            }
        }
        if (!DIRECT) {
            const int64_t left = load_left > 0 ? load_end - load_l : 0;
            lp.load(load_l, left);
            lq.load(load_l, left);
        }
    };

    // A step is two halves of 32 sums, each of MT chunks: 16 rows of p times the wave's columns.  A chunk's
    // fragment of p is followed, where it was, by that of the chunk a half later; q's of the half
    // to come are held beside those in use.  Within the second half the waves meet: all have read the step's
    // fragments (its slot is free for the loads of a later step), and the next step's tiles are in LDS.
    f4 acc[MT][NT][2];
    s8 fp[MT], fq[2][NT][2];
    const uint32_t base_p = lds0 + PTile::base(lane, wm * WTM), base_q = lds0 + PTile::kBytes + QTile::base(lane, wn * WTN);
    auto read_p = [&](uint32_t slot, int h, int i) __attribute__((always_inline)) { fp[i] = PTile::fragment(base_p + slot, i, 0, h); };
    // those of q that go with chunk i of n
    auto read_q = [&](uint32_t slot, int h, int i, int n) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < 2 * NT; j++)
            if (j * n / (2 * NT) == i) fq[h][j / 2][j % 2] = QTile::fragment(base_q + slot, j / 2, j % 2, h);
    };
    auto read_first = [&](uint32_t slot) __attribute__((always_inline)) {
        read_q(slot, 0, 0, 1);
#pragma unroll
        for (int i = 0; i < MT; i++) read_p(slot, 0, i);
    };
    // the loads that go with chunk i of n
    auto issue = [&](uint32_t to, int i, int n) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < kLoads; j++)
            if (j * n / kLoads == i) {
                if (j < PLoads::kCount) lp.direct(from_p, lds0 + to, j);
                else lq.direct(from_q, lds0 + to + PTile::kBytes, j - PLoads::kCount);
            }
    };
    // half h, with the reads of the other (from_h, in slot `from`) and the loads to `to`; `meet` is called
    // behind the first chunk, when the reads before it have had its time to come back
    auto half = [&](int h, uint32_t from, int from_h, bool loads, uint32_t to, auto meet) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < MT; i++) {
            if (i > 0) {
                read_q(from, from_h, i, MT);
                if (loads) issue(to, i, MT);
            }
#pragma unroll
            for (int j = 0; j < NT; j++)
#pragma unroll
                for (int s = 0; s < 2; s++) acc[i][j][s] = mfma(T{}, fq[h][j][s], fp[i], acc[i][j][s]);
            if (i == 0) {
                meet();
                read_q(from, from_h, 0, MT);
                if (loads) issue(to, 0, MT);
            }
            read_p(from, from_h, i);
            __builtin_amdgcn_sched_barrier(0);
        }
    };

    uint32_t slot = 0;
    if (DIRECT) {
#pragma unroll
        for (int t = 0; t < STAGES; t++) {
            next_load();
            issue(t * kStage, 0, 1);
        }
        // (the first step's loads are the oldest)
        asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"((STAGES - 1) * kLoads) : "memory");
    } else {
        next_load();
        lp.store(lds0);
        lq.store(lds0 + PTile::kBytes);
        __syncthreads();
        next_load();
    }
    read_first(0);

    constexpr int kLanes = WTN / 8, kRows = 64 / kLanes, kTurns = 16 / kRows;      // of the epilogue
    for (int tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
        const Place at = place_of(tile, tm, tn, splits);
        int64_t k0, k1;
        const int steps = sums_of(at, k0, k1);
#pragma unroll
        for (int i = 0; i < MT; i++)
#pragma unroll
            for (int j = 0; j < NT; j++) acc[i][j][0] = acc[i][j][1] = f4{0.0f, 0.0f, 0.0f, 0.0f};
        for (int t = 0; t < steps; t++) {
            half(0, slot, 1, false, 0, [] {});
            const uint32_t to = slot;
            slot = slot + kStage == STAGES * kStage ? 0 : slot + kStage;
            if (DIRECT) next_load();
            half(1, slot, 0, DIRECT, to, [&]() __attribute__((always_inline)) {
                if (DIRECT) {
                    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"((STAGES - 2) * kLoads) : "memory");
                } else {
                    lp.store(lds0 + slot);
                    lq.store(lds0 + slot + PTile::kBytes);
                    __syncthreads();
                    next_load();
                }
            });
        }

        // The sums go through LDS, 16 rows of the wave's tile at a time, so that neighbouring lanes store
        // neighbouring columns and the epilogue is one loop.  What it reads is loaded a turn ahead: loads
        // and stores are counted in order, and a wait for a load would be one for the stores before it.
        const uint32_t mine = lds0 + STAGES * kStage + wave * kOut;
        const int me = fresh(lane);
        const int64_t i0 = (int64_t)at.m * BM + wm * WTM + me / kLanes, j = (int64_t)at.n * BN + wn * WTN + 8 * (me % kLanes);
        const int have = a.n - j >= 8 ? 8 : a.n - j < 0 ? 0 : (int)(a.n - j);
        float bias[8];
        Pack<T, 8> side[kTurns];
        if (splits == 1) {
            load_bias<T>(a.e, j, have, bias);
#pragma unroll
            for (int u = 0; u < kTurns; u++) load_side<T>(a.e, i0 + u * kRows, j, i0 + u * kRows < a.m ? have : 0, side[u]);
        }
#pragma unroll 1
        for (int pass = 0; pass < MT; pass++) {
#pragma unroll
            for (int i = 0; i < MT; i++)
                if (i == pass) {
                    const int r = me & 15;
#pragma unroll
                    for (int x = 0; x < NT; x++)
#pragma unroll
                        for (int s = 0; s < 2; s++) {
                            const int c = (8 * x + 2 * (me >> 4) + s) ^ (r & (WTN / 4 - 1));
                            *(lptr<f4>)(uintptr_t)(mine + r * (WTN * 4) + c * 16) = acc[i][x][s];
                        }
                }
            Pack<T, 8> now[kTurns];
#pragma unroll
            for (int u = 0; u < kTurns; u++) {
                const int64_t i = i0 + (pass + 1) * 16 + u * kRows;
                now[u] = side[u];
                if (splits == 1 && pass + 1 < MT) load_side<T>(a.e, i, j, i < a.m ? have : 0, side[u]);
            }
            __builtin_amdgcn_wave_barrier();
#pragma unroll
            for (int u = 0; u < kTurns; u++) {
                const int r = me / kLanes + u * kRows;
                const int64_t i = i0 + pass * 16 + u * kRows;
                float v[8];
#pragma unroll
                for (int s = 0; s < 2; s++) {
                    const int c = (2 * (me % kLanes) + s) ^ (r & (WTN / 4 - 1));
                    const f4 x = *(lptr<const f4>)(uintptr_t)(mine + r * (WTN * 4) + c * 16);
#pragma unroll
                    for (int b = 0; b < 4; b++) v[4 * s + b] = x[b];
                }
                if (i >= a.m || have == 0) continue;
                if (splits > 1) {
                    Pack<float, 8> p;
                    p.from(v);
                    p.store(part + (at.split * a.m + i) * a.n + j, have);
                } else {
                    finish<T>(a.e, i, j, have, v, bias, now[u]);
                }
            }
            __builtin_amdgcn_wave_barrier();
        }
        read_first(slot);     // (again: held through the epilogue, they would cost it their registers)
    }
    if (DIRECT) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");      // (no load to LDS outlives its workgroup)
}

// The parts of a product whose sums were cut, joined in order.
template <class T>
__global__ void __launch_bounds__(256) k_product_join(Product a, const float *part, int splits) {
    const int64_t packs = (a.n + 7) / 8, total = packs * a.m;
    for (int64_t t = blockIdx.x * (int64_t)256 + threadIdx.x; t < total; t += (int64_t)gridDim.x * 256) {
        const int64_t i = t / packs, j = (t - i * packs) * 8;
        const int have = a.n - j >= 8 ? 8 : (int)(a.n - j);
        const float *p = part + i * a.n + j;
        float v[8] = {};
        for (int s = 0; s < splits; s++, p += a.m * a.n) {
            Pack<float, 8> b;
            float x[8];
            b.load(p, have);
            b.to(x);
#pragma unroll
            for (int c = 0; c < 8; c++) v[c] += x[c];
        }
        float bias[8];
        Pack<T, 8> side;
        load_bias<T>(a.e, j, have, bias);
        load_side<T>(a.e, i, j, have, side);
        finish<T>(a.e, i, j, have, v, bias, side);
    }
}

// --- which tiles, and how sums are cut -------------------------------------------
struct Plan {
    int tile;                   // rows of p a workgroup has: 16, 128 or 256
    int tm, tn, splits;
    int64_t k_part;
};

int64_t tiles_of(int64_t x, int64_t n) { return (x + n - 1) / n; }

constexpr int kUnits = 256;     // compute units

Plan plan_of(int64_t m, int64_t n, int64_t k, bool direct) {
    Plan p;
    const int64_t t128 = tiles_of(m, 128) * tiles_of(n, 128), t256 = tiles_of(m, 256) * tiles_of(n, 256);
    if (m <= 16) {
        p.tile = 16;
    } else {
        // rounds of the compute units (two small tiles to each), a large tile at 5/4 of the rate
        const int64_t r256 = tiles_of(t256, kUnits) * 4 * 4, r128 = tiles_of(t128, 2 * kUnits) * 2 * 5;
        p.tile = direct && r256 <= r128 ? 256 : 128;
    }
    const int64_t rows = p.tile, cols = p.tile == 256 ? 256 : 128;
    const int64_t tm = tiles_of(m, rows), tn = tiles_of(n, cols), tiles = tm * tn;
    const int64_t want = p.tile == 16 ? 4 * kUnits : p.tile == 128 ? 2 * kUnits : kUnits;
    int64_t splits = want / tiles, most = k / 256;
    if (splits > most) splits = most;
    if (splits < 1) splits = 1;
    p.k_part = tiles_of(tiles_of(k, splits), 64) * 64;
    if (p.k_part < 64) p.k_part = 64;       // (k == 0)
    p.splits = (int)tiles_of(k, p.k_part);
    if (p.splits < 1) p.splits = 1;
    p.tm = (int)tm;
    p.tn = (int)tn;
    return p;
}

size_t plan_work(const Plan &p, int64_t m, int64_t n) { return p.splits > 1 ? (size_t)p.splits * (size_t)m * (size_t)n * sizeof(float) : 0; }

// An operand that loads go to LDS directly from: 16 bytes in a row lie aligned, all of
// one row (or one l), and a tile spans less than 2 GiB.
bool aligned_operand(const void *p, int64_t stride, bool by_rows, int64_t count, int64_t k) {
    return reinterpret_cast<uintptr_t>(p) % 16 == 0 && stride % 8 == 0 && (by_rows ? k : count) % 8 == 0 && stride < (int64_t(1) << 22);
}

template <class T, bool PROWS, bool QROWS, int BM, int BN, int WM, int WN, int STAGES, int PER_CU, bool DIRECT>
void run_product(const Product &a, const Plan &p, float *part, hipStream_t s) {
    const int tiles = p.tm * p.tn * p.splits, grid = tiles < PER_CU * kUnits ? tiles : PER_CU * kUnits;
    k_product<T, PROWS, QROWS, BM, BN, WM, WN, STAGES, PER_CU, DIRECT><<<grid, 64 * WM * WN, 0, s>>>(a, part, p.tm, p.tn, p.splits, p.k_part);
}
template <class T, bool PROWS, bool QROWS>
void product(const Product &a, const Plan &p, bool direct, float *part, hipStream_t s) {
    if (direct) {
        if (p.tile == 16) run_product<T, PROWS, QROWS, 16, 128, 1, 4, 2, 3, true>(a, p, part, s);
        else if (p.tile == 128) run_product<T, PROWS, QROWS, 128, 128, 2, 2, 2, 2, true>(a, p, part, s);
        else run_product<T, PROWS, QROWS, 256, 256, 2, 4, 2, 1, true>(a, p, part, s);
    } else if (p.tile == 16) {
        run_product<T, PROWS, QROWS, 16, 128, 1, 4, 2, 3, false>(a, p, part, s);
    } else {
        run_product<T, PROWS, QROWS, 128, 128, 2, 2, 2, 2, false>(a, p, part, s);
    }
}
template <class T>
hipError_t product(const Product &a, float *part, hipStream_t s) {
    const bool direct = aligned_operand(a.p, a.p_stride, a.p_by_rows, a.m, a.k) && aligned_operand(a.q, a.q_stride, a.q_by_rows, a.n, a.k);
    const Plan p = plan_of(a.m, a.n, a.k, direct);
    if (a.p_by_rows && a.q_by_rows) product<T, true, true>(a, p, direct, part, s);
    else if (a.p_by_rows) product<T, true, false>(a, p, direct, part, s);
    else product<T, false, false>(a, p, direct, part, s);
    if (p.splits > 1) {
        const int64_t need = tiles_of(a.m * tiles_of(a.n, 8), 256);
        k_product_join<T><<<(unsigned)(need < 8 * kUnits ? need : 8 * kUnits), 256, 0, s>>>(a, part, p.splits);
    }
    return hipGetLastError();
}

// --- sums over rows, and an activation's derivative -------------------------------
// Workgroup (i, j) has 256 columns and the j-th run of rows, eight rows at a time,
// and writes its sums to part j (a single one: to the output); then 32 threads a
// column join the parts in order.
constexpr int kSumParts = 256, kSumCols = 256, kSumRows = 8;

__device__ __forceinline__ void store_as(void *p, int32_t type, int64_t i, float x) {
    if (type == DD_F32) static_cast<float *>(p)[i] = x;
    else if (type == DD_BF16) static_cast<bf16_t *>(p)[i] = (bf16_t)x;
    else static_cast<f16_t *>(p)[i] = (f16_t)x;
}

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
    const int64_t blocks = tiles_of(cols, kSumCols);
    int64_t n = tiles_of(4 * kUnits, blocks), most = rows / 32;
    if (n > most) n = most;
    if (n > kSumParts) n = kSumParts;
    return n < 1 ? 1 : (int)n;
}

// Bound: HBM.
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

size_t product_work(int64_t m, int64_t n, int64_t k) {
    const size_t a = plan_work(plan_of(m, n, k, true), m, n), b = plan_work(plan_of(m, n, k, false), m, n);
    return a > b ? a : b;
}

bool product_fits(int64_t m, int64_t n, int64_t k) {
    for (bool direct : {true, false}) {       // (tiles are counted in 32 bits)
        const Plan p = plan_of(m, n, k, direct);
        if (tiles_of(m, p.tile) * (int64_t)p.tn * p.splits >= (int64_t(1) << 30)) return false;
    }
    return true;
}

hipError_t launch_product(const Product &p, void *work, hipStream_t s) {
    return p.type == DD_BF16 ? product<bf16_t>(p, static_cast<float *>(work), s) : product<f16_t>(p, static_cast<float *>(work), s);
}

size_t column_sum_work(int64_t rows, int64_t cols) {
    const int n = sum_parts(rows, cols);
    return n > 1 ? (size_t)n * (size_t)cols * sizeof(float) : 0;
}

hipError_t launch_column_sum(const void *x, int64_t stride, int64_t rows, int64_t cols, int32_t type, void *out, int32_t out_type, void *work,
                             hipStream_t s) {
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
