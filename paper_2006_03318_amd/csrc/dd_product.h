// The kernel of a product, for one type of elements (instances by layout, tile and alignment are
// in the sources that include this).
//
//   out(i, j) = sum over l of p(i, l) q(l, j), and the epilogue of it
#pragma once

#include "dd_epilogue.h"

namespace dd {

// Which tiles, and how the sums are cut.
struct Plan {
    int tile;                   // rows of p a workgroup has: 128 or 256; 16 or 64 with waves that share the sums
    int tm, tn, splits;
    int64_t k_part;             // sums of a part: a multiple of 64
    double us;                  // expected
};
constexpr int kUnits = 256;     // compute units
template <bool DIRECT>
constexpr int kApart = DIRECT ? 4 : 8;      // waves that share the sums of a tile of 64 rows

// the tiles' passes; of a plan for aligned operands (DIRECT) or any
template <class T, bool DIRECT>
void launch_tiles(const Product &a, const Plan &p, float *part, hipStream_t s);
// both products of a layer's gradients in tiles of 64 x 64, uncut, with aligned operands
template <class T>
void launch_two(const Product &a, const Product &b, hipStream_t s);

}  // namespace dd

#ifdef DD_PRODUCT_KERNEL
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
    static constexpr int kN = N, kBytes = N * BK * 2, kLoads = kBytes / 1024;
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
    uint32_t off[kCount];        // bytes from the tile's beginning on
    Pack<T, 8> v[DIRECT ? 1 : kCount];
    bool plain;                  // not DIRECT: a whole step's loads are where off says
    const T *base;               // of the tile's first row, at l = 0
    int64_t stride;
    int rows, lane, wave;        // rows: that the operand has from the tile's first on

    static __device__ __forceinline__ int number(int wave, int j) {
        return kCount * WAVES == TILE::kLoads ? wave * kCount + j : (wave * kCount + j) % TILE::kLoads;
    }
    // (wave: among those that share the tiles)
    __device__ __forceinline__ void init(const T *p, int64_t ld, int64_t first, int64_t count, int of_wave) {
        lane = threadIdx.x & 63;
        wave = of_wave;
        stride = ld;
        base = p + (ROWS ? first * ld : first);
        rows = count - first < (1 << 20) ? (int)(count - first) : 1 << 20;
        // (what rows or columns beyond the end hold counts for nothing.  Not DIRECT: such rows are the last one
        // again, and such columns what follows in memory, which it does but for the last l)
        plain = stride < (1 << 22) && (ROWS || stride >= 8);
        const int mine = fresh(lane);
#pragma unroll
        for (int j = 0; j < kCount; j++) {
            int row, l;
            TILE::source(number(wave, j), mine, row, l);
            if (!DIRECT) row = row < rows ? row : ROWS ? rows - 1 : 0;
            off[j] = !DIRECT || row < rows ? (uint32_t)((ROWS ? row * ld + l : l * ld + row) * 2) : 0x80000000u;
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
    __device__ __forceinline__ i4 buffer_at(uint64_t from) const {
        return {__builtin_amdgcn_readfirstlane((int)(uint32_t)from), __builtin_amdgcn_readfirstlane((int)(uint32_t)(from >> 32)), (int)0x80000000u, 0x00020000};
    }
    // loads j and j + 1 of the tile that begins at `from`, to LDS at `to`.  m0 is the place in LDS.  The text waits by itself, as
    // the compiler does not look into it: one state between m0 and a load, and five between a vector instruction that
    // wrote a scalar operand and the load.
    __device__ __forceinline__ void direct(uint64_t from, uint32_t to, int j) const {
        static_assert(kCount % 2 == 0, "pairs");
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 3\n\tbuffer_load_dwordx4 %2, %4, 0 offen lds\n\t"
                     "s_mov_b32 m0, %1\n\ts_nop 0\n\tbuffer_load_dwordx4 %3, %4, 0 offen lds" ::"s"(to + number(wave, j) * 1024),
                     "s"(to + number(wave, j + 1) * 1024), "v"(off[j]), "v"(off[j + 1]), "s"(buffer_at(from)) : "m0");
    }
    // whether a step of `full` sums, of those `left`, is loaded without a look at what is there
    __device__ __forceinline__ bool quick(int64_t left, int full) const {
        return plain && (left > full || (left == full && (ROWS || rows >= TILE::kN)));
    }
    __device__ __forceinline__ void load_quick(int64_t l0) {
        const char *b = reinterpret_cast<const char *>(base + (ROWS ? l0 : l0 * stride));
#pragma unroll
        for (int j = 0; j < kCount; j++) v[j].load(reinterpret_cast<const T *>(b + off[j]));
    }
    __device__ __forceinline__ void load_slowly(int64_t l0, int64_t left) {
        const int mine = fresh(lane);
#pragma unroll
        for (int j = 0; j < kCount; j++) {
            int row, l;
            TILE::source(number(wave, j), mine, row, l);
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

// (one branch for both operands: loads under way in one of two ways would be waited for before those of the next)
template <class P, class Q>
__device__ __forceinline__ void load_step(P &p, Q &q, int64_t l0, int64_t left, int full) {
    if (p.quick(left, full) && q.quick(left, full)) {
        p.load_quick(l0);
        q.load_quick(l0);
    } else {
        p.load_slowly(l0, left);
        q.load_slowly(l0, left);
    }
}

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
//   Bound: the matrix instructions, fed by a barrier a step.  256 x 256 tiles (two stages of 64 KB) use each element
// from L2 256 times: 8,192^3 bf16 in 770 to 790 us (1.4 PFLOP/s);
// 65,536 x 8,192 -> 2,048 into a residual 1,700 to 1,725; 16,384 x 2,048 -> 8,192 477, 530 to 555 with bias, GELU and both
// outputs.  128 x 128 (four stages of 32 KB) where 256 x 256 would leave compute units without a tile: 4,096 x 1,280 ->
// 768 in 17.  Fewer or more stages, deeper prefetch in the epilogue, and tiles by 32 sums were slower.
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
                lp.init(static_cast<const T *>(a.p), a.p_stride, (int64_t)at.m * BM, a.m, wave);
                lq.init(static_cast<const T *>(a.q), a.q_stride, (int64_t)at.n * BN, a.n, wave);
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
            load_step(lp, lq, load_l, left, BK);
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
        for (int j = 0; j < kLoads; j += 2)
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

// Small products, whose bound are the weight's bytes or the latency of a step's loads.  A workgroup has one
// tile of 16 MT rows by 64 columns, and each of its waves a run of the sums with tiles of its own in LDS, so that
// no wave waits for another until the waves' sums are joined in order at the end.  4 x 2,048 -> 8,192 bf16 with GELU 9.4 us (33.6 MB
// of weight at 3.6 TB/s, launch included); 1,021 x 1,237 -> 777 f16 with its copies 16.5, 24 with 128 x 128.
template <int MT, int WAVES, bool DIRECT>
constexpr int kApartBytes = WAVES * (DIRECT ? 2 : 1) * (16 * MT + 64) * 64 * 2;
template <class T, bool PROWS, bool QROWS, int MT, int WAVES, bool DIRECT>
__device__ __forceinline__ void apart(const Product &a, float *part, int tm, int tn, int splits, int64_t k_part, int block, char *lds) {
    constexpr int BK = 64, BN = 64, NT = BN / 32, STAGES = DIRECT ? 2 : 1;
    typedef Tile<PROWS, false, 16 * MT, BK> PTile;
    typedef Tile<QROWS, true, BN, BK> QTile;
    typedef Loads<T, PTile, PROWS, 1, DIRECT> PLoads;
    typedef Loads<T, QTile, QROWS, 1, DIRECT> QLoads;
    constexpr int kStage = PTile::kBytes + QTile::kBytes, kLoads = PLoads::kCount + QLoads::kCount, kSums = 16 * MT * BN * 4;
    static_assert(kSums <= STAGES * kStage && WAVES * STAGES * kStage == kApartBytes<MT, WAVES, DIRECT>, "room");
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t lds0 = (uint32_t)(uintptr_t)(lptr<char>)(lds), mine = lds0 + wave * (STAGES * kStage);
    // (few rows: what is read is the weight, a part of it by each workgroup alone)
    const Place at = MT == 1 ? Place{0, block % tn, block / tn} : place_of(block, tm, tn, splits);
    const int64_t m0 = (int64_t)at.m * (16 * MT), n0 = (int64_t)at.n * BN, s0 = at.split * k_part, s1 = s0 + k_part < a.k ? s0 + k_part : a.k;
    const int64_t each = ((s1 - s0 + WAVES * BK - 1) / (WAVES * BK)) * BK;
    const int64_t k0 = s0 + wave * each, k1 = k0 + each < s1 ? k0 + each : s1;
    const int steps = k1 > k0 ? (int)((k1 - k0 + BK - 1) / BK) : 0;

    PLoads lp;
    QLoads lq;
    lp.init(static_cast<const T *>(a.p), a.p_stride, m0, a.m, 0);
    lq.init(static_cast<const T *>(a.q), a.q_stride, n0, a.n, 0);
    f4 acc[MT][NT][2] = {};
    auto load = [&](int t) __attribute__((always_inline)) {
        const int64_t l0 = k0 + (int64_t)t * BK, left = k1 - l0 > 0 ? k1 - l0 : 0;
        if (DIRECT) {
            if (left < BK) {
                lp.cut(left);
                lq.cut(left);
            }
            const uint32_t to = mine + (t & 1) * kStage;
            const uint64_t fp = lp.from(l0), fq = lq.from(l0);
#pragma unroll
            for (int j = 0; j < QLoads::kCount; j += 2) lq.direct(fq, to + PTile::kBytes, j);
#pragma unroll
            for (int j = 0; j < PLoads::kCount; j += 2) lp.direct(fp, to, j);
        } else {
            load_step(lp, lq, l0, left, BK);
        }
    };
    load(0);
    if (DIRECT) load(1);
    for (int t = 0; t < steps; t++) {
        const uint32_t from = mine + (DIRECT ? (t & 1) * kStage : 0);
        if (DIRECT) {
            asm volatile("s_waitcnt vmcnt(%0)" ::"n"(kLoads) : "memory");
        } else {
            lp.store(from);
            lq.store(from + PTile::kBytes);
            load(t + 1);
        }
        const uint32_t base_p = from + PTile::base(lane, 0), base_q = from + PTile::kBytes + QTile::base(lane, 0);
        s8 fp[2][MT], fq[2][NT][2];
#pragma unroll
        for (int h = 0; h < 2; h++) {
#pragma unroll
            for (int j = 0; j < 2 * NT; j++) fq[h][j / 2][j % 2] = QTile::fragment(base_q, j / 2, j % 2, h);
#pragma unroll
            for (int i = 0; i < MT; i++) fp[h][i] = PTile::fragment(base_p, i, 0, h);
        }
        if (DIRECT) {       // (all read: the slot is free)
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            load(t + 2);
        }
#pragma unroll
        for (int h = 0; h < 2; h++)
#pragma unroll
            for (int i = 0; i < MT; i++)
#pragma unroll
                for (int j = 0; j < 2 * NT; j++) acc[i][j / 2][j % 2] = mfma(T{}, fq[h][j / 2][j % 2], fp[h][i], acc[i][j / 2][j % 2]);
    }
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    __syncthreads();
    // the waves' sums, chunks of a row permuted as in k_product
#pragma unroll
    for (int i = 0; i < MT; i++)
#pragma unroll
        for (int j = 0; j < 2 * NT; j++) {
            const int r = lane & 15, c = (8 * (j / 2) + 2 * (lane >> 4) + j % 2) ^ r;
            *(lptr<f4>)(uintptr_t)(lds0 + wave * kSums + (16 * i + r) * (BN * 4) + c * 16) = acc[i][j / 2][j % 2];
        }
    __syncthreads();
    for (int t = threadIdx.x; t < 16 * MT * (BN / 8); t += 64 * WAVES) {
        const int r = t / (BN / 8);
        const int64_t i = m0 + r, j = n0 + 8 * (t % (BN / 8));
        const int have = i < a.m ? a.n - j >= 8 ? 8 : a.n - j < 0 ? 0 : (int)(a.n - j) : 0;
        if (have == 0) continue;
        float v[8] = {};
        for (int w = 0; w < WAVES; w++)
#pragma unroll
            for (int s = 0; s < 2; s++) {
                const f4 x = *(lptr<const f4>)(uintptr_t)(lds0 + w * kSums + r * (BN * 4) + ((2 * (t % (BN / 8)) + s) ^ (r & 15)) * 16);
#pragma unroll
                for (int b = 0; b < 4; b++) v[4 * s + b] += x[b];
            }
        if (splits > 1) {
            Pack<float, 8> p;
            p.from(v);
            p.store(part + (at.split * a.m + i) * a.n + j, have);
        } else {
            float bias[8];
            Pack<T, 8> side;
            load_bias<T>(a.e, j, have, bias);
            load_side<T>(a.e, i, j, have, side);
            finish<T>(a.e, i, j, have, v, bias, side);
        }
    }
}

template <class T, bool PROWS, bool QROWS, int MT, int WAVES, bool DIRECT>
__global__ void __launch_bounds__(64 * WAVES) k_product_apart(Product a, float *part, int tm, int tn, int splits, int64_t k_part) {
    __shared__ __attribute__((aligned(1024))) char lds[kApartBytes<MT, WAVES, DIRECT>];
    apart<T, PROWS, QROWS, MT, WAVES, DIRECT>(a, part, tm, tn, splits, k_part, blockIdx.x, lds);
}

// Both products of a layer's gradients, where neither fills the compute units: the gradient of the weight (a) by the first
// workgroups, that of the rows (b) by those from `second` on, a multiple of eight (the XCDs).  256 rows of 256 x 256 bf16, with
// db, 10 us, 14.5 in launches of their own; 1,021 of 777 x 1,237 30, 35.
template <class T, bool QROWS>
__global__ void __launch_bounds__(64 * kApart<true>) k_product_two(Product a, Product b, int atm, int atn, int btm, int btn, int second) {
    __shared__ __attribute__((aligned(1024))) char lds[kApartBytes<4, kApart<true>, true>];
    if ((int)blockIdx.x < atm * atn) apart<T, false, false, 4, kApart<true>, true>(a, nullptr, atm, atn, 1, (a.k + 63) / 64 * 64, blockIdx.x, lds);
    else if ((int)blockIdx.x >= second) apart<T, true, QROWS, 4, kApart<true>, true>(b, nullptr, btm, btn, 1, (b.k + 63) / 64 * 64, blockIdx.x - second, lds);
}

template <class T, bool PROWS, bool QROWS, int BM, int BN, int WM, int WN, int STAGES, int PER_CU, bool DIRECT>
void run_product(const Product &a, const Plan &p, float *part, hipStream_t s) {
    const int tiles = p.tm * p.tn * p.splits, grid = tiles < PER_CU * kUnits ? tiles : PER_CU * kUnits;
    k_product<T, PROWS, QROWS, BM, BN, WM, WN, STAGES, PER_CU, DIRECT><<<grid, 64 * WM * WN, 0, s>>>(a, part, p.tm, p.tn, p.splits, p.k_part);
}
template <class T, bool DIRECT, bool PROWS, bool QROWS>
void run_plan(const Product &a, const Plan &p, float *part, hipStream_t s) {
    const int tiles = p.tm * p.tn * p.splits;
    if (PROWS && p.tile == 16) k_product_apart<T, true, QROWS, 1, 8, DIRECT><<<tiles, 512, 0, s>>>(a, part, p.tm, p.tn, p.splits, p.k_part);
    else if (p.tile <= 64) k_product_apart<T, PROWS, QROWS, 4, kApart<DIRECT>, DIRECT><<<tiles, 64 * kApart<DIRECT>, 0, s>>>(a, part, p.tm, p.tn, p.splits, p.k_part);
    else if (!DIRECT || p.tile == 128) run_product<T, PROWS, QROWS, 128, 128, 2, 4, DIRECT ? 4 : 2, 1, DIRECT>(a, p, part, s);
    else run_product<T, PROWS, QROWS, 256, 256, 2, 4, 2, 1, true>(a, p, part, s);
}

}  // namespace

template <class T>
void launch_two(const Product &a, const Product &b, hipStream_t s) {
    const int atm = (int)((a.m + 63) / 64), atn = (int)((a.n + 63) / 64), btm = (int)((b.m + 63) / 64), btn = (int)((b.n + 63) / 64);
    const int second = (atm * atn + 7) / 8 * 8;
    if (b.q_by_rows) k_product_two<T, true><<<second + btm * btn, 64 * kApart<true>, 0, s>>>(a, b, atm, atn, btm, btn, second);
    else k_product_two<T, false><<<second + btm * btn, 64 * kApart<true>, 0, s>>>(a, b, atm, atn, btm, btn, second);
}

template <class T, bool DIRECT>
void launch_tiles(const Product &a, const Plan &p, float *part, hipStream_t s) {
    if (a.p_by_rows && a.q_by_rows) run_plan<T, DIRECT, true, true>(a, p, part, s);
    else if (a.p_by_rows) run_plan<T, DIRECT, true, false>(a, p, part, s);
    else run_plan<T, DIRECT, false, false>(a, p, part, s);
}

}  // namespace dd
#endif
