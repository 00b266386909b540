// The embedding: rows of a table for a batch's tokens, and the table's gradient.
//
//   out[t] = scale * table[ids[t]]
//   dtable[v] = scale * sum of dy[t] over the tokens with ids[t] = v
//
// The gradient sorts the tokens by id (stable), so that a row's sum is taken over a
// run of neighbours in the tokens' order: no atomics on sums, the same bits on every call.
#include "dd_elem.h"
#include "dd_layers.h"

namespace dd {

namespace {

__device__ __forceinline__ int64_t id_at(const void *ids, int bytes, int64_t t) {
    return bytes == 8 ? static_cast<const int64_t *>(ids)[t] : static_cast<const int32_t *>(ids)[t];
}
__host__ __device__ inline int have_of(int64_t n, int64_t i) { return n - i >= 8 ? 8 : n - i < 0 ? 0 : (int)(n - i); }

// A thread has eight columns of a token, or of EACH tokens whose rows are loaded at once.  Bound: HBM; few
// tokens, the launch.
template <class T, int EACH>
__global__ void __launch_bounds__(256) k_embed(dd_embed_args a, uint32_t packs) {
    const int64_t total = a.tokens * packs;
    for (int64_t i0 = blockIdx.x * (int64_t)(256 * EACH) + threadIdx.x; i0 < total; i0 += (int64_t)gridDim.x * (256 * EACH)) {
        int64_t t[EACH], c[EACH], id[EACH];
        Pack<T, 8> p[EACH];
#pragma unroll
        for (int u = 0; u < EACH; u++) {
            const int64_t i = i0 + 256 * u < total ? i0 + 256 * u : i0;
            t[u] = (uint64_t)i >> 32 ? i / packs : (int64_t)((uint32_t)i / packs);
            c[u] = (i - t[u] * packs) * 8;
            id[u] = id_at(a.ids, a.id_bytes, t[u]);
        }
#pragma unroll
        for (int u = 0; u < EACH; u++) {
            const bool there = id[u] >= 0 && id[u] < a.vocab;
            p[u].load(static_cast<const T *>(a.table) + (there ? id[u] : 0) * a.table_stride + c[u], there ? have_of(a.cols, c[u]) : 0);
        }
#pragma unroll
        for (int u = 0; u < EACH; u++) {
            if (i0 + 256 * u >= total) continue;
            const bool there = id[u] >= 0 && id[u] < a.vocab;
            float x[8];
            p[u].to(x);
#pragma unroll
            for (int j = 0; j < 8; j++) x[j] = there ? x[j] * a.scale : __builtin_nanf("");
            p[u].from(x);
            p[u].store(static_cast<T *>(a.out) + t[u] * a.out_stride + c[u], have_of(a.cols, c[u]));
        }
    }
}

// --- the tokens in the order of their ids -------------------------------------------
// Least significant digits of eight bits first, stable.  Ids that do not count (pad, or not in
// the table) are `vocab`, behind all others.
constexpr int kDigits = 256;

struct Sorted {
    uint32_t *key, *place;       // id and token
};

__device__ __forceinline__ uint32_t key_of(const dd_embed_grad_args &a, int64_t t) {
    const int64_t id = id_at(a.ids, a.id_bytes, t);
    return id < 0 || id >= a.vocab || id == a.pad ? (uint32_t)a.vocab : (uint32_t)id;
}

// Lanes of the wave, among those that are in, with this lane's digit.
__device__ __forceinline__ uint64_t peers_of(uint32_t digit, bool in) {
    uint64_t same = __ballot(in);
#pragma unroll
    for (int b = 0; b < 8; b++) {
        const uint64_t set = __ballot(digit >> b & 1);
        same &= digit >> b & 1 ? set : ~set;
    }
    return same;
}
__device__ __forceinline__ int rank_among(uint64_t peers) { return __popcll(peers & ((uint64_t(1) << (threadIdx.x & 63)) - 1)); }

// Exclusive running sum over the first 256 threads (a multiple of 64, all of whose waves call), by `room` of LDS.
__device__ __forceinline__ uint32_t digits_before(uint32_t x, uint32_t *room) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    uint32_t run = x;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const uint32_t y = __shfl_up(run, o, 64);
        if (lane >= o) run += y;
    }
    if (lane == 63) room[wave] = run;
    __syncthreads();
    run -= x;
    for (int w = 0; w < wave; w++) run += room[w];
    return run;
}

// Zeros in the table's first `rows` rows, eight columns a thread, by the workgroups from `first` on of a launch.
template <class T>
__device__ __forceinline__ void fill_table(const dd_embed_grad_args &a, int64_t rows, int64_t first) {
    Pack<T, 8> zero;
    zero.v = 0;
    const int64_t me = (blockIdx.x - first) * (int64_t)blockDim.x + threadIdx.x, all = (gridDim.x - first) * (int64_t)blockDim.x;
    T *to = static_cast<T *>(a.dtable);
    if (a.dtable_stride == a.cols) {        // (16 bytes a thread: whole lines)
        constexpr int kE = 16 / sizeof(T);
        Pack<T, kE> z;
        z.v = 0;
        const int64_t n = rows * a.cols, whole = n / kE;
        for (int64_t i = me; i < whole; i += all) z.store(to + kE * i);
        if (me < n - whole * kE) global(to)[whole * kE + me] = (T)0.0f;
        return;
    }
    const int64_t packs = (a.cols + 7) / 8, n = rows * packs;
    for (int64_t i = me; i < n; i += all) {
        const int64_t r = i / packs, c = (i - r * packs) * 8;
        zero.store(to + r * a.dtable_stride + c, have_of(a.cols, c));
    }
}

// Few tokens: one workgroup sorts them in LDS, EACH to a thread, while the others may fill the table (50,021 x 513
// f32 in 15 us, 6.6 TB/s: the fill's time).
constexpr int kSmallThreads = 1024, kSmallWaves = kSmallThreads / 64;
template <class T, int EACH>
__global__ void __launch_bounds__(kSmallThreads) k_embed_sort(dd_embed_grad_args a, Sorted to, int passes, int64_t rows) {
    if (blockIdx.x > 0) {
        fill_table<T>(a, rows, 1);
        return;
    }
    __shared__ uint32_t keys[kSmallThreads * EACH], next[kSmallWaves][kDigits], room[kSmallWaves];
    __shared__ uint16_t places[kSmallThreads * EACH];
    const int n = (int)a.tokens, lane = threadIdx.x & 63, wave = threadIdx.x >> 6, first = wave * (64 * EACH);
    uint32_t key[EACH], place[EACH], before[EACH];
#pragma unroll
    for (int i = 0; i < EACH; i++) {
        place[i] = first + i * 64 + lane;
        key[i] = (int)place[i] < n ? key_of(a, place[i]) : 0;
    }
    for (int pass = 0; pass < passes; pass++) {
        for (int d = lane; d < kDigits; d += 64) next[wave][d] = 0;
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int i = 0; i < EACH; i++) {
            const bool in = first + i * 64 + lane < n;
            const uint32_t d = key[i] >> (8 * pass) & (kDigits - 1);
            const uint64_t peers = peers_of(d, in);
            const int rank = rank_among(peers);
            before[i] = next[wave][d] + rank;
            __builtin_amdgcn_wave_barrier();
            if (in && rank == 0) next[wave][d] += __popcll(peers);
            __builtin_amdgcn_wave_barrier();
        }
        __syncthreads();
        uint32_t all = 0;
        if (threadIdx.x < kDigits)
            for (int w = 0; w < kSmallWaves; w++) all += next[w][threadIdx.x];
        uint32_t at = digits_before(threadIdx.x < kDigits ? all : 0, room);
        if (threadIdx.x < kDigits)
            for (int w = 0; w < kSmallWaves; w++) {
                const uint32_t x = next[w][threadIdx.x];
                next[w][threadIdx.x] = at;
                at += x;
            }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < EACH; i++) {
            if (first + i * 64 + lane >= n) continue;
            const uint32_t p = next[wave][key[i] >> (8 * pass) & (kDigits - 1)] + before[i];
            if (pass + 1 == passes) {
                to.key[p] = key[i];
                to.place[p] = place[i];
            } else {
                keys[p] = key[i];
                places[p] = (uint16_t)place[i];
            }
        }
        if (pass + 1 == passes) return;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < EACH; i++) {
            const int p = first + i * 64 + lane;
            key[i] = p < n ? keys[p] : 0;
            place[i] = p < n ? places[p] : 0;
        }
        __syncthreads();
    }
}

// More: a workgroup has kSortBlock places in a row and a wave a run of them, so ranks count waves, then lanes.
// Bound: latency; 65,536 tokens take 5 us to count and 7 to place, a pass (16 waves with two keys a lane; four with
// eight 6 and 8, and with one key and twice the workgroups 200,000 tokens take 15 us longer).
constexpr int kSortThreads = 1024, kSortWaves = kSortThreads / 64, kSortEach = 2, kSortBlock = kSortThreads * kSortEach;
static_assert(kSortThreads >= kDigits, "a thread has a digit");

// A workgroup's places with each digit lie digit by digit (those to be summed by a scan) or workgroup by
// workgroup (which threads of a digit each read side by side).
constexpr int kManyBlocks = 512;
__device__ __forceinline__ int64_t count_at(int digit, int64_t block, int64_t blocks) {
    return blocks > kManyBlocks ? digit * blocks + block : block * kDigits + digit;
}

// the counts; the workgroups behind fill the table
template <class T, bool FIRST>
__global__ void __launch_bounds__(kSortThreads) k_embed_count(dd_embed_grad_args a, Sorted from, int shift, int blocks, uint32_t *counts, int64_t rows) {
    if ((int)blockIdx.x >= blocks) {
        fill_table<T>(a, rows, blocks);
        return;
    }
    __shared__ uint32_t n[kDigits];
    if (threadIdx.x < kDigits) n[threadIdx.x] = 0;
    __syncthreads();
    const int64_t first = (int64_t)blockIdx.x * kSortBlock;
    uint32_t key[kSortEach];
#pragma unroll
    for (int i = 0; i < kSortEach; i++) {
        const int64_t t = first + i * kSortThreads + threadIdx.x;
        key[i] = t >= a.tokens ? 0 : FIRST ? key_of(a, t) : from.key[t];
    }
#pragma unroll
    for (int i = 0; i < kSortEach; i++)
        if (first + i * kSortThreads + threadIdx.x < a.tokens) atomicAdd(&n[key[i] >> shift & (kDigits - 1)], 1u);
    __syncthreads();
    if (threadIdx.x < kDigits) counts[count_at(threadIdx.x, blockIdx.x, blocks)] = n[threadIdx.x];
}

// Where there are too many workgroups for each to sum the others' counts: a workgroup has a digit, makes running sums of its
// counts in place, and puts their sum behind all counts.
__global__ void __launch_bounds__(256) k_embed_scan(uint32_t *counts, int64_t blocks) {
    __shared__ uint32_t room[4];
    uint32_t *row = counts + blockIdx.x * blocks, sum = 0;
    for (int64_t i0 = 0; i0 < blocks; i0 += 1024) {
        const int64_t i = i0 + 4 * threadIdx.x;
        uint32_t x[4], each = 0;
#pragma unroll
        for (int u = 0; u < 4; u++) each += x[u] = i + u < blocks ? row[i + u] : 0;
        uint32_t before = sum + digits_before(each, room);
#pragma unroll
        for (int u = 0; u < 4; u++) {
            if (i + u < blocks) row[i + u] = before;
            before += x[u];
        }
        sum += room[0] + room[1] + room[2] + room[3];
        __syncthreads();
    }
    if (threadIdx.x == 0) counts[kDigits * blocks + blockIdx.x] = sum;
}

// Every place to where the counts and its rank in the workgroup say.  (Counting the next pass's digits here, by
// atomics where the places go, takes 85 us of 65,536 words of a language, whose high digits are mostly one.)
template <bool FIRST>
__global__ void __launch_bounds__(kSortThreads) k_embed_scatter(dd_embed_grad_args a, Sorted from, Sorted to, int shift, const uint32_t *counts) {
    __shared__ uint32_t next[kSortWaves][kDigits], room[kSortWaves];      // next: first counts, then places to come
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, blocks = gridDim.x;
    for (int i = lane; i < kDigits; i += 64) next[wave][i] = 0;
    const int64_t first = (int64_t)blockIdx.x * kSortBlock + wave * (kSortBlock / kSortWaves);
    uint32_t key[kSortEach], place[kSortEach], before[kSortEach];
#pragma unroll
    for (int i = 0; i < kSortEach; i++) {
        const int64_t t = first + i * 64 + lane;
        const bool in = t < a.tokens;
        key[i] = !in ? 0 : FIRST ? key_of(a, t) : from.key[t];
        place[i] = !in ? 0 : FIRST ? (uint32_t)t : from.place[t];
    }
    // this thread's digit: places of earlier digits, and of earlier workgroups
    uint32_t all = 0, mine = 0;
    if (threadIdx.x < kDigits) {
        if (blocks > kManyBlocks) {
            all = counts[(int64_t)kDigits * blocks + threadIdx.x];
            mine = counts[count_at(threadIdx.x, blockIdx.x, blocks)];
        } else {
            for (int b = 0; b < blocks; b += 16) {
                uint32_t x[16];
#pragma unroll
                for (int u = 0; u < 16; u++) x[u] = b + u < blocks ? counts[count_at(threadIdx.x, b + u, blocks)] : 0;
#pragma unroll
                for (int u = 0; u < 16; u++) {
                    all += x[u];
                    mine += b + u < (int)blockIdx.x ? x[u] : 0;
                }
            }
        }
    }
    uint32_t at = digits_before(all, room) + mine;
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int i = 0; i < kSortEach; i++) {
        const bool in = first + i * 64 + lane < a.tokens;
        const uint32_t d = key[i] >> shift & (kDigits - 1);
        const uint64_t peers = peers_of(d, in);
        const int rank = rank_among(peers);
        before[i] = next[wave][d] + rank;
        __builtin_amdgcn_wave_barrier();
        if (in && rank == 0) next[wave][d] += __popcll(peers);
        __builtin_amdgcn_wave_barrier();
    }
    __syncthreads();
    if (threadIdx.x < kDigits)
#pragma unroll
        for (int w = 0; w < kSortWaves; w++) {
            const uint32_t x = next[w][threadIdx.x];
            next[w][threadIdx.x] = at;
            at += x;
        }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kSortEach; i++) {
        if (first + i * 64 + lane >= a.tokens) continue;
        const uint32_t p = next[wave][key[i] >> shift & (kDigits - 1)] + before[i];
        to.key[p] = key[i];
        to.place[p] = place[i];
    }
}

// --- sums of runs --------------------------------------------------------------------
// LANES lanes have a chunk of CHUNK sorted places and 8 LANES columns.  A run of one id
// that lies in the chunk is stored; the part of a run that begins before the chunk goes to
// part 0 of the chunk, that of a run which goes on behind it to part 1 (a run that does
// both, to part 0).  Bound: HBM.  65,536 words of 32,000 x 1,024 bf16 in 47 us: 200 MB at 4.3 TB/s.

template <int LANES>
__device__ __forceinline__ uint32_t of_lane(uint32_t x, int i) {
    if (LANES == 64) return (uint32_t)__builtin_amdgcn_readlane((int)x, i);
    return __shfl(x, i, LANES);
}

template <class T>
__device__ __forceinline__ void store_scaled(const dd_embed_grad_args &a, int64_t id, int64_t c, int have, float (&s)[8]) {
    Pack<T, 8> p;
    float x[8];
#pragma unroll
    for (int j = 0; j < 8; j++) x[j] = s[j] * a.scale;
    p.from(x);
    p.store(static_cast<T *>(a.dtable) + id * a.dtable_stride + c, have);
}

// The first place from lo on, before hi, whose id is not k (k's come first): a wave looks at 64 places at once.
__device__ __forceinline__ int64_t behind(const uint32_t *key, int64_t lo, int64_t hi, uint32_t k) {
    while (lo < hi) {
        const int64_t step = (hi - lo + 63) / 64, p = lo + (threadIdx.x & 63) * step;
        const uint64_t past = __ballot(p >= hi || key[p < hi ? p : hi - 1] != k);
        const int n = past ? __builtin_ctzll(past) : 64;
        if (n == 0) break;
        if (lo + n * step < hi) hi = lo + n * step;
        lo += (n - 1) * step + 1;
    }
    return lo;
}

// Zeros in the rows of the table that no token has, kRowsOfWave from `filled` on by a wave: a lane looks one up,
// all of them write the row.  (200,000 tokens of 100,000 x 512 bf16: the gradient 125 us, 130 with each lane's search
// over all places.)
constexpr int kRowsOfWave = 16;
template <class T>
__device__ __forceinline__ void fill_others(const dd_embed_grad_args &a, const Sorted &in, int64_t filled, int64_t wave) {
    const int64_t first = filled + wave * kRowsOfWave, id = first + (threadIdx.x & 63);
    // the places with ids of these rows lie in [from, to): each time narrowed by what 64 places hold
    int64_t from = 0, to = a.tokens;
    for (int64_t step = 0; step != 1 && to - from > 1;) {
        const int64_t was = step, p = from + (threadIdx.x & 63) * (step = (to - from + 63) / 64);
        const uint32_t k = p < to ? in.key[p] : 0xffffffffu;
        const int64_t below = __popcll(__ballot(k < (uint64_t)first)), under = __popcll(__ballot(k < (uint64_t)first + kRowsOfWave));
        if (from + under * step < to) to = from + under * step;
        if (below) from += (below - 1) * step + 1;
        if (was && step * 2 > was) break;       // (a common word's places)
    }
    bool there = (threadIdx.x & 63) >= kRowsOfWave || id >= a.vocab;
    if (!there) {
        int64_t lo = from, hi = to;      // the first place with an id of at least this
        while (lo < hi) {
            const int64_t mid = (lo + hi) >> 1;
            if (in.key[mid] < (uint32_t)id) lo = mid + 1;
            else hi = mid;
        }
        there = lo < a.tokens && in.key[lo] == (uint32_t)id;
    }
    uint64_t none = __ballot(!there);
    Pack<T, 8> zero;
    zero.v = 0;
    while (none) {
        const int r = __builtin_ctzll(none);
        // rows in a row, where they lie end to end, are written as one
        const uint64_t after = ~(none >> r);
        const int rows = a.dtable_stride != a.cols ? 1 : after ? __builtin_ctzll(after) < 64 - r ? __builtin_ctzll(after) : 64 - r : 64 - r;
        none &= r + rows < 64 ? ~uint64_t(0) << (r + rows) : 0;
        T *to = static_cast<T *>(a.dtable) + (first + r) * a.dtable_stride;
        const int64_t n = rows * a.cols;
        for (int64_t c = 8 * (threadIdx.x & 63); c < n; c += 512) zero.store(to + c, have_of(n, c));
    }
}

// Few tokens: a workgroup has kPlaces sorted places and 128 columns, and as many groups of 16 lanes,
// each of which sums the run that begins at its place as far as the workgroup's places go.  The last run, where it goes
// on behind them, is summed by all groups, eight places each in turn, joined in order: no parts, and
// no launch to join them (2,047 tokens of 513 columns f32: 7 us, 11 with both; 2,048 times one id of 1,024
// columns bf16, all of the gradient: 32, and 30).  Bound: latency; for one id in many places, what one compute unit loads, and so few columns.
constexpr int kPlaces = 16, kFewLanes = 16;
template <class T>
__global__ void __launch_bounds__(kPlaces * kFewLanes) k_embed_few(dd_embed_grad_args a, Sorted in, int64_t blocks_of_runs, int64_t strips, int64_t filled) {
    if (blockIdx.x >= blocks_of_runs) {
        fill_others<T>(a, in, filled, (blockIdx.x - blocks_of_runs) * (kPlaces * kFewLanes / 64) + threadIdx.x / 64);
        return;
    }
    __shared__ float lds[kPlaces][8 * kFewLanes];
    const int lane = threadIdx.x % kFewLanes, wave_lane = threadIdx.x & 63;
    const int g = threadIdx.x / kFewLanes;
    const int n_tokens = (int)a.tokens, p0 = (int)(blockIdx.x / strips) * kPlaces;
    const int64_t strip = (blockIdx.x % strips) * (8 * kFewLanes), c = strip + 8 * lane;
    const int have = have_of(a.cols, c), n = n_tokens - p0 < kPlaces ? n_tokens - p0 : kPlaces;
    // ids of the places from the one before on
    const int at = p0 - 1 + wave_lane;
    const uint32_t none = 0xffffffffu, key = wave_lane <= n + 1 && at >= 0 && at < n_tokens ? in.key[at] : none;
    const uint32_t place = wave_lane < n ? in.place[p0 + wave_lane] : 0;
    const uint32_t next = __shfl_down(key, 1, 64);
    const uint64_t starts = __ballot(key != next) & ((uint64_t(1) << n) - 1);      // bit i: place i begins a run
    const bool goes_on = ((__ballot(key == next) >> n) & 1) && p0 + n < n_tokens;
    const T *dy = static_cast<const T *>(a.dy) + c;
    const uint32_t mine = __shfl(key, g + 1, 64);
    const int last = starts ? 63 - __builtin_clzll(starts) : -1;       // where the workgroup's last run begins
    const uint64_t later = starts >> g >> 1;
    const int len = !(starts >> g & 1) || mine >= (uint32_t)a.vocab || (g == last && goes_on) ? 0 : later ? __builtin_ctzll(later) + 1 : n - g;
    if (__any(len > 0)) {
        float s[8] = {};
#pragma unroll
        for (int b = 0; b < kPlaces; b += 8) {
            if (!__any(b < len)) break;
            Pack<T, 8> p[8];
#pragma unroll
            for (int i = 0; i < 8; i++) p[i].load(dy + (int64_t)__shfl(place, b + i < len ? g + b + i : g, 64) * a.dy_stride, len > 0 ? have : 0);
#pragma unroll
            for (int i = 0; i < 8; i++) {
                float x[8];
                p[i].to(x);
#pragma unroll
                for (int j = 0; j < 8; j++) s[j] += b + i < len ? x[j] : 0.0f;
            }
        }
        if (len > 0 && have > 0) store_scaled<T>(a, mine, c, have, s);
    }
    const uint32_t k = __shfl(key, last + 1, 64);
    if (last < 0 || !goes_on || k >= (uint32_t)a.vocab) return;
    const int end = (int)behind(in.key, p0 + n, n_tokens, k);
    float s[8] = {};
    // (the places are loaded a turn ahead, by as many lanes)
    auto ahead = [&](int q) { return in.place[q + (lane & 7) < end ? q + (lane & 7) : end - 1]; };
    uint32_t to_come = ahead(p0 + last + 8 * g);
    for (int q0 = p0 + last; q0 < end; q0 += 8 * kPlaces) {
        const int q = q0 + 8 * g;
        const uint32_t places = to_come;
        to_come = ahead(q + 8 * kPlaces);
        Pack<T, 8> p[8];
#pragma unroll
        for (int i = 0; i < 8; i++) p[i].load(dy + (int64_t)of_lane<kFewLanes>(places, i) * a.dy_stride, have);
#pragma unroll
        for (int i = 0; i < 8; i++) {
            float x[8];
            p[i].to(x);
#pragma unroll
            for (int j = 0; j < 8; j++) s[j] += q + i < end ? x[j] : 0.0f;
        }
    }
#pragma unroll
    for (int j = 0; j < 8; j++) lds[g][8 * lane + j] = s[j];
    __syncthreads();
    const int col = threadIdx.x;
    if (col >= 8 * kFewLanes || strip + col >= a.cols) return;
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < kPlaces; i++) sum += lds[i][col];
    static_cast<T *>(a.dtable)[k * a.dtable_stride + strip + col] = (T)(sum * a.scale);
}

template <class T, int LANES, int CHUNK>
__global__ void __launch_bounds__(256) k_embed_runs(dd_embed_grad_args a, Sorted in, float *part, int64_t chunks, uint32_t blocks_of_rows, int64_t strips, int64_t filled) {
    constexpr int kGroups = 256 / LANES;
    const int lane = threadIdx.x % LANES;
    if (blockIdx.x < blocks_of_rows) {      // (first: their lookups take time, but little else)
        fill_others<T>(a, in, filled, (int64_t)blockIdx.x * 4 + threadIdx.x / 64);
        return;
    }
    const int64_t task = (int64_t)(blockIdx.x - blocks_of_rows) * kGroups + threadIdx.x / LANES;
    const int64_t chunk = LANES == 64 ? __builtin_amdgcn_readfirstlane((int)(task / strips)) : task / strips;
    if (chunk >= chunks) return;
    const int64_t c = (task - chunk * strips) * (8 * LANES) + 8 * lane;
    const int have = have_of(a.cols, c);
    const int64_t p0 = chunk * CHUNK;
    const int n = a.tokens - p0 < CHUNK ? (int)(a.tokens - p0) : CHUNK;
    constexpr int kHold = CHUNK > LANES ? CHUNK / LANES : 1;
    uint32_t key[kHold], place[kHold];
#pragma unroll
    for (int h = 0; h < kHold; h++) {
        const int i = lane + h * LANES < n ? lane + h * LANES : n - 1;
        key[h] = in.key[p0 + i];
        place[h] = in.place[p0 + i];
    }
    auto key_at = [&](int i) { return of_lane<LANES>(key[i / LANES % kHold], i % LANES); };
    const bool from_before = p0 > 0 && in.key[p0 - 1] == key_at(0);
    const bool goes_on = p0 + n < a.tokens && in.key[p0 + n] == of_lane<LANES>(key[(CHUNK - 1) / LANES], (CHUNK - 1) % LANES);
    const T *dy = static_cast<const T *>(a.dy) + c;
    float s[8] = {};
    bool whole = !from_before;      // the run began in this chunk
#pragma unroll
    for (int b = 0; b < CHUNK; b += 8) {
        if (b >= n) break;
        Pack<T, 8> p[8];
#pragma unroll
        for (int i = 0; i < 8; i++) {
            const uint32_t t = of_lane<LANES>(place[(b + i) / LANES % kHold], (b + i) % LANES);
            const bool real = b + i < n && key_at(b + i) < (uint32_t)a.vocab;
            p[i].load(dy + (int64_t)t * a.dy_stride, real ? have : 0);
        }
#pragma unroll
        for (int i = 0; i < 8; i++) {
            if (b + i >= n) break;
            const uint32_t k = key_at(b + i);
            float x[8];
            p[i].to(x);
#pragma unroll
            for (int j = 0; j < 8; j++) s[j] += x[j];
            const bool last = b + i + 1 == n;
            if (!last && key_at(b + i + 1 < CHUNK ? b + i + 1 : b + i) == k) continue;
            // the run ends, or the chunk does
            if (have > 0 && k < (uint32_t)a.vocab) {
                if (whole && !(last && goes_on)) {
                    store_scaled<T>(a, k, c, have, s);
                } else {
                    Pack<float, 8> f;
                    f.from(s);
                    f.store(part + (2 * chunk + (whole ? 1 : 0)) * a.cols + c, have);
                }
            }
            whole = true;
#pragma unroll
            for (int j = 0; j < 8; j++) s[j] = 0.0f;
        }
    }
}

// Runs over several chunks.  A wave looks at the chunk that a run may begin in, for 256 columns.  It sums the
// parts of a short run by itself; those of a longer one are summed by the workgroup's waves, each in turn eight of
// them, and joined in order.
constexpr int kJoinWaves = 8, kJoinAtOnce = 8, kJoinAlone = 2 * kJoinAtOnce;
template <class T, int CHUNK>
__global__ void __launch_bounds__(64 * kJoinWaves) k_embed_join(dd_embed_grad_args a, Sorted in, const float *part) {
    __shared__ float lds[kJoinWaves][256];
    __shared__ int lasts[kJoinWaves];
    __shared__ uint32_t ids[kJoinWaves];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int first = blockIdx.x * kJoinWaves, mine = first + wave;
    const int64_t end = (int64_t)(mine + 1) * CHUNK;
    // (0: no run over several chunks begins in the wave's)
    int last = 0;
    uint32_t id = 0;
    if (end < a.tokens) {
        id = in.key[end - 1];
        const uint32_t next = in.key[end], begin = in.key[end - CHUNK], before = in.key[mine > 0 ? end - CHUNK - 1 : 0];
        if (id < (uint32_t)a.vocab && next == id && !(begin == id && mine > 0 && before == id)) last = __builtin_amdgcn_readfirstlane((int)((behind(in.key, end, a.tokens, id) - 1) / CHUNK));
    }
    if (lane == 0) {
        lasts[wave] = last;
        ids[wave] = id;
    }
    __syncthreads();
    auto sum = [&](int chunk, int to, int i, int by, int64_t c, int have, float (&s)[4]) __attribute__((always_inline)) {
        for (; i <= to; i += by * kJoinAtOnce) {
            Pack<float, 4> f[kJoinAtOnce];
#pragma unroll
            for (int u = 0; u < kJoinAtOnce; u++) {
                f[u].v = 0.0f;
                if (i + by * u <= to) f[u].load(part + (2 * (int64_t)(i + by * u) + (i + by * u == chunk ? 1 : 0)) * a.cols + c, have);
            }
#pragma unroll
            for (int u = 0; u < kJoinAtOnce; u++) {
                float v[4];
                f[u].to(v);
#pragma unroll
                for (int j = 0; j < 4; j++) s[j] += v[j];
            }
        }
    };
    for (int64_t c0 = (int64_t)blockIdx.y * 256; c0 < a.cols; c0 += (int64_t)gridDim.y * 256) {
        const int64_t c = c0 + 4 * lane;
        const int have = a.cols - c >= 4 ? 4 : a.cols - c < 0 ? 0 : (int)(a.cols - c);
        if (last && last - mine < kJoinAlone) {
            float s[4] = {};
            sum(mine, last, mine, 1, c, have, s);
            Pack<T, 4> p;
#pragma unroll
            for (int j = 0; j < 4; j++) s[j] *= a.scale;
            p.from(s);
            p.store(static_cast<T *>(a.dtable) + id * a.dtable_stride + c, have);
        }
        for (int w = 0; w < kJoinWaves; w++) {
            const int chunk = first + w, to = __builtin_amdgcn_readfirstlane(lasts[w]);
            if (!to || to - chunk < kJoinAlone) continue;
            float s[4] = {};
            sum(chunk, to, chunk + wave, kJoinWaves, c, have, s);
            __syncthreads();
#pragma unroll
            for (int j = 0; j < 4; j++) lds[wave][4 * lane + j] = s[j];
            __syncthreads();
            if (threadIdx.x < 256 && c0 + threadIdx.x < a.cols) {
                float t = 0.0f;
#pragma unroll
                for (int g = 0; g < kJoinWaves; g++) t += lds[g][threadIdx.x];
                static_cast<T *>(a.dtable)[ids[w] * a.dtable_stride + c0 + threadIdx.x] = (T)(t * a.scale);
            }
        }
    }
}

// Working memory of the gradient: two lists of sorted tokens, counts, parts.
// Few tokens are summed without parts unless a group's one load at a time counts (8,192 tokens of 32,000 x 1,024 bf16:
// 45 us, 41 with parts), and in short chunks, as there is little to go round.
constexpr int64_t kSmallTokens = kSmallThreads * 8;
int chunk_of(int64_t tokens) { return tokens <= kSmallTokens ? 8 : 32; }
bool without_parts(int64_t tokens, int64_t cols) { return tokens <= kSmallTokens && tokens * cols <= (1 << 22); }
struct Room {
    int64_t blocks, chunks, counts, part, bytes;     // places in bytes
    int passes;
};
Room room_of(int64_t tokens, int64_t vocab, int64_t cols) {
    Room r;
    r.blocks = (tokens + kSortBlock - 1) / kSortBlock;
    r.chunks = without_parts(tokens, cols) ? 0 : (tokens + chunk_of(tokens) - 1) / chunk_of(tokens);
    r.passes = 1;
    while (r.passes < 4 && (uint64_t)vocab >> (8 * r.passes)) r.passes++;
    r.counts = (tokens * 16 + 15) / 16 * 16;
    r.part = r.counts + (r.blocks + 1) * kDigits * 4;
    r.bytes = r.part + r.chunks * 2 * cols * 4;
    return r;
}

// filled: rows that are zeros; of the others, those that no token has are looked up and written too
int64_t waves_of_rows(const dd_embed_grad_args &a, int64_t filled) { return (a.vocab - filled + kRowsOfWave - 1) / kRowsOfWave; }

template <class T>
void few_runs(const dd_embed_grad_args &a, const Sorted &in, int64_t filled, hipStream_t s) {
    const int64_t strips = (a.cols + 8 * kFewLanes - 1) / (8 * kFewLanes), waves = kPlaces * kFewLanes / 64;
    const int64_t of_runs = (a.tokens + kPlaces - 1) / kPlaces * strips, of_rows = (waves_of_rows(a, filled) + waves - 1) / waves;
    k_embed_few<T><<<(unsigned)(of_runs + of_rows), kPlaces * kFewLanes, 0, s>>>(a, in, of_runs, strips, filled);
}

template <class T, int LANES, int CHUNK>
void runs(const dd_embed_grad_args &a, const Sorted &in, float *part, const Room &r, int64_t filled, hipStream_t s) {
    const int64_t strips = (a.cols + 8 * LANES - 1) / (8 * LANES), groups = 256 / LANES;
    const int64_t of_runs = (r.chunks * strips + groups - 1) / groups, of_rows = (waves_of_rows(a, filled) + 3) / 4;
    k_embed_runs<T, LANES, CHUNK><<<(unsigned)(of_runs + of_rows), 256, 0, s>>>(a, in, part, r.chunks, (uint32_t)of_rows, strips, filled);
    if (r.chunks < 2) return;
    const int64_t y = (a.cols + 255) / 256;
    k_embed_join<T, CHUNK><<<dim3((unsigned)((r.chunks + kJoinWaves - 1) / kJoinWaves), (unsigned)(y < 1024 ? y : 1024)), 64 * kJoinWaves, 0, s>>>(a, in, part);
}

template <class T>
void embed_grad(const dd_embed_grad_args &a, void *work, hipStream_t s) {
    const Room r = room_of(a.tokens, a.vocab, a.cols);
    char *w = static_cast<char *>(work);
    uint32_t *list = reinterpret_cast<uint32_t *>(w);
    float *part = reinterpret_cast<float *>(w + r.part);
    Sorted from{list, list + a.tokens}, to{list + 2 * a.tokens, list + 3 * a.tokens};
    // Few tokens in a large table: nearly all of it is zeros, written while the tokens are sorted (a row that a
    // token has twice then).  Many: the rows that no token has are looked up and written beside the sums.  2,047 tokens
    // of 50,021 x 513 f32 take 30 us, 35 with the rows looked up.
    const int64_t filled = a.tokens > 0 && a.tokens < a.vocab / 8 ? a.vocab : 0;
    const int64_t packs = filled * ((a.cols + 7) / 8);
    auto fillers = [&](int threads) { return (packs + 4 * threads - 1) / (4 * threads) < 2048 ? (packs + 4 * threads - 1) / (4 * threads) : 2048; };
    if (a.tokens > 0 && a.tokens <= kSmallTokens) {
        const unsigned grid = (unsigned)(1 + fillers(kSmallThreads));
        if (a.tokens <= 2 * kSmallThreads) k_embed_sort<T, 2><<<grid, kSmallThreads, 0, s>>>(a, from, r.passes, filled);
        else k_embed_sort<T, 8><<<grid, kSmallThreads, 0, s>>>(a, from, r.passes, filled);
    } else if (a.tokens > 0) {
        uint32_t *counts = reinterpret_cast<uint32_t *>(w + r.counts);
        const unsigned blocks = (unsigned)r.blocks;
        for (int i = 0; i < r.passes; i++) {
            if (i == 0) k_embed_count<T, true><<<(unsigned)(r.blocks + fillers(kSortThreads)), kSortThreads, 0, s>>>(a, from, 0, (int)r.blocks, counts, filled);
            else k_embed_count<T, false><<<blocks, kSortThreads, 0, s>>>(a, from, 8 * i, (int)r.blocks, counts, 0);
            if (r.blocks > kManyBlocks) k_embed_scan<<<kDigits, 256, 0, s>>>(counts, r.blocks);
            if (i == 0) k_embed_scatter<true><<<blocks, kSortThreads, 0, s>>>(a, from, to, 0, counts);
            else k_embed_scatter<false><<<blocks, kSortThreads, 0, s>>>(a, from, to, 8 * i, counts);
            const Sorted x = from;
            from = to;
            to = x;
        }
    }
    if (without_parts(a.tokens, a.cols)) few_runs<T>(a, from, filled, s);
    else if (a.tokens <= kSmallTokens) a.cols <= 128 ? runs<T, 16, 8>(a, from, part, r, filled, s) : runs<T, 64, 8>(a, from, part, r, filled, s);
    else a.cols <= 128 ? runs<T, 16, 32>(a, from, part, r, filled, s) : runs<T, 64, 32>(a, from, part, r, filled, s);
}

}  // namespace

template <class T>
static void embed(const dd_embed_args &a, hipStream_t s) {
    // (two of 16 bits fill the compute units' queues: 65,536 words of 32,000 x 1,024 bf16 43 us, 49 with one, 42 with
    // eight; 32 bits have two loads as it is: x 1,000 87, 88 with two)
    constexpr int kEach = sizeof(T) == 2 ? 2 : 1;
    const int64_t packs = (a.cols + 7) / 8, need = (a.tokens * packs + 255) / 256;
    if (need < 4096) k_embed<T, 1><<<(unsigned)need, 256, 0, s>>>(a, (uint32_t)packs);
    else k_embed<T, kEach><<<(unsigned)(need / kEach < (1 << 20) ? (need + kEach - 1) / kEach : (1 << 20)), 256, 0, s>>>(a, (uint32_t)packs);
}

hipError_t launch_embed(const dd_embed_args &a, hipStream_t s) {
    if (a.type == DD_F32) embed<float>(a, s);
    else if (a.type == DD_BF16) embed<bf16_t>(a, s);
    else embed<f16_t>(a, s);
    return hipGetLastError();
}

size_t embed_grad_work(int64_t tokens, int64_t vocab, int64_t cols) { return tokens > 0 ? (size_t)room_of(tokens, vocab, cols).bytes : 0; }

hipError_t launch_embed_grad(const dd_embed_grad_args &a, void *work, hipStream_t s) {
    if (a.type == DD_F32) embed_grad<float>(a, work, s);
    else if (a.type == DD_BF16) embed_grad<bf16_t>(a, work, s);
    else embed_grad<f16_t>(a, work, s);
    return hipGetLastError();
}

}  // namespace dd
