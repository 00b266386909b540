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

// A thread has eight columns of a token.  Bound: HBM; few tokens, the launch.
template <class T>
__global__ void __launch_bounds__(256) k_embed(dd_embed_args a, uint32_t packs) {
    const int64_t total = a.tokens * packs;
    for (int64_t i = blockIdx.x * (int64_t)256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
        const int64_t t = (uint64_t)i >> 32 ? i / packs : (int64_t)((uint32_t)i / packs);
        const int64_t c = (i - t * packs) * 8;
        const int have = have_of(a.cols, c);
        const int64_t id = id_at(a.ids, a.id_bytes, t);
        Pack<T, 8> p;
        float x[8];
        if (id >= 0 && id < a.vocab) {
            p.load(static_cast<const T *>(a.table) + id * a.table_stride + c, have);
            p.to(x);
#pragma unroll
            for (int j = 0; j < 8; j++) x[j] *= a.scale;
        } else {
#pragma unroll
            for (int j = 0; j < 8; j++) x[j] = __builtin_nanf("");
        }
        p.from(x);
        p.store(static_cast<T *>(a.out) + t * a.out_stride + c, have);
    }
}

// --- the tokens in the order of their ids -------------------------------------------
// Least significant digits of eight bits first.  A workgroup has kSortBlock places in a row
// and a wave a run of them, so ranks count waves, then lanes, in order (stable).  Ids
// that do not count (pad, or not in the table) are `vocab`, behind all others.
constexpr int kSortThreads = 256, kSortWaves = kSortThreads / 64, kSortEach = 8, kSortBlock = kSortThreads * kSortEach, kDigits = 256;

struct Sorted {
    uint32_t *key, *place;       // id and token
};

__device__ __forceinline__ uint32_t key_of(const dd_embed_grad_args &a, int64_t t) {
    const int64_t id = id_at(a.ids, a.id_bytes, t);
    return id < 0 || id >= a.vocab || id == a.pad ? (uint32_t)a.vocab : (uint32_t)id;
}

// counts[digit][workgroup]: a workgroup's places with each digit
template <bool FIRST>
__global__ void __launch_bounds__(kSortThreads) k_embed_count(dd_embed_grad_args a, Sorted from, int shift, uint32_t *counts) {
    __shared__ uint32_t n[kDigits];
    n[threadIdx.x] = 0;
    __syncthreads();
    const int64_t first = (int64_t)blockIdx.x * kSortBlock;
#pragma unroll
    for (int i = 0; i < kSortEach; i++) {
        const int64_t t = first + i * kSortThreads + threadIdx.x;
        if (t < a.tokens) atomicAdd(&n[(FIRST ? key_of(a, t) : from.key[t]) >> shift & (kDigits - 1)], 1u);
    }
    __syncthreads();
    counts[(int64_t)threadIdx.x * gridDim.x + blockIdx.x] = n[threadIdx.x];
}

// Running sums of all counts, in place: each of 1,024 threads has a run of them.
__global__ void __launch_bounds__(1024) k_embed_scan(uint32_t *counts, int64_t n) {
    __shared__ uint32_t of_wave[16];
    const int64_t each = (n + 1023) / 1024, i0 = threadIdx.x * each, i1 = i0 + each < n ? i0 + each : n;
    uint32_t sum = 0;
    for (int64_t i = i0; i < i1; i++) sum += counts[i];
    uint32_t run = sum;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const uint32_t x = __shfl_up(run, o, 64);
        if ((threadIdx.x & 63) >= (unsigned)o) run += x;
    }
    if ((threadIdx.x & 63) == 63) of_wave[threadIdx.x >> 6] = run;
    __syncthreads();
    uint32_t before = run - sum;
    for (int w = 0; w < (int)(threadIdx.x >> 6); w++) before += of_wave[w];
    for (int64_t i = i0; i < i1; i++) {
        const uint32_t x = counts[i];
        counts[i] = before;
        before += x;
    }
}

// Every place to where the running sums and its rank in the workgroup say.
template <bool FIRST>
__global__ void __launch_bounds__(kSortThreads) k_embed_scatter(dd_embed_grad_args a, Sorted from, Sorted to, int shift, const uint32_t *sums) {
    __shared__ uint32_t next[kSortWaves][kDigits];      // first counts, then places to come
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (int i = lane; i < kDigits; i += 64) next[wave][i] = 0;
    __syncthreads();
    const int64_t first = (int64_t)blockIdx.x * kSortBlock + wave * (kSortBlock / kSortWaves);
    uint32_t key[kSortEach], place[kSortEach], before[kSortEach];
#pragma unroll
    for (int i = 0; i < kSortEach; i++) {
        const int64_t t = first + i * 64 + lane;
        const bool in = t < a.tokens;
        key[i] = !in ? 0 : FIRST ? key_of(a, t) : from.key[t];
        place[i] = !in ? 0 : FIRST ? (uint32_t)t : from.place[t];
    }
#pragma unroll
    for (int i = 0; i < kSortEach; i++) {
        const bool in = first + i * 64 + lane < a.tokens;
        const uint32_t d = key[i] >> shift & (kDigits - 1);
        uint64_t same = __ballot(in);
#pragma unroll
        for (int b = 0; b < 8; b++) {
            const uint64_t set = __ballot(d >> b & 1);
            same &= d >> b & 1 ? set : ~set;
        }
        const uint32_t rank = __popcll(same & ((uint64_t(1) << lane) - 1));
        before[i] = next[wave][d] + rank;
        __builtin_amdgcn_wave_barrier();
        if (in && rank == 0) next[wave][d] += __popcll(same);
        __builtin_amdgcn_wave_barrier();
    }
    __syncthreads();
    uint32_t at = sums[(int64_t)threadIdx.x * gridDim.x + blockIdx.x];
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
// LANES lanes have a chunk of kChunk sorted places and 8 LANES columns.  A run of one id
// that lies in the chunk is stored; the part of a run that begins before the chunk goes to
// part 0 of the chunk, that of a run which goes on behind it to part 1 (a run that does
// both, to part 0).
constexpr int kChunk = 32;

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

template <class T, int LANES>
__global__ void __launch_bounds__(256) k_embed_runs(dd_embed_grad_args a, Sorted in, float *part, int64_t chunks, int64_t blocks_of_runs, int64_t strips) {
    constexpr int kGroups = 256 / LANES;
    const int lane = threadIdx.x % LANES;
    if (blockIdx.x >= blocks_of_runs) {
        // rows of the table that no token has: a lane looks one up, all of them write the row
        const int64_t first = (blockIdx.x - blocks_of_runs) * 256 + threadIdx.x / 64 * 64;
        const int64_t id = first + (threadIdx.x & 63);
        bool there = id >= a.vocab;
        if (!there) {
            int64_t lo = 0, hi = a.tokens;      // the first place with an id of at least this
            while (lo < hi) {
                const int64_t mid = (lo + hi) >> 1;
                if (in.key[mid] < (uint32_t)id) lo = mid + 1;
                else hi = mid;
            }
            there = lo < a.tokens && in.key[lo] == (uint32_t)id;
        }
        uint64_t none = __ballot(!there);
        while (none) {
            const int64_t row = first + __builtin_ctzll(none);
            none &= none - 1;
            for (int64_t c = 8 * (threadIdx.x & 63); c < a.cols; c += 512) {
                float zero[8] = {};
                store_scaled<T>(a, row, c, have_of(a.cols, c), zero);
            }
        }
        return;
    }
    const int64_t task = (int64_t)blockIdx.x * kGroups + threadIdx.x / LANES;
    const int64_t chunk = LANES == 64 ? __builtin_amdgcn_readfirstlane((int)(task / strips)) : task / strips;
    if (chunk >= chunks) return;
    const int64_t c = (task - chunk * strips) * (8 * LANES) + 8 * lane;
    const int have = have_of(a.cols, c);
    const int64_t p0 = chunk * kChunk;
    const int n = a.tokens - p0 < kChunk ? (int)(a.tokens - p0) : kChunk;
    constexpr int kHold = kChunk > LANES ? kChunk / LANES : 1;
    uint32_t key[kHold], place[kHold];
#pragma unroll
    for (int h = 0; h < kHold; h++) {
        const int i = lane + h * LANES < n ? lane + h * LANES : n - 1;
        key[h] = in.key[p0 + i];
        place[h] = in.place[p0 + i];
    }
    auto key_at = [&](int i) { return of_lane<LANES>(key[i / LANES % kHold], i % LANES); };
    const bool from_before = p0 > 0 && in.key[p0 - 1] == key_at(0);
    const bool goes_on = p0 + n < a.tokens && in.key[p0 + n] == of_lane<LANES>(key[(kChunk - 1) / LANES], (kChunk - 1) % LANES);
    const T *dy = static_cast<const T *>(a.dy) + c;
    float s[8] = {};
    bool whole = !from_before;      // the run began in this chunk
#pragma unroll
    for (int b = 0; b < kChunk; b += 8) {
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
            if (!last && key_at(b + i + 1 < kChunk ? b + i + 1 : b + i) == k) continue;
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

// Runs over several chunks.  A workgroup has the chunk a run begins in and 64 columns: its 32
// groups of eight lanes sum every 32nd of the run's parts, and the groups are joined in
// order.
template <class T>
__global__ void __launch_bounds__(256) k_embed_join(dd_embed_grad_args a, Sorted in, const float *part, int64_t chunks) {
    __shared__ float lds[32][64];
    __shared__ int64_t last_chunk;
    const int64_t chunk = blockIdx.x, end = (chunk + 1) * kChunk;
    if (end >= a.tokens) return;
    const uint32_t k = in.key[end - 1];
    if (k >= (uint32_t)a.vocab || in.key[end] != k) return;
    // (begun in this chunk: its first place has another id, or follows one)
    if (in.key[end - kChunk] == k && chunk > 0 && in.key[end - kChunk - 1] == k) return;
    if (threadIdx.x == 0) {
        int64_t lo = end, hi = a.tokens;        // the first place behind the run
        while (lo < hi) {
            const int64_t mid = (lo + hi) >> 1;
            if (in.key[mid] == k) lo = mid + 1;
            else hi = mid;
        }
        last_chunk = (lo - 1) / kChunk;
    }
    __syncthreads();
    const int64_t last = last_chunk;
    const int x = threadIdx.x & 7, y = threadIdx.x >> 3;
    for (int64_t c0 = (int64_t)blockIdx.y * 64; c0 < a.cols; c0 += (int64_t)gridDim.y * 64) {
        const int64_t c = c0 + 8 * x;
        const int have = have_of(a.cols, c);
        float s[8] = {};
        for (int64_t i = chunk + y; i <= last; i += 32) {
            Pack<float, 8> f;
            float v[8];
            f.load(part + (2 * i + (i == chunk ? 1 : 0)) * a.cols + c, have);
            f.to(v);
#pragma unroll
            for (int j = 0; j < 8; j++) s[j] += v[j];
        }
        __syncthreads();
#pragma unroll
        for (int j = 0; j < 8; j++) lds[y][8 * x + j] = s[j];
        __syncthreads();
        if (y == 0) {
#pragma unroll
            for (int j = 0; j < 8; j++) s[j] = 0.0f;
            for (int g = 0; g < 32; g++)
#pragma unroll
                for (int j = 0; j < 8; j++) s[j] += lds[g][8 * x + j];
            if (have > 0) store_scaled<T>(a, k, c, have, s);
        }
    }
}

// Working memory of the gradient: two lists of sorted tokens, counts, parts.
struct Room {
    int64_t blocks, chunks, counts, part, bytes;     // places in bytes
    int passes;
};
Room room_of(int64_t tokens, int64_t vocab, int64_t cols) {
    Room r;
    r.blocks = (tokens + kSortBlock - 1) / kSortBlock;
    r.chunks = (tokens + kChunk - 1) / kChunk;
    r.passes = 1;
    while (r.passes < 4 && (uint64_t)vocab >> (8 * r.passes)) r.passes++;
    r.counts = (tokens * 16 + 15) / 16 * 16;
    r.part = r.counts + r.blocks * kDigits * 4;
    r.bytes = r.part + r.chunks * 2 * cols * 4;
    return r;
}

template <class T, int LANES>
void runs(const dd_embed_grad_args &a, const Sorted &in, float *part, const Room &r, hipStream_t s) {
    const int64_t strips = (a.cols + 8 * LANES - 1) / (8 * LANES), groups = 256 / LANES;
    const int64_t of_runs = (r.chunks * strips + groups - 1) / groups, of_rows = (a.vocab + 255) / 256;
    k_embed_runs<T, LANES><<<(unsigned)(of_runs + of_rows), 256, 0, s>>>(a, in, part, r.chunks, of_runs, strips);
    if (r.chunks > 1)
        k_embed_join<T><<<dim3((unsigned)r.chunks, (unsigned)((a.cols + 63) / 64 < 1024 ? (a.cols + 63) / 64 : 1024)), 256, 0, s>>>(a, in, part, r.chunks);
}

template <class T>
void embed_grad(const dd_embed_grad_args &a, void *work, hipStream_t s) {
    const Room r = room_of(a.tokens, a.vocab, a.cols);
    char *w = static_cast<char *>(work);
    uint32_t *list = reinterpret_cast<uint32_t *>(w), *counts = reinterpret_cast<uint32_t *>(w + r.counts);
    float *part = reinterpret_cast<float *>(w + r.part);
    Sorted from{list, list + a.tokens}, to{list + 2 * a.tokens, list + 3 * a.tokens};
    for (int i = 0; i < r.passes && a.tokens > 0; i++) {
        if (i == 0) k_embed_count<true><<<(unsigned)r.blocks, kSortThreads, 0, s>>>(a, from, 8 * i, counts);
        else k_embed_count<false><<<(unsigned)r.blocks, kSortThreads, 0, s>>>(a, from, 8 * i, counts);
        k_embed_scan<<<1, 1024, 0, s>>>(counts, r.blocks * kDigits);
        if (i == 0) k_embed_scatter<true><<<(unsigned)r.blocks, kSortThreads, 0, s>>>(a, from, to, 8 * i, counts);
        else k_embed_scatter<false><<<(unsigned)r.blocks, kSortThreads, 0, s>>>(a, from, to, 8 * i, counts);
        const Sorted x = from;
        from = to;
        to = x;
    }
    if (a.cols <= 128) runs<T, 16>(a, from, part, r, s);
    else runs<T, 64>(a, from, part, r, s);
}

}  // namespace

hipError_t launch_embed(const dd_embed_args &a, hipStream_t s) {
    const int64_t packs = (a.cols + 7) / 8, need = (a.tokens * packs + 255) / 256;
    const unsigned grid = (unsigned)(need < (1 << 20) ? need : (1 << 20));
    if (a.type == DD_F32) k_embed<float><<<grid, 256, 0, s>>>(a, (uint32_t)packs);
    else if (a.type == DD_BF16) k_embed<bf16_t><<<grid, 256, 0, s>>>(a, (uint32_t)packs);
    else k_embed<f16_t><<<grid, 256, 0, s>>>(a, (uint32_t)packs);
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
