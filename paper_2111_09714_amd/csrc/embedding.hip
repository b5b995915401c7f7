// Embedding lookup with positions, and its gradient by sorted tokens (gfx950).
//
//   y[t] = scale table[ids[t]] + pos[t mod n];  ids outside [0, vocab) have no row (0)
//   dtable[v] = scale sum_{t : ids[t] = v} dy[t],   dpos[p] = sum_b dy[b n + p]
//
// The lookup is a gather of rows, L lanes to a row.  The gradient never adds to memory: tokens are
// put in the order of their ids and every row of dtable is one sum in the order of its tokens,
// the same bits every time.
//
//   rank   per block of tokens: how many fall into each bucket of W = 2^s neighbouring ids (at most 4096
//          buckets), and each token's rank among them, from ballots over its wave; place  the block's start
//          in every bucket from all blocks' counts, then each token to its place.  Both are short and
//          use few CUs; the rest of the card writes dtable's zeros meanwhile (half in each launch),
//          which the rows that occur overwrite.  Few tokens are ranked and placed by one block.
//   sum    one workgroup per chunk of up to E tokens, of a few neighbouring buckets or a part of a full
//          one: orders them by id in LDS, then groups of lanes add their shares of that order, runs that
//          cross groups through LDS.  Buckets within one chunk end in dtable; of a bucket of several
//          (frequent ids) each chunk leaves fp32 rows of its ids,
//   join   and those are added in chunk order.
#include "common.h"
#include "launch.h"
#include "rows.h"
#include "timing.h"

namespace yoso {

namespace {

// ------------------------------------------------------------------ lookup

constexpr int kLookThreads = 256;

template <bool BF16, int LAYOUT, int L, typename ID>
__global__ __launch_bounds__(kLookThreads) void embedding_kernel(Embedding a) {
    constexpr int N = Vec<BF16>::N, G = kLookThreads / L;
    using Cols = Columns<BF16, LAYOUT>;
    const int lane = threadIdx.x % L, group = threadIdx.x / L, d = a.d, nvec = (d + N - 1) / N;
    const int64_t step = static_cast<int64_t>(gridDim.x) * G;
    for (int64_t t = static_cast<int64_t>(blockIdx.x) * G + group; t < a.tokens; t += step) {
        const int64_t id = static_cast<const ID *>(a.ids)[t];
        const bool named = id >= 0 && id < a.vocab;
        const int64_t from = named ? id * d : 0;
        const int64_t pos = a.n ? static_cast<int64_t>(static_cast<uint32_t>(t) % static_cast<uint32_t>(a.n)) * d : 0;
#pragma unroll 4
        for (int i = lane; i < nvec; i += L) {
            const Cols col(i, d);
            const raw4 v = load_vec(a.table, from, col, d, named);
            float f[N];
            if (a.n) {
                const raw4 p = load_vec(a.pos, pos, col, d, true);
#pragma unroll
                for (int j = 0; j < N; j++)
                    f[j] = named ? fmaf(a.scale, value<BF16>(v, j), value<BF16>(p, j)) : value<BF16>(p, j);
            } else {
#pragma unroll
                for (int j = 0; j < N; j++) f[j] = named ? a.scale * value<BF16>(v, j) : 0.f;
            }
            store_vec(a.y, t * d, col, d, true, pack<BF16>(f));
        }
    }
}

// ------------------------------------------------------------------ order of the tokens

constexpr int kSortThreads = 512, kSortWaves = kSortThreads / 64;
constexpr int kMaxBuckets = 4096, kOwn = kMaxBuckets / kSortThreads;  // buckets of a thread
constexpr int kBatch = 2048, kPer = kBatch / kSortThreads;            // tokens ranked at once, by a block and by a thread
constexpr int kMaxEntries = 256;
constexpr uint32_t kNoSlot = 0xFFFFFFFFu;

struct Order {
    const void *ids;
    int64_t tokens, vocab;
    int shift, buckets, blocks, entries;  // entries: of a chunk, at most
    int64_t block_tokens;
    uint16_t *counts;  // [blocks][kMaxBuckets]
    uint16_t *rank;    // [tokens] within the block's tokens of the bucket
    uint32_t *token;   // [tokens] in bucket order
    uint32_t *id;      // their ids
    uint4 *items;      // chunks: first entry, entries, slot of partial rows
    uint4 *multi;      // buckets of several chunks: bucket, first slot, chunks
    uint32_t *head;    // number of items, of buckets of several chunks
    // zeros written beside
    uint4 *zero;
    int64_t zero_from, zero_to;  // 16-byte vectors
    int64_t zero_bytes;          // the end, where it is not a whole vector
};

constexpr int kZeroPerThread = 16;  // vectors

__device__ __forceinline__ void write_zeros(const Order &o, int64_t block) {
    const int64_t at = o.zero_from + block * kSortThreads * kZeroPerThread + threadIdx.x;
#pragma unroll
    for (int k = 0; k < kZeroPerThread; k++) {
        const int64_t v = at + static_cast<int64_t>(k) * kSortThreads;
        if (v < o.zero_to) {
            if (16 * v + 16 <= o.zero_bytes)
                o.zero[v] = make_uint4(0, 0, 0, 0);
            else
                for (int64_t b = 16 * v; b < o.zero_bytes; b += 2) *reinterpret_cast<uint16_t *>(reinterpret_cast<char *>(o.zero) + b) = 0;
        }
    }
}

// the id of token t, or -1 where it names no row
template <typename ID>
__device__ __forceinline__ int id_of(const Order &o, int64_t t, int64_t end) {
    if (t >= end) return -1;
    const int64_t id = static_cast<const ID *>(o.ids)[t];
    return id >= 0 && id < o.vocab ? static_cast<int>(id) : -1;
}

// Ranks of kBatch tokens from `at`: wave w takes the tokens w 64 kPer ... of them, 64 at a time.  The
// rank counts tokens of the same bucket that come before: in this batch, and in `run`, [kMaxBuckets],
// which is counted on.  wave_counts [kSortWaves][kMaxBuckets]; ends with a barrier.
template <typename ID>
__device__ __forceinline__ void rank_batch(const Order &o, int64_t at, int64_t end, uint16_t *wave_counts, uint16_t *run,
                                           int (&id)[kPer], uint32_t (&rank)[kPer]) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t t0 = at + wave * 64 * kPer + lane;
#pragma unroll
    for (int k = 0; k < kPer; k++) id[k] = id_of<ID>(o, t0 + 64 * k, end);
    uint16_t *count = wave_counts + wave * kMaxBuckets;
    for (int i = lane; i < (o.buckets + 7) / 8; i += 64) reinterpret_cast<uint4 *>(count)[i] = make_uint4(0, 0, 0, 0);
    const int bits = 32 - __clz(o.buckets - 1);  // (0 for one bucket: clz(0) = 32)
#pragma unroll
    for (int k = 0; k < kPer; k++) {
        const int b = id[k] >> o.shift;
        unsigned long long same = __ballot(id[k] >= 0);
        for (int i = 0; i < bits; i++) {
            const unsigned long long m = __ballot((b >> i) & 1);
            same &= (b >> i) & 1 ? m : ~m;
        }
        rank[k] = 0;
        if (id[k] >= 0) {
            const uint32_t before = count[b];
            rank[k] = before + __popcll(same & ((1ull << lane) - 1));
            if (lane == 63 - __clzll(same)) count[b] = static_cast<uint16_t>(rank[k] + 1);
        }
    }
    __syncthreads();
    for (int b = threadIdx.x; b < o.buckets; b += kSortThreads) {
        uint32_t sum = run[b];
#pragma unroll
        for (int w = 0; w < kSortWaves; w++) {
            const uint32_t c = wave_counts[w * kMaxBuckets + b];
            wave_counts[w * kMaxBuckets + b] = static_cast<uint16_t>(sum);
            sum += c;
        }
        run[b] = static_cast<uint16_t>(sum);
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kPer; k++)
        if (id[k] >= 0) rank[k] += count[id[k] >> o.shift];
    __syncthreads();
}

constexpr size_t kRankLds = (kSortWaves + 1) * kMaxBuckets * sizeof(uint16_t);

template <typename ID>
__global__ __launch_bounds__(kSortThreads) void embedding_rank_kernel(Order o) {
    if (static_cast<int>(blockIdx.x) >= o.blocks) return write_zeros(o, blockIdx.x - o.blocks);
    extern __shared__ uint16_t lds16[];
    uint16_t *run = lds16, *wave_counts = lds16 + kMaxBuckets;
    for (int b = threadIdx.x; b < kMaxBuckets; b += kSortThreads) run[b] = 0;
    const int64_t from = blockIdx.x * o.block_tokens, to = from + o.block_tokens;
    const int64_t end = to < o.tokens ? to : o.tokens;
    for (int64_t at = from; at < end; at += kBatch) {
        int id[kPer];
        uint32_t rank[kPer];
        rank_batch<ID>(o, at, end, wave_counts, run, id, rank);
        const int64_t t0 = at + (threadIdx.x >> 6) * 64 * kPer + (threadIdx.x & 63);
#pragma unroll
        for (int k = 0; k < kPer; k++)
            if (id[k] >= 0) o.rank[t0 + 64 * k] = static_cast<uint16_t>(rank[k]);
    }
    uint4 *out = reinterpret_cast<uint4 *>(o.counts + static_cast<int64_t>(blockIdx.x) * kMaxBuckets);
    for (int i = threadIdx.x; i < kMaxBuckets / 8; i += kSortThreads) out[i] = reinterpret_cast<const uint4 *>(run)[i];
}

// exclusive sums of four values over the workgroup's threads
struct Four {
    uint32_t v[4];
};

__device__ __forceinline__ Four scan4(Four own, Four *wave_sums, Four &total) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    Four s = own;
#pragma unroll
    for (int k = 1; k < 64; k *= 2)
#pragma unroll
        for (int q = 0; q < 4; q++) {
            const uint32_t x = __shfl_up(s.v[q], k);
            s.v[q] += lane >= k ? x : 0;
        }
    if (lane == 63) wave_sums[wave] = s;
    __syncthreads();
#pragma unroll
    for (int q = 0; q < 4; q++) {
        s.v[q] -= own.v[q];
        total.v[q] = 0;
    }
#pragma unroll
    for (int w = 0; w < kSortWaves; w++)
#pragma unroll
        for (int q = 0; q < 4; q++) {
            const uint32_t x = wave_sums[w].v[q];
            s.v[q] += w < wave ? x : 0;
            total.v[q] += x;
        }
    return s;
}

// ONE: a single block, which ranks for itself.
template <typename ID, bool ONE>
__global__ __launch_bounds__(kSortThreads) void embedding_place_kernel(Order o) {
    if (static_cast<int>(blockIdx.x) >= o.blocks) return write_zeros(o, blockIdx.x - o.blocks);
    extern __shared__ uint16_t lds16[];
    __shared__ uint32_t start[kMaxBuckets];  // where this block's tokens of a bucket go
    __shared__ Four wave_sums[kSortWaves];
    const int64_t from = blockIdx.x * o.block_tokens, to = from + o.block_tokens;
    const int64_t end = to < o.tokens ? to : o.tokens;
    int id[kPer];
    uint32_t rank[kPer];
    const auto token = [&](int64_t at, int k) { return at + (threadIdx.x >> 6) * 64 * kPer + (threadIdx.x & 63) + 64 * k; };
    const auto fetch = [&](int64_t at) {
#pragma unroll
        for (int k = 0; k < kPer; k++) {
            id[k] = id_of<ID>(o, token(at, k), end);
            rank[k] = id[k] >= 0 ? o.rank[token(at, k)] : 0;
        }
    };
    uint32_t total[kOwn], before[kOwn];
    const int own = threadIdx.x * kOwn;
    const auto add = [&](uint32_t (&to8)[kOwn], const uint4 &c) {
        const uint32_t w[4] = {c.x, c.y, c.z, c.w};
#pragma unroll
        for (int k = 0; k < kOwn; k++) to8[k] += k & 1 ? w[k / 2] >> 16 : w[k / 2] & 0xFFFFu;
    };
#pragma unroll
    for (int k = 0; k < kOwn; k++) total[k] = before[k] = 0;
    if constexpr (ONE) {
        uint16_t *run = lds16, *wave_counts = lds16 + kMaxBuckets;
        for (int b = threadIdx.x; b < kMaxBuckets; b += kSortThreads) run[b] = 0;
        rank_batch<ID>(o, from, end, wave_counts, run, id, rank);
        add(total, *reinterpret_cast<const uint4 *>(run + own));
    } else {
        fetch(from);
        if (own < o.buckets) {
            const int self = blockIdx.x;
            const uint16_t *column = o.counts + own;
#pragma unroll 8
            for (int q = 0; q < self; q++) add(before, *reinterpret_cast<const uint4 *>(column + static_cast<int64_t>(q) * kMaxBuckets));
#pragma unroll 8
            for (int q = self; q < o.blocks; q++) add(total, *reinterpret_cast<const uint4 *>(column + static_cast<int64_t>(q) * kMaxBuckets));
#pragma unroll
            for (int k = 0; k < kOwn; k++) total[k] += before[k];
        }
    }
    // A thread packs its own neighbouring buckets into chunks of at most E entries; larger buckets are split.
    // Before its buckets: entries, chunks, chunks of split buckets, split buckets.
    const uint32_t E = o.entries;
    const auto chunks_of = [&](auto &&emit) {
        Four n{};
        uint32_t pack = 0;  // entries of the open chunk
        const auto close = [&]() {
            if (pack) {
                emit(n, pack, -1, 0u);
                n.v[1]++;
                n.v[0] += pack;
                pack = 0;
            }
        };
#pragma unroll
        for (int k = 0; k < kOwn; k++) {
            if (pack + total[k] > E) close();
            if (total[k] > E) {
                const uint32_t parts = (total[k] + E - 1) / E;
                emit(n, total[k], k, parts);
                n.v[0] += total[k];
                n.v[1] += parts;
                n.v[2] += parts;
                n.v[3]++;
            } else {
                pack += total[k];
            }
        }
        close();
        return n;
    };
    Four all;
    const Four prior = scan4(chunks_of([](const Four &, uint32_t, int, uint32_t) {}), wave_sums, all);
    uint32_t at = prior.v[0];
#pragma unroll
    for (int k = 0; k < kOwn; k++) {
        start[own + k] = at + before[k];
        at += total[k];
    }
    if (blockIdx.x == 0) {
        chunks_of([&](const Four &n, uint32_t entries, int k, uint32_t parts) {
            const uint32_t first = prior.v[0] + n.v[0], item = prior.v[1] + n.v[1], slot = prior.v[2] + n.v[2];
            if (parts == 0) {
                o.items[item] = make_uint4(first, entries, kNoSlot, 0);
            } else {
                o.multi[prior.v[3] + n.v[3]] = make_uint4(own + k, slot, parts, 0);
                for (uint32_t q = 0; q < parts; q++)
                    o.items[item + q] = make_uint4(first + q * E, min(E, entries - q * E), slot + q, 0);
            }
        });
        if (threadIdx.x == 0) {
            o.head[0] = all.v[1];
            o.head[1] = all.v[3];
        }
    }
    __syncthreads();
    for (int64_t batch = from; batch < end; batch += kBatch) {
        if (!ONE && batch > from) fetch(batch);
#pragma unroll
        for (int k = 0; k < kPer; k++)
            if (id[k] >= 0) {
                const uint32_t to_entry = start[id[k] >> o.shift] + rank[k];
                o.token[to_entry] = static_cast<uint32_t>(token(batch, k));
                o.id[to_entry] = static_cast<uint32_t>(id[k]);
            }
    }
}

// ------------------------------------------------------------------ sums

constexpr int kSumThreads = 256;

struct Sums {
    const void *dy;
    void *dtable;
    int64_t d;
    float scale;
    int shift;
    const uint32_t *token, *id;
    const uint4 *items, *multi;
    const uint32_t *head;
    uint32_t *present;  // [slots][8] ids of the bucket that a chunk has
    float *partial;     // [slots][W][stride]
    int64_t stride;
};

template <bool BF16, int LAYOUT, int L, int NV>
__global__ __launch_bounds__(kSumThreads) void embedding_sum_kernel(Sums a) {
    constexpr int N = Vec<BF16>::N, G = kSumThreads / L;
    constexpr int U = NV >= 3 ? 4 : 8;  // rows in flight
    using Cols = Columns<BF16, LAYOUT>;
    __shared__ __align__(16) uint32_t key[kMaxEntries];
    __shared__ uint32_t token[kMaxEntries], ids[kMaxEntries];
    __shared__ uint32_t present[8];
    __shared__ float carry[G][NV][N][L];  // a group's first run, where it began in a group before
    __shared__ int open[G];               // ... and it goes on behind the group
    if (blockIdx.x >= a.head[0]) return;
    const uint4 it = a.items[blockIdx.x];  // first entry, entries, slot
    const int len = it.y, tid = threadIdx.x, d = static_cast<int>(a.d);
    if (tid < 8) present[tid] = 0;
    {
        // place among the chunk's entries by (id, order); a chunk's ids lie within kOwn W <= 2^11 of each other
        uint32_t t = 0, id = 0, k = 0xFFFFFFFFu;
        if (tid < len) {
            t = a.token[it.x + tid];
            id = a.id[it.x + tid];
            k = (id & ((static_cast<uint32_t>(kOwn) << a.shift) - 1)) << 8 | tid;
        }
        key[tid] = k;
        __syncthreads();
        int at = 0;
        for (int i = 0; i < len; i += 4) {
            const uint4 other = *reinterpret_cast<const uint4 *>(&key[i]);
            at += (other.x < k) + (other.y < k) + (other.z < k) + (other.w < k);
        }
        if (tid < len) {
            token[at] = t;
            ids[at] = id;
            const uint32_t local = id & ((1u << a.shift) - 1);
            if (it.z != kNoSlot) atomicOr(&present[local >> 5], 1u << (local & 31));
        }
        __syncthreads();
        if (it.z != kNoSlot && blockIdx.y == 0 && tid < 8) a.present[static_cast<int64_t>(it.z) * 8 + tid] = present[tid];
    }
    const int lane = tid % L, group = tid / L;
    const int per = (len + G - 1) / G;
    const int p0 = min(group * per, len), p1 = min(p0 + per, len);
    const int index = blockIdx.y * (64 * NV);  // first vector of this block of columns (L = 64 where there are several)
    float acc[NV][N];
#pragma unroll
    for (int i = 0; i < NV; i++)
#pragma unroll
        for (int j = 0; j < N; j++) acc[i][j] = 0.f;
    const auto finish = [&](uint32_t id) {
#pragma unroll
        for (int i = 0; i < NV; i++) {
            const Cols col(index + i * L + lane, d);
            if (it.z == kNoSlot) {
                float f[N];
#pragma unroll
                for (int j = 0; j < N; j++) f[j] = acc[i][j] * a.scale;
                store_vec(a.dtable, static_cast<int64_t>(id) * d, col, d, true, pack<BF16>(f));
            } else if (col.in) {
                float *to = a.partial + ((static_cast<int64_t>(it.z) << a.shift) + (id & ((1u << a.shift) - 1))) * a.stride + col.c;
                if constexpr (LAYOUT == kTiny) {
                    for (int j = 0; j < d; j++) to[j] = acc[i][j];
                } else {
#pragma unroll
                    for (int j = 0; j < N; j += 4) {
                        float4_any v = {acc[i][j], acc[i][j + 1], acc[i][j + 2], acc[i][j + 3]};
                        *reinterpret_cast<float4_any *>(to + j) = v;
                    }
                }
            }
        }
    };
    const auto keep = [&]() {
#pragma unroll
        for (int i = 0; i < NV; i++)
#pragma unroll
            for (int j = 0; j < N; j++) carry[group][i][j][lane] = acc[i][j];
    };
    bool from_before = p0 < p1 && p0 > 0 && ids[p0 - 1] == ids[p0];
    uint32_t cur = p0 < p1 ? ids[p0] : 0;
    if (lane == 0) open[group] = 0;
    for (int p = p0; p < p1; p += U) {
        raw4 v[U][NV];
#pragma unroll
        for (int u = 0; u < U; u++) {
            const bool there = p + u < p1;
            const int64_t row = there ? static_cast<int64_t>(token[p + u]) * d : 0;
#pragma unroll
            for (int i = 0; i < NV; i++) v[u][i] = load_vec(a.dy, row, Cols(index + i * L + lane, d), d, there);
        }
#pragma unroll
        for (int u = 0; u < U; u++) {
            if (p + u < p1) {
                if (ids[p + u] != cur) {
                    if (from_before)
                        keep();
                    else
                        finish(cur);
                    from_before = false;
                    cur = ids[p + u];
#pragma unroll
                    for (int i = 0; i < NV; i++)
#pragma unroll
                        for (int j = 0; j < N; j++) acc[i][j] = 0.f;
                }
#pragma unroll
                for (int i = 0; i < NV; i++)
#pragma unroll
                    for (int j = 0; j < N; j++) acc[i][j] += value<BF16>(v[u][i], j);
            }
        }
    }
    const bool goes_on = p0 < p1 && p1 < len && ids[p1] == cur;
    if (p0 < p1) {
        if (from_before) {
            keep();
            if (lane == 0) open[group] = goes_on;
        } else if (!goes_on) {
            finish(cur);
        }
    }
    __syncthreads();
    if (p0 < p1 && !from_before && goes_on) {
        for (int g = group + 1; g < G; g++) {
#pragma unroll
            for (int i = 0; i < NV; i++)
#pragma unroll
                for (int j = 0; j < N; j++) acc[i][j] += carry[g][i][j][lane];
            if (!open[g]) break;
        }
        finish(cur);
    }
}

// The rows of buckets of several chunks: 16 waves of 64 lanes, four columns a lane, each wave a share of the chunks.
constexpr int kJoinThreads = 1024, kJoinWaves = kJoinThreads / 64;

template <bool BF16>
__global__ __launch_bounds__(kJoinThreads) void embedding_join_kernel(Sums a) {
    __shared__ float4 sums[kJoinWaves][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int column_blocks = static_cast<int>((a.d + 255) / 256);
    const int64_t items = (static_cast<int64_t>(a.head[1]) << a.shift) * column_blocks;
    for (int64_t i = blockIdx.x; i < items; i += gridDim.x) {
        const int c = static_cast<int>(i % column_blocks) * 256 + lane * 4;
        const int64_t q = i / column_blocks;
        const uint32_t id = static_cast<uint32_t>(q) & ((1u << a.shift) - 1);
        const uint4 m = a.multi[q >> a.shift];  // bucket, first slot, chunks
        const int chunks = m.z, per = (chunks + kJoinWaves - 1) / kJoinWaves;
        const int from = wave * per, to = min(from + per, chunks);
        float s[4] = {0.f, 0.f, 0.f, 0.f};
        uint32_t any = 0;
#pragma unroll 4
        for (int k = from; k < to; k++) {
            const int64_t slot = m.y + k;
            if (a.present[slot * 8 + (id >> 5)] >> (id & 31) & 1) {
                any = 1;
                if (c < a.d) {
                    const float4 v = *reinterpret_cast<const float4 *>(a.partial + ((slot << a.shift) + id) * a.stride + c);
                    s[0] += v.x; s[1] += v.y; s[2] += v.z; s[3] += v.w;
                }
            }
        }
        sums[wave][lane] = make_float4(s[0], s[1], s[2], s[3]);
        const bool occurs = __syncthreads_or(any);
        if (occurs && wave == 0 && c < a.d) {
            float t[4] = {0.f, 0.f, 0.f, 0.f};
            for (int w = 0; w < kJoinWaves; w++) {
                const float4 v = sums[w][lane];
                t[0] += v.x; t[1] += v.y; t[2] += v.z; t[3] += v.w;
            }
            const int64_t row = ((static_cast<int64_t>(m.x) << a.shift) + id) * a.d;
            for (int j = 0; j < 4 && c + j < a.d; j++) {
                if constexpr (BF16)
                    static_cast<__bf16 *>(a.dtable)[row + c + j] = static_cast<__bf16>(t[j] * a.scale);
                else
                    static_cast<float *>(a.dtable)[row + c + j] = t[j] * a.scale;
            }
        }
        __syncthreads();
    }
}

// ------------------------------------------------------------------ positions

// dpos[p], or of `parts` > 1 a part's fp32 sums [part][n][d]: a group of lanes takes one position and
// the sequences of one part.
template <bool BF16, int LAYOUT, int L, int NV>
__global__ __launch_bounds__(kSumThreads) void embedding_pos_kernel(const void *dy, int64_t n, int64_t batch, int64_t dd,
                                                                    void *dpos, float *partial) {
    constexpr int N = Vec<BF16>::N, G = kSumThreads / L, U = NV >= 3 ? 4 : 8;
    using Cols = Columns<BF16, LAYOUT>;
    const int lane = threadIdx.x % L, d = static_cast<int>(dd), index = blockIdx.y * (64 * NV);
    const int64_t parts = gridDim.z, part = blockIdx.z, per = (batch + parts - 1) / parts;
    const int64_t b0 = part * per, b1 = b0 + per < batch ? b0 + per : batch;
    const int64_t p = static_cast<int64_t>(blockIdx.x) * G + threadIdx.x / L;
    if (p >= n) return;
    float acc[NV][N];
#pragma unroll
    for (int i = 0; i < NV; i++)
#pragma unroll
        for (int j = 0; j < N; j++) acc[i][j] = 0.f;
    for (int64_t b = b0; b < b1; b += U) {
        raw4 v[U][NV];
#pragma unroll
        for (int u = 0; u < U; u++)
#pragma unroll
            for (int i = 0; i < NV; i++)
                v[u][i] = load_vec(dy, b + u < b1 ? ((b + u) * n + p) * d : 0, Cols(index + i * L + lane, d), d, b + u < b1);
#pragma unroll
        for (int u = 0; u < U; u++)
#pragma unroll
            for (int i = 0; i < NV; i++)
#pragma unroll
                for (int j = 0; j < N; j++) acc[i][j] += value<BF16>(v[u][i], j);
    }
#pragma unroll
    for (int i = 0; i < NV; i++) {
        const Cols col(index + i * L + lane, d);
        if (parts == 1) {
            store_vec(dpos, p * d, col, d, true, pack<BF16>(acc[i]));
        } else if (col.in) {
            float *to = partial + (part * n + p) * d + col.c;
#pragma unroll
            for (int j = 0; j < N; j++)
                if (LAYOUT != kTiny || j < d) to[j] = acc[i][j];
        }
    }
}

template <bool BF16>
__global__ __launch_bounds__(kSumThreads) void embedding_pos_join_kernel(const float *partial, int64_t values, int parts, void *dpos) {
    for (int64_t e = static_cast<int64_t>(blockIdx.x) * kSumThreads + threadIdx.x; e < values; e += static_cast<int64_t>(gridDim.x) * kSumThreads) {
        float s = 0.f;
#pragma unroll 8
        for (int q = 0; q < parts; q++) s += partial[q * values + e];
        if constexpr (BF16)
            static_cast<__bf16 *>(dpos)[e] = static_cast<__bf16>(s);
        else
            static_cast<float *>(dpos)[e] = s;
    }
}

// ------------------------------------------------------------------ host

int64_t up(int64_t a, int64_t b) { return (a + b - 1) / b; }

int shift_of(int64_t vocab) {
    int s = 0;
    while (((vocab - 1) >> s) + 1 > kMaxBuckets) s++;
    return s;
}

// Parts of the positions' sums: few positions of many sequences are split until about 512 groups of lanes work.
int64_t pos_parts(int64_t n, int64_t batch) {
    if (n == 0 || n >= 512 || batch <= 16) return 1;
    const int64_t want = up(512, n), most = batch / 8;
    return want < most ? want : most;
}

struct Layout {
    size_t counts, rank, token, id, items, multi, head, present, partial, pos, total;
    int64_t blocks, block_tokens, max_items, max_multi, stride;
    int shift, entries;
};

Layout layout_of(int64_t tokens, int64_t n, int64_t vocab, int d) {
    Layout l{};
    l.shift = shift_of(vocab);
    // 64 blocks of tokens, less where there are few; more where a block's tokens would pass the 16-bit ranks
    l.blocks = up(tokens, kBatch);
    const int64_t most = up(tokens, 65535);
    if (l.blocks > 64) l.blocks = most > 64 ? most : 64;
    l.block_tokens = l.blocks ? up(tokens, l.blocks) : 0;
    // entries of a chunk: fewer where there are few tokens, for several workgroups to a CU
    l.entries = 32;
    while (l.entries < kMaxEntries && tokens >= 1024 * static_cast<int64_t>(l.entries)) l.entries *= 2;
    // A chunk and the next one of the same thread hold more than E entries, but for the last part of a split bucket
    // (there are fewer than tokens / E such): at most 4 tokens / E chunks and one more a thread.
    const int64_t chunks = 4 * (tokens / l.entries) + kSortThreads + 4;
    l.max_items = tokens < chunks ? tokens : chunks;
    l.max_multi = tokens / (l.entries + 1);
    l.stride = up(d, 8) * 8;
    const int64_t slots = l.max_multi ? 2 * (tokens / l.entries) : 0;
    size_t at = 0;
    const auto place = [&](size_t &off, size_t bytes) {
        off = at;
        at += (bytes + 255) / 256 * 256;
    };
    place(l.counts, l.blocks > 1 ? static_cast<size_t>(l.blocks) * kMaxBuckets * 2 : 0);
    place(l.rank, l.blocks > 1 ? static_cast<size_t>(tokens) * 2 : 0);
    place(l.token, static_cast<size_t>(tokens) * 4);
    place(l.id, static_cast<size_t>(tokens) * 4);
    place(l.items, static_cast<size_t>(l.max_items) * 16);
    place(l.multi, static_cast<size_t>(l.max_multi) * 16);
    place(l.head, tokens ? 16 : 0);
    place(l.present, static_cast<size_t>(slots) * 32);
    place(l.partial, (static_cast<size_t>(slots) << l.shift) * l.stride * 4);
    const int64_t parts = pos_parts(n, n ? tokens / n : 0);
    place(l.pos, parts > 1 ? static_cast<size_t>(parts) * n * d * 4 : 0);
    l.total = at;
    return l;
}

// Lanes and vectors for a row, or a block of its columns where a wave of four (16 bits: two) vectors a lane does
// not take it.
struct Form {
    int lanes, vectors, blocks;
};

Form form_of(bool bf16, int d) {
    const int n = bf16 ? 8 : 4, nvec = (d + n - 1) / n, most = bf16 ? 2 : 4;
    int lanes = 4;
    while (lanes < 64 && nvec > 2 * lanes) lanes *= 2;
    const int blocks = static_cast<int>(up(nvec, 64 * most));
    return {lanes, static_cast<int>(up(nvec, static_cast<int64_t>(lanes) * blocks)), blocks};
}

template <bool BF16, int LAYOUT, typename F>
void with_form(int d, F f) {
    const Form form = form_of(BF16, d);
#define YOSO_ROW_FORM(L_, NV_) \
    if (form.lanes == L_ && form.vectors == NV_) return f.template operator()<BF16, LAYOUT, L_, NV_>(form.blocks);
    YOSO_ROW_FORM(4, 1)
    if constexpr (LAYOUT != kTiny) {
        YOSO_ROW_FORM(4, 2) YOSO_ROW_FORM(8, 2) YOSO_ROW_FORM(16, 2) YOSO_ROW_FORM(32, 2) YOSO_ROW_FORM(64, 2)
        if constexpr (!BF16) {
            YOSO_ROW_FORM(64, 3) YOSO_ROW_FORM(64, 4)
        }
    }
#undef YOSO_ROW_FORM
}

template <bool BF16, typename F>
void with_layout(int d, F f) {
    constexpr int N = Vec<BF16>::N;
    if (d % N == 0)
        with_form<BF16, kAligned>(d, f);
    else if (d > N)
        with_form<BF16, kOverlap>(d, f);
    else
        with_form<BF16, kTiny>(d, f);
}

struct Sum {
    const Sums &a;
    int64_t items;
    hipStream_t stream;
    template <bool BF16, int LAYOUT, int L, int NV>
    void operator()(int blocks) const {
        hipLaunchKernelGGL((embedding_sum_kernel<BF16, LAYOUT, L, NV>), dim3(static_cast<unsigned>(items), blocks),
                           dim3(kSumThreads), 0, stream, a);
    }
};

struct Pos {
    const EmbeddingBackward &a;
    int64_t parts;
    float *partial;
    hipStream_t stream;
    template <bool BF16, int LAYOUT, int L, int NV>
    void operator()(int blocks) const {
        hipLaunchKernelGGL((embedding_pos_kernel<BF16, LAYOUT, L, NV>),
                           dim3(static_cast<unsigned>(up(a.n, kSumThreads / L)), blocks, static_cast<unsigned>(parts)),
                           dim3(kSumThreads), 0, stream, a.dy, a.n, a.tokens / a.n, static_cast<int64_t>(a.d), a.dpos, partial);
    }
};

template <bool BF16, int LAYOUT, typename ID>
void lookup(const Embedding &a, hipStream_t stream) {
    constexpr int N = Vec<BF16>::N;
    const int64_t nvec = up(a.d, N);
#define YOSO_LOOKUP(L_)                                                                                          \
    {                                                                                                            \
        const int64_t need = up(a.tokens, kLookThreads / L_);                                                    \
        hipLaunchKernelGGL((embedding_kernel<BF16, LAYOUT, L_, ID>), dim3(static_cast<unsigned>(need < 16384 ? need : 16384)), \
                           dim3(kLookThreads), 0, stream, a);                                                    \
    }
    if (nvec <= 8) YOSO_LOOKUP(4)
    else if (nvec <= 64) YOSO_LOOKUP(16)
    else if (nvec <= 256) YOSO_LOOKUP(64)
    else YOSO_LOOKUP(256)
#undef YOSO_LOOKUP
}

template <bool BF16, typename ID>
void lookup(const Embedding &a, hipStream_t stream) {
    constexpr int N = Vec<BF16>::N;
    if (a.d % N == 0)
        lookup<BF16, kAligned, ID>(a, stream);
    else if (a.d > N)
        lookup<BF16, kOverlap, ID>(a, stream);
    else
        lookup<BF16, kTiny, ID>(a, stream);
}

}  // namespace

size_t embedding_backward_workspace(int64_t tokens, int64_t n, int64_t vocab, int d) {
    return layout_of(tokens, n, vocab, d).total;
}

hipError_t launch_embedding(const Embedding &a, bool bf16, bool wide, hipStream_t stream) {
    if (a.tokens == 0) return hipSuccess;
    KernelTimer timer("embedding_kernel", stream);
    if (wide)
        bf16 ? lookup<true, int64_t>(a, stream) : lookup<false, int64_t>(a, stream);
    else
        bf16 ? lookup<true, int32_t>(a, stream) : lookup<false, int32_t>(a, stream);
    return hipGetLastError();
}

hipError_t launch_embedding_backward(const EmbeddingBackward &a, bool bf16, bool wide, hipStream_t stream) {
    const Layout l = layout_of(a.tokens, a.n, a.vocab, a.d);
    char *ws = static_cast<char *>(a.workspace);
    Order o{};
    o.ids = a.ids;
    o.tokens = a.tokens;
    o.vocab = a.vocab;
    o.shift = l.shift;
    o.buckets = static_cast<int>(((a.vocab - 1) >> l.shift) + 1);
    o.blocks = static_cast<int>(l.blocks);
    o.block_tokens = l.block_tokens;
    o.entries = l.entries;
    o.counts = reinterpret_cast<uint16_t *>(ws + l.counts);
    o.rank = reinterpret_cast<uint16_t *>(ws + l.rank);
    o.token = reinterpret_cast<uint32_t *>(ws + l.token);
    o.id = reinterpret_cast<uint32_t *>(ws + l.id);
    o.items = reinterpret_cast<uint4 *>(ws + l.items);
    o.multi = reinterpret_cast<uint4 *>(ws + l.multi);
    o.head = reinterpret_cast<uint32_t *>(ws + l.head);
    hipError_t e = hipSuccess;
    // zeros of dtable: in one launch or half in each of the two
    const int64_t block_vectors = int64_t{kSortThreads} * kZeroPerThread;
    o.zero = static_cast<uint4 *>(a.dtable);
    o.zero_bytes = a.vocab * a.d * (bf16 ? 2 : 4);
    const int64_t vectors = up(o.zero_bytes, 16), half = up(vectors, 2 * block_vectors) * block_vectors;
    const int64_t cut = l.blocks > 1 && half < vectors ? half : 0;
    if (l.blocks != 1) {
        KernelTimer timer("embedding_rank_kernel", stream);
        o.zero_from = 0;
        o.zero_to = l.blocks ? cut : vectors;
        const unsigned grid = static_cast<unsigned>(l.blocks + up(o.zero_to - o.zero_from, block_vectors));
        if (wide)
            hipLaunchKernelGGL(embedding_rank_kernel<int64_t>, dim3(grid), dim3(kSortThreads), kRankLds, stream, o);
        else
            hipLaunchKernelGGL(embedding_rank_kernel<int32_t>, dim3(grid), dim3(kSortThreads), kRankLds, stream, o);
        if ((e = hipGetLastError()) != hipSuccess) return e;
    }
    if (l.blocks) {
        KernelTimer timer("embedding_place_kernel", stream);
        o.zero_from = cut;
        o.zero_to = vectors;
        const unsigned grid = static_cast<unsigned>(l.blocks + up(o.zero_to - o.zero_from, block_vectors));
        const size_t lds = l.blocks == 1 ? kRankLds : 0;
        auto *f = wide ? (l.blocks == 1 ? embedding_place_kernel<int64_t, true> : embedding_place_kernel<int64_t, false>)
                       : (l.blocks == 1 ? embedding_place_kernel<int32_t, true> : embedding_place_kernel<int32_t, false>);
        hipLaunchKernelGGL(f, dim3(grid), dim3(kSortThreads), lds, stream, o);
        if ((e = hipGetLastError()) != hipSuccess) return e;

        const Sums s{a.dy, a.dtable, a.d, a.scale, l.shift, o.token, o.id, o.items, o.multi, o.head,
                     reinterpret_cast<uint32_t *>(ws + l.present), reinterpret_cast<float *>(ws + l.partial), l.stride};
        {
            KernelTimer sum_timer("embedding_sum_kernel", stream);
            const Sum run{s, l.max_items, stream};
            bf16 ? with_layout<true>(a.d, run) : with_layout<false>(a.d, run);
            if ((e = hipGetLastError()) != hipSuccess) return e;
        }
        if (l.max_multi) {
            KernelTimer join_timer("embedding_join_kernel", stream);
            const int64_t items = (l.max_multi << l.shift) * up(a.d, 256);
            auto *j = bf16 ? embedding_join_kernel<true> : embedding_join_kernel<false>;
            hipLaunchKernelGGL(j, dim3(static_cast<unsigned>(items < 512 ? items : 512)), dim3(kJoinThreads), 0, stream, s);
            if ((e = hipGetLastError()) != hipSuccess) return e;
        }
    }
    if (a.n == 0) return e;
    if (a.tokens == 0) {
        KernelTimer timer("embedding_pos_kernel", stream);
        Order z{};
        z.zero = static_cast<uint4 *>(a.dpos);
        z.zero_bytes = a.n * a.d * (bf16 ? 2 : 4);
        z.zero_to = up(z.zero_bytes, 16);
        hipLaunchKernelGGL(embedding_rank_kernel<int32_t>, dim3(static_cast<unsigned>(up(z.zero_to, block_vectors))), dim3(kSortThreads), 0, stream, z);
        return hipGetLastError();
    }
    const int64_t parts = pos_parts(a.n, a.tokens / a.n);
    float *partial = reinterpret_cast<float *>(ws + l.pos);
    {
        KernelTimer timer("embedding_pos_kernel", stream);
        const Pos run{a, parts, partial, stream};
        bf16 ? with_layout<true>(a.d, run) : with_layout<false>(a.d, run);
        if ((e = hipGetLastError()) != hipSuccess || parts == 1) return e;
    }
    KernelTimer timer("embedding_pos_join_kernel", stream);
    const int64_t values = a.n * a.d, blocks = up(values, kSumThreads);
    auto *j = bf16 ? embedding_pos_join_kernel<true> : embedding_pos_join_kernel<false>;
    hipLaunchKernelGGL(j, dim3(static_cast<unsigned>(blocks < 4096 ? blocks : 4096)), dim3(kSumThreads), 0, stream,
                       static_cast<const float *>(partial), values, static_cast<int>(parts), a.dpos);
    return hipGetLastError();
}

}  // namespace yoso
