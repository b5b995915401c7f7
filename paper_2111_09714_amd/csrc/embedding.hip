// Embedding lookup with positions, and its gradient by sorted tokens (gfx950).
//
//   y[t] = scale table[ids[t]] + pos[t mod n];  ids outside [0, vocab) have no row (0)
//   dtable[v] = scale sum_{t : ids[t] = v} dy[t],   dpos[p] = sum_b dy[b n + p]
//
// The lookup is a gather of rows, L lanes to a row.  The gradient never adds to memory: tokens are
// put in the order of their ids and every row of dtable is one sum in the order of its tokens,
// the same bits every time.
//
//   count  per block of tokens, how many fall into each bucket of W = 2^s neighbouring ids (at most
//          4096 buckets); place  tokens to their bucket, stable: the block's start in a bucket from all
//          blocks' counts, a token's place from ballots over its wave.  Both are short and use few
//          CUs; the rest of the card writes dtable's zeros meanwhile (half in each launch), which
//          the rows that occur overwrite.
//   sum    one workgroup per kChunk tokens of one bucket: orders them by id in LDS, then groups of lanes
//          add their shares of that order, runs that cross groups through LDS.  A bucket of one chunk
//          ends in dtable; of more chunks (frequent ids), each leaves fp32 rows of its ids,
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
constexpr int kBlockTokens = 2048;  // tokens of a block, while 64 blocks do
constexpr int kChunk = 256;
constexpr uint32_t kNoSlot = 0xFFFFFFFFu;

struct Order {
    const void *ids;
    int64_t tokens, vocab;
    int shift, buckets, blocks;
    int64_t block_tokens;
    uint32_t *counts;  // [blocks][kMaxBuckets]
    uint32_t *token;   // [tokens] in bucket order
    uint8_t *local;    // their ids within the bucket
    uint4 *items;      // chunks: first entry, entries, bucket, slot of partial rows
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

// bucket of token t, or -1 where it has no row
template <typename ID>
__device__ __forceinline__ int bucket_of(const Order &o, int64_t t, int64_t end, uint32_t &local) {
    if (t >= end) return -1;
    const int64_t id = static_cast<const ID *>(o.ids)[t];
    if (id < 0 || id >= o.vocab) return -1;
    local = static_cast<uint32_t>(id) & ((1u << o.shift) - 1);
    return static_cast<int>(static_cast<uint32_t>(id) >> o.shift);
}

template <typename ID>
__global__ __launch_bounds__(kSortThreads) void embedding_count_kernel(Order o) {
    if (static_cast<int>(blockIdx.x) >= o.blocks) return write_zeros(o, blockIdx.x - o.blocks);
    __shared__ uint32_t count[kMaxBuckets];
    for (int b = threadIdx.x; b < kMaxBuckets; b += kSortThreads) count[b] = 0;
    __syncthreads();
    const int64_t from = blockIdx.x * o.block_tokens, to = from + o.block_tokens;
    const int64_t end = to < o.tokens ? to : o.tokens;
    for (int64_t t = from + threadIdx.x; t < end; t += kSortThreads) {
        uint32_t local;
        const int b = bucket_of<ID>(o, t, end, local);
        if (b >= 0) atomicAdd(&count[b], 1u);
    }
    __syncthreads();
    uint32_t *out = o.counts + static_cast<int64_t>(blockIdx.x) * kMaxBuckets;
    for (int b = threadIdx.x; b < kMaxBuckets; b += kSortThreads) out[b] = count[b];
}

// exclusive sums over the workgroup's threads of two values each
__device__ __forceinline__ uint2 scan2(uint2 v, uint2 *wave_sums, uint2 &total) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    uint2 s = v;
#pragma unroll
    for (int k = 1; k < 64; k *= 2) {
        const uint32_t x = __shfl_up(s.x, k), y = __shfl_up(s.y, k);
        if (lane >= k) {
            s.x += x;
            s.y += y;
        }
    }
    __syncthreads();
    if (lane == 63) wave_sums[wave] = s;
    __syncthreads();
    uint2 before = make_uint2(s.x - v.x, s.y - v.y);
    total = make_uint2(0, 0);
#pragma unroll
    for (int w = 0; w < kSortWaves; w++) {
        const uint2 t = wave_sums[w];
        if (w < wave) {
            before.x += t.x;
            before.y += t.y;
        }
        total.x += t.x;
        total.y += t.y;
    }
    return before;
}

// ONE: a single block, which counts for itself.
template <typename ID, bool ONE>
__global__ __launch_bounds__(kSortThreads) void embedding_place_kernel(Order o) {
    if (static_cast<int>(blockIdx.x) >= o.blocks) return write_zeros(o, blockIdx.x - o.blocks);
    extern __shared__ uint32_t lds[];
    uint32_t *start = lds;                       // [kMaxBuckets] where this block's tokens of a bucket go
    uint32_t *first = lds + kMaxBuckets;         // (until the ranks) first entry, entries, first item, first slot
    uint32_t *size = first + kMaxBuckets;
    uint32_t *item = size + kMaxBuckets;
    uint32_t *slot = item + kMaxBuckets;
    uint16_t *rank = reinterpret_cast<uint16_t *>(first);  // [kSortWaves][kMaxBuckets], the same 64 KiB
    __shared__ uint2 wave_sums[kSortWaves];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t from = blockIdx.x * o.block_tokens, to = from + o.block_tokens;
    const int64_t end = to < o.tokens ? to : o.tokens;

    uint32_t total[kOwn], before[kOwn];
    const int own = threadIdx.x * kOwn;
    if constexpr (ONE) {
        for (int b = threadIdx.x; b < kMaxBuckets; b += kSortThreads) size[b] = 0;
        __syncthreads();
        for (int64_t t = from + threadIdx.x; t < end; t += kSortThreads) {
            uint32_t local;
            const int b = bucket_of<ID>(o, t, end, local);
            if (b >= 0) atomicAdd(&size[b], 1u);
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < kOwn; k++) {
            total[k] = size[own + k];
            before[k] = 0;
        }
    } else {
#pragma unroll
        for (int k = 0; k < kOwn; k++) total[k] = before[k] = 0;
#pragma unroll 4
        for (int q = 0; q < o.blocks; q++) {
            const uint4 *row = reinterpret_cast<const uint4 *>(o.counts + static_cast<int64_t>(q) * kMaxBuckets + own);
            const uint4 x = row[0], y = row[1];
            const uint32_t c[kOwn] = {x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
#pragma unroll
            for (int k = 0; k < kOwn; k++) {
                total[k] += c[k];
                before[k] += q < static_cast<int>(blockIdx.x) ? c[k] : 0;
            }
        }
    }
    // entries and chunks before each bucket; slots (chunks of buckets that have several) and such buckets
    uint2 mine = make_uint2(0, 0), several = make_uint2(0, 0), all, all_several;
#pragma unroll
    for (int k = 0; k < kOwn; k++) {
        const uint32_t chunks = (total[k] + kChunk - 1) / kChunk;
        mine.x += total[k];
        mine.y += chunks;
        several.x += chunks > 1 ? chunks : 0;
        several.y += chunks > 1;
    }
    mine = scan2(mine, wave_sums, all);
    several = scan2(several, wave_sums, all_several);
#pragma unroll
    for (int k = 0; k < kOwn; k++) {
        const uint32_t chunks = (total[k] + kChunk - 1) / kChunk;
        start[own + k] = mine.x + before[k];
        first[own + k] = mine.x;
        size[own + k] = total[k];
        item[own + k] = mine.y;
        slot[own + k] = chunks > 1 ? several.x : kNoSlot;
        if (chunks > 1 && blockIdx.x == 0) o.multi[several.y] = make_uint4(own + k, several.x, chunks, 0);
        mine.x += total[k];
        mine.y += chunks;
        several.x += chunks > 1 ? chunks : 0;
        several.y += chunks > 1;
    }
    if (blockIdx.x == 0 && threadIdx.x == 0) {
        o.head[0] = all.y;
        o.head[1] = all_several.y;
    }
    __syncthreads();
    // the blocks share the list of chunks: chunk i lies in the last bucket whose first item is at most i (buckets
    // without tokens have none, and the same first item as the next)
    for (uint32_t i = blockIdx.x * kSortThreads + threadIdx.x; i < all.y; i += o.blocks * kSortThreads) {
        int lo = 0, hi = kMaxBuckets - 1;
        while (lo < hi) {
            const int mid = (lo + hi + 1) / 2;
            if (item[mid] <= i)
                lo = mid;
            else
                hi = mid - 1;
        }
        const uint32_t part = i - item[lo], at = part * kChunk, left = size[lo] - at;
        o.items[i] = make_uint4(first[lo] + at, left < kChunk ? left : kChunk, lo, slot[lo] == kNoSlot ? kNoSlot : slot[lo] + part);
    }
    __syncthreads();

    // ranks: each wave takes a stretch of the block's tokens, counts its buckets, and, once the counts of the waves before
    // it are known, places its tokens
    for (int b = threadIdx.x; b < kSortWaves * kMaxBuckets / 2; b += kSortThreads) reinterpret_cast<uint32_t *>(rank)[b] = 0;
    __syncthreads();
    const int64_t stretch = (o.block_tokens + 64 * kSortWaves - 1) / (64 * kSortWaves) * 64;
    const int64_t wave_from = from + wave * stretch, wave_to = wave_from + stretch;
    const int64_t wave_end = wave_to < end ? wave_to : end;
    uint16_t *counter = rank + wave * kMaxBuckets;
    const int bits = 32 - __clz(o.buckets);
    const auto same_bucket = [&](int b) {
        unsigned long long same = __ballot(b >= 0);
        for (int i = 0; i < bits; i++) {
            const unsigned long long m = __ballot((b >> i) & 1);
            same &= (b >> i) & 1 ? m : ~m;
        }
        return same;
    };
    for (int64_t t = wave_from; t < wave_end; t += 64) {
        uint32_t local;
        const int b = bucket_of<ID>(o, t + lane, wave_end, local);
        const unsigned long long same = same_bucket(b);
        if (b >= 0 && lane == __ffsll(same) - 1) counter[b] += __popcll(same);
    }
    __syncthreads();
    for (int b = threadIdx.x; b < kMaxBuckets; b += kSortThreads) {
        uint32_t sum = 0;
#pragma unroll
        for (int w = 0; w < kSortWaves; w++) {
            const uint32_t c = rank[w * kMaxBuckets + b];
            rank[w * kMaxBuckets + b] = static_cast<uint16_t>(sum);
            sum += c;
        }
    }
    __syncthreads();
    for (int64_t t = wave_from; t < wave_end; t += 64) {
        uint32_t local = 0;
        const int b = bucket_of<ID>(o, t + lane, wave_end, local);
        const unsigned long long same = same_bucket(b);
        if (b >= 0) {
            const uint32_t at = start[b] + counter[b] + __popcll(same & ((1ull << lane) - 1));
            o.token[at] = static_cast<uint32_t>(t + lane);
            o.local[at] = static_cast<uint8_t>(local);
            if (lane == 63 - __clzll(same)) counter[b] = static_cast<uint16_t>(counter[b] + __popcll(same));
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
    const uint32_t *token;
    const uint8_t *local;
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
    __shared__ uint32_t key[kChunk], token[kChunk];
    __shared__ uint32_t local[kChunk + 1];
    __shared__ uint32_t present[8];
    __shared__ float carry[G][NV][N][L];  // a group's first run, where it began in a group before
    __shared__ int open[G];               // ... and it goes on behind the group
    if (blockIdx.x >= a.head[0]) return;
    const uint4 it = a.items[blockIdx.x];
    const int len = it.y, tid = threadIdx.x, d = static_cast<int>(a.d);
    if (tid < 8) present[tid] = 0;
    {
        uint32_t t = 0, l = 0;
        if (tid < len) {
            t = a.token[it.x + tid];
            l = a.local[it.x + tid];
            key[tid] = l << 8 | tid;
        }
        __syncthreads();
        if (tid < len) {
            int at = tid;
            if (a.shift) {  // place among the chunk's entries by (id, order)
                const uint32_t k = l << 8 | tid;
                at = 0;
                for (int i = 0; i < len; i++) at += key[i] < k;
            }
            token[at] = t;
            local[at] = l;
            if (it.w != kNoSlot) atomicOr(&present[l >> 5], 1u << (l & 31));
        }
        __syncthreads();
        if (it.w != kNoSlot && blockIdx.y == 0 && tid < 8) a.present[static_cast<int64_t>(it.w) * 8 + tid] = present[tid];
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
            if (it.w == kNoSlot) {
                float f[N];
#pragma unroll
                for (int j = 0; j < N; j++) f[j] = acc[i][j] * a.scale;
                store_vec(a.dtable, ((static_cast<int64_t>(it.z) << a.shift) + id) * d, col, d, true, pack<BF16>(f));
            } else if (col.in) {
                float *to = a.partial + ((static_cast<int64_t>(it.w) << a.shift) + id) * a.stride + col.c;
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
    bool from_before = p0 < p1 && p0 > 0 && local[p0 - 1] == local[p0];
    uint32_t cur = p0 < p1 ? local[p0] : 0;
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
                if (local[p + u] != cur) {
                    if (from_before)
                        keep();
                    else
                        finish(cur);
                    from_before = false;
                    cur = local[p + u];
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
    const bool goes_on = p0 < p1 && p1 < len && local[p1] == cur;
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
    size_t counts, token, local, items, multi, head, present, partial, pos, total;
    int64_t blocks, block_tokens, max_items, max_multi, stride;
    int shift;
};

Layout layout_of(int64_t tokens, int64_t n, int64_t vocab, int d) {
    Layout l{};
    l.shift = shift_of(vocab);
    // 64 blocks of tokens, less where there are few; more where a block's tokens would pass the waves' 16-bit counters
    l.blocks = up(tokens, kBlockTokens);
    const int64_t most = up(tokens, 65535);
    if (l.blocks > 64) l.blocks = most > 64 ? most : 64;
    l.block_tokens = l.blocks ? up(tokens, l.blocks) : 0;
    const int64_t buckets = ((vocab - 1) >> l.shift) + 1;
    l.max_items = (tokens < buckets ? tokens : buckets) + tokens / kChunk;
    l.max_multi = tokens / (kChunk + 1) < buckets ? tokens / (kChunk + 1) : buckets;
    l.stride = up(d, 8) * 8;
    const int64_t slots = tokens > kChunk ? 2 * (tokens / kChunk) : 0;
    size_t at = 0;
    const auto place = [&](size_t &off, size_t bytes) {
        off = at;
        at += (bytes + 255) / 256 * 256;
    };
    place(l.counts, l.blocks > 1 ? static_cast<size_t>(l.blocks) * kMaxBuckets * 4 : 0);
    place(l.token, static_cast<size_t>(tokens) * 4);
    place(l.local, static_cast<size_t>(tokens));
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
    o.counts = reinterpret_cast<uint32_t *>(ws + l.counts);
    o.token = reinterpret_cast<uint32_t *>(ws + l.token);
    o.local = reinterpret_cast<uint8_t *>(ws + l.local);
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
        KernelTimer timer("embedding_count_kernel", stream);
        o.zero_from = 0;
        o.zero_to = l.blocks ? cut : vectors;
        const unsigned grid = static_cast<unsigned>(l.blocks + up(o.zero_to - o.zero_from, block_vectors));
        if (wide)
            hipLaunchKernelGGL(embedding_count_kernel<int64_t>, dim3(grid), dim3(kSortThreads), 0, stream, o);
        else
            hipLaunchKernelGGL(embedding_count_kernel<int32_t>, dim3(grid), dim3(kSortThreads), 0, stream, o);
        if ((e = hipGetLastError()) != hipSuccess) return e;
    }
    if (l.blocks) {
        KernelTimer timer("embedding_place_kernel", stream);
        o.zero_from = cut;
        o.zero_to = vectors;
        const unsigned grid = static_cast<unsigned>(l.blocks + up(o.zero_to - o.zero_from, block_vectors));
        const size_t lds = 5 * kMaxBuckets * sizeof(uint32_t);
        auto *f = wide ? (l.blocks == 1 ? embedding_place_kernel<int64_t, true> : embedding_place_kernel<int64_t, false>)
                       : (l.blocks == 1 ? embedding_place_kernel<int32_t, true> : embedding_place_kernel<int32_t, false>);
        hipLaunchKernelGGL(f, dim3(grid), dim3(kSortThreads), lds, stream, o);
        if ((e = hipGetLastError()) != hipSuccess) return e;

        const Sums s{a.dy, a.dtable, a.d, a.scale, l.shift, o.token, o.local, o.items, o.multi, o.head,
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
        hipLaunchKernelGGL(embedding_count_kernel<int32_t>, dim3(static_cast<unsigned>(up(z.zero_to, block_vectors))), dim3(kSortThreads), 0, stream, z);
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
