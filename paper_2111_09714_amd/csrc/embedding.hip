// Embedding lookup with positions, and its gradient by sorted tokens (gfx950).
//
//   y[t] = scale table[ids[t]] + pos[t mod n];  ids outside [0, vocab) have no row (0)
//   dtable[v] = scale sum_{t : ids[t] = v} dy[t],   dpos[p] = sum_b dy[b n + p]
//
// The lookup is a gather of rows, L lanes to a row.  The gradient never adds to memory: tokens are
// put in the order of their ids and every row of dtable is one sum in the order of its tokens,
// the same bits every time.
//
//   rank   per block of tokens: how many fall into each bucket of W = 2^s neighbouring ids (at most 2048
//          buckets), and each token's rank among them, from ballots over its wave.  That leaves most of
//          the card idle; other workgroups sum the positions meanwhile;
//   place  the block's start in every bucket from all blocks' counts, then each token to its place.  Few
//          tokens are ranked and placed by one block;
//   sum    one workgroup per chunk of up to E tokens, of a few neighbouring buckets or a part of a full
//          one: orders them by id in LDS, then groups of lanes add their shares of that order, runs that
//          cross groups through LDS.  Buckets within one chunk end in dtable; of a bucket of several
//          (frequent ids) each chunk leaves fp32 rows of its ids.  Beside them one workgroup per bucket
//          writes zeros to the rows that do not occur;
//   join   adds the rows that chunks left, in chunk order.
//
// Up to 512 tokens take one launch: a workgroup per range of ids looks through all tokens.
//
// Bound by memory where tables or rows are large (dy read once, a second time for the positions; dtable
// written once), by the latency of four short launches otherwise.  16384 tokens x 768 fp32 into 30000 rows with
// positions: 53 us, 44 where the outputs' memory is used again (rank with positions 13 to 20, place 6, sum 21, join 6 to 7);
// 65536 x 768 bf16 55 us (8, 8, 34, 5); 65536 x 128 bf16 into 256 rows 26 us (6, 6, 10, 4); 512 x 768 fp32 16 us, which
// is the rate of a fill.
#include "common.h"
#include "launch.h"
#include "rows.h"
#include "timing.h"

namespace yoso {

namespace {

// ------------------------------------------------------------------ lookup

// 16384 tokens x 768 bf16 with positions 8.3 us, 5 TB/s; one token 2 us, and 8 with the host's call.
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

// ------------------------------------------------------------------ positions

constexpr int kSumThreads = 256;

struct Sums {
    const void *dy;
    void *dtable;
    int64_t d;
    float scale;
    int shift, entries_log;
    const uint2 *entry;
    const uint4 *items, *multi;
    const uint32_t *head, *bucket;
    const void *ids;  // of up to kScanTokens tokens, not sorted
    int64_t tokens, vocab;
    bool wide;
    int range;       // ids of a workgroup, then
    uint2 *present;  // [slots][kMaxWords] 32 ids of the bucket each: those that the chunk has, and how many it has before them
    float *partial;  // rows [stride] of a chunk's ids, from row slot slot_rows on, or, where that is 0, from its first entry's
    int64_t stride;
    uint32_t slot_rows;
    // positions
    int64_t item_blocks, zero_blocks, pos_blocks, n, batch, parts;
    int split;
    void *dpos;
    float *pos_partial;  // [parts][n][d]
};

// The block of positions of this workgroup, of a grid whose first `others` columns are not for positions (pos_grid).
__device__ __forceinline__ int64_t position_block(int64_t others) {
    return blockIdx.x - others + blockIdx.z * (gridDim.x - others);
}

// dpos[p], or of `parts` > 1 a part's fp32 sums [part][n][d]: `split` groups of lanes take one position, each every
// split-th sequence of the part, and join through `sums`, [T / L][NV][N][L] floats of LDS.
template <bool BF16, int LAYOUT, int L, int NV, int T>
__device__ __forceinline__ void sum_positions(const Sums &a, int64_t block, float *sums) {
    if (block >= a.pos_blocks) return;
    constexpr int N = Vec<BF16>::N, G = T / L, U = NV >= 3 ? 4 : 8;
    using Cols = Columns<BF16, LAYOUT>;
    const int lane = threadIdx.x % L, group = threadIdx.x / L, d = static_cast<int>(a.d), index = blockIdx.y * (64 * NV);
    const int split = a.split, sub = group % split;
    const int64_t n = a.n, blocks = (n + G / split - 1) / (G / split), part = block / blocks;
    const int64_t per = (a.batch + a.parts - 1) / a.parts;
    const int64_t p = block % blocks * (G / split) + group / split;
    const int64_t end = part * per + per < a.batch ? part * per + per : a.batch, b1 = p < n ? end : 0;
    float acc[NV][N];
#pragma unroll
    for (int i = 0; i < NV; i++)
#pragma unroll
        for (int j = 0; j < N; j++) acc[i][j] = 0.f;
    for (int64_t b = part * per + sub; b < b1; b += static_cast<int64_t>(U) * split) {
        raw4 v[U][NV];
#pragma unroll
        for (int u = 0; u < U; u++) {
            const int64_t q = b + u * split;
#pragma unroll
            for (int i = 0; i < NV; i++)
                v[u][i] = load_vec(a.dy, q < b1 ? (q * n + p) * d : 0, Cols(index + i * L + lane, d), d, q < b1);
        }
#pragma unroll
        for (int u = 0; u < U; u++)
#pragma unroll
            for (int i = 0; i < NV; i++)
#pragma unroll
                for (int j = 0; j < N; j++) acc[i][j] += value<BF16>(v[u][i], j);
    }
    if (split > 1) {
#pragma unroll
        for (int i = 0; i < NV; i++)
#pragma unroll
            for (int j = 0; j < N; j++) sums[((group * NV + i) * N + j) * L + lane] = acc[i][j];
        __syncthreads();
        if (sub) return;
        for (int q = 1; q < split; q++)
#pragma unroll
            for (int i = 0; i < NV; i++)
#pragma unroll
                for (int j = 0; j < N; j++) acc[i][j] += sums[(((group + q) * NV + i) * N + j) * L + lane];
    }
    if (p >= n) return;
#pragma unroll
    for (int i = 0; i < NV; i++) {
        const Cols col(index + i * L + lane, d);
        if (a.parts == 1) {
            store_vec(a.dpos, p * d, col, d, true, pack<BF16>(acc[i]));
        } else if (col.in) {
            float *to = a.pos_partial + (part * n + p) * d + col.c;
#pragma unroll
            for (int j = 0; j < N; j++)
                if (LAYOUT != kTiny || j < d) to[j] = acc[i][j];
        }
    }
}

// ------------------------------------------------------------------ order of the tokens

constexpr int kSortThreads = 512, kSortWaves = kSortThreads / 64;
constexpr int kMaxBuckets = 2048, kMaxWords = 16, kOwn = kMaxBuckets / kSortThreads;  // buckets of a thread
// tokens ranked at once, by a block and by a thread: with 4096 a rank takes 9 us, with 2048 6 (its rounds follow one another)
constexpr int kBatch = 2048, kPer = kBatch / kSortThreads;
constexpr int kMaxEntries = 1024;
constexpr uint32_t kNoSlot = 0xFFFFFFFFu;

struct Order {
    const void *ids;
    bool wide;
    int64_t tokens, vocab;
    int shift, buckets, blocks, entries_log;  // 2^entries_log entries of a chunk at most
    int64_t block_tokens;
    uint16_t *counts;  // [blocks][kMaxBuckets]
    uint16_t *rank;    // [tokens] within the block's tokens of the bucket
    uint2 *entry;      // [tokens] tokens and their ids, in bucket order
    uint4 *items;      // chunks: first entry, entries, slot of partial rows
    uint4 *multi;      // buckets of several chunks: bucket, first slot, chunks, first entry
    uint32_t *head;    // number of items, of buckets of several chunks
    uint32_t *bucket;  // [buckets + 1] first entries
};

// the id of token t, or -1 where it names no row
__device__ __forceinline__ int id_of(const Order &o, int64_t t, int64_t end) {
    if (t >= end) return -1;
    const int64_t id = o.wide ? static_cast<const int64_t *>(o.ids)[t] : static_cast<const int32_t *>(o.ids)[t];
    return id >= 0 && id < o.vocab ? static_cast<int>(id) : -1;
}

// Ranks of kBatch tokens from `at`: wave w takes the tokens w 64 kPer ... of them, 64 at a time.  The
// rank counts tokens of the same bucket that come before: in this batch, and in `run`, [kMaxBuckets],
// which is counted on.  wave_counts [kSortWaves][kMaxBuckets]; ends with a barrier.
__device__ __forceinline__ void rank_batch(const Order &o, int64_t at, int64_t end, uint16_t *wave_counts, uint16_t *run,
                                           int (&id)[kPer], uint32_t (&rank)[kPer]) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t t0 = at + wave * 64 * kPer + lane;
#pragma unroll
    for (int k = 0; k < kPer; k++) id[k] = id_of(o, t0 + 64 * k, end);
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

// Blocks of tokens, then positions, whose reads the card has time for meanwhile.
template <bool BF16, int LAYOUT, int L, int NV>
__global__ __launch_bounds__(kSortThreads) void embedding_rank_kernel(Order o, Sums a) {
    extern __shared__ uint4 lds[];
    static_assert(kSortThreads * NV * Vec<BF16>::N * sizeof(float) <= kRankLds, "the positions' sums");
    if (static_cast<int>(blockIdx.x) >= o.blocks)
        return sum_positions<BF16, LAYOUT, L, NV, kSortThreads>(a, position_block(o.blocks), reinterpret_cast<float *>(lds));
    if (blockIdx.y || blockIdx.z) return;  // (those are for the positions)
    uint16_t *run = reinterpret_cast<uint16_t *>(lds), *wave_counts = run + kMaxBuckets;
    for (int b = threadIdx.x; b < kMaxBuckets; b += kSortThreads) run[b] = 0;
    const int64_t from = blockIdx.x * o.block_tokens, to = from + o.block_tokens;
    const int64_t end = to < o.tokens ? to : o.tokens;
    for (int64_t at = from; at < end; at += kBatch) {
        int id[kPer];
        uint32_t rank[kPer];
        rank_batch(o, at, end, wave_counts, run, id, rank);
        const int64_t t0 = at + (threadIdx.x >> 6) * 64 * kPer + (threadIdx.x & 63);
#pragma unroll
        for (int k = 0; k < kPer; k++)
            if (id[k] >= 0) o.rank[t0 + 64 * k] = static_cast<uint16_t>(rank[k]);
    }
    uint4 *out = reinterpret_cast<uint4 *>(o.counts + static_cast<int64_t>(blockIdx.x) * kMaxBuckets);
    for (int i = threadIdx.x; i < kMaxBuckets / 8; i += kSortThreads) out[i] = reinterpret_cast<const uint4 *>(run)[i];
}

// exclusive sums of Q values over the workgroup's threads
template <int Q>
struct Counts {
    uint32_t v[Q];
};

template <int Q>
__device__ __forceinline__ Counts<Q> scan(const Counts<Q> &own, Counts<Q> *wave_sums, Counts<Q> &total) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    Counts<Q> s = own;
#pragma unroll
    for (int k = 1; k < 64; k *= 2)
#pragma unroll
        for (int q = 0; q < Q; q++) {
            const uint32_t x = __shfl_up(s.v[q], k);
            s.v[q] += lane >= k ? x : 0;
        }
    if (lane == 63) wave_sums[wave] = s;
    __syncthreads();
#pragma unroll
    for (int q = 0; q < Q; q++) {
        s.v[q] -= own.v[q];
        total.v[q] = 0;
    }
#pragma unroll
    for (int w = 0; w < kSortWaves; w++)
#pragma unroll
        for (int q = 0; q < Q; q++) {
            const uint32_t x = wave_sums[w].v[q];
            s.v[q] += w < wave ? x : 0;
            total.v[q] += x;
        }
    return s;
}

// The list of chunks, by one workgroup: a thread packs its own neighbouring buckets into chunks of at most E = 2^e entries;
// larger buckets are split, which all threads write.
struct Split {
    uint32_t bucket, first, size, item, slot;
};

__device__ __forceinline__ void list_chunks(const Order &o, const uint32_t (&total)[kOwn], Split *split) {
    __shared__ Counts<4> wave_sums[kSortWaves];
    const uint32_t e = o.entries_log, E = 1u << e;
    // entries, chunks, chunks of split buckets, split buckets
    const auto walk = [&](auto &&chunk, auto &&large) {
        Counts<4> n{};
        uint32_t pack = 0;
#pragma unroll
        for (int k = 0; k <= kOwn; k++) {
            const uint32_t t = k < kOwn ? total[k] : E;  // (the end closes the last chunk)
            if (pack && pack + t > E) {
                chunk(n, pack);
                n.v[1]++;
                n.v[0] += pack;
                pack = 0;
            }
            if (k < kOwn && t > E) {
                const uint32_t parts = (t + E - 1) >> e;
                large(n, k, t);
                n.v[0] += t;
                n.v[1] += parts;
                n.v[2] += parts;
                n.v[3]++;
            } else if (k < kOwn) {
                pack += t;
            }
        }
        return n;
    };
    Counts<4> all;
    const Counts<4> own = walk([](const Counts<4> &, uint32_t) {}, [](const Counts<4> &, int, uint32_t) {});
    const Counts<4> prior = scan<4>(own, wave_sums, all);
    walk([&](const Counts<4> &n, uint32_t entries) {
             o.items[prior.v[1] + n.v[1]] = make_uint4(prior.v[0] + n.v[0], entries, kNoSlot, 0);
         },
         [&](const Counts<4> &n, int k, uint32_t t) {
             split[prior.v[3] + n.v[3]] = {static_cast<uint32_t>(threadIdx.x) * kOwn + k, prior.v[0] + n.v[0], t,
                                           prior.v[1] + n.v[1], prior.v[2] + n.v[2]};
         });
    uint32_t first = prior.v[0];
#pragma unroll
    for (int k = 0; k < kOwn; k++) {
        const int b = threadIdx.x * kOwn + k;
        if (b < o.buckets) o.bucket[b] = first;
        first += total[k];
    }
    if (threadIdx.x == 0) {
        o.head[0] = all.v[1];
        o.head[1] = all.v[3];
        o.bucket[o.buckets] = all.v[0];
    }
    __syncthreads();
    for (uint32_t i = threadIdx.x >> 6; i < all.v[3]; i += kSortWaves) {
        const Split w = split[i];
        const uint32_t parts = (w.size + E - 1) >> e;
        if ((threadIdx.x & 63) == 0) o.multi[i] = make_uint4(w.bucket, w.slot, parts, w.first);
        for (uint32_t q = threadIdx.x & 63; q < parts; q += 64)
            o.items[w.item + q] = make_uint4(w.first + (q << e), min(E, w.size - (q << e)), w.slot + q, 0);
    }
}

// (a single block's split buckets, at most kBatch / 33, take the place of its ranks)
static_assert(kBatch / 33 * sizeof(Split) <= kRankLds, "the list of a single block");

// Blocks of tokens, then one for the list of chunks.  ONE: a single block, which ranks for itself and makes
// the list too.
template <bool ONE>
__global__ __launch_bounds__(kSortThreads) void embedding_place_kernel(Order o) {
    const int lister = ONE ? 0 : o.blocks;
    extern __shared__ uint4 lds[];
    __shared__ uint32_t start[kMaxBuckets];  // where this block's tokens of a bucket go
    __shared__ Counts<1> wave_sums[kSortWaves];
    const int64_t from = blockIdx.x * o.block_tokens, to = from + o.block_tokens;
    const int64_t end = to < o.tokens ? to : o.tokens;
    int id[kPer];
    uint32_t rank[kPer];
    const auto token = [&](int64_t at, int k) { return at + (threadIdx.x >> 6) * 64 * kPer + (threadIdx.x & 63) + 64 * k; };
    const auto fetch = [&](int64_t at) {
#pragma unroll
        for (int k = 0; k < kPer; k++) {
            id[k] = id_of(o, token(at, k), end);
            rank[k] = token(at, k) < end ? o.rank[token(at, k)] : 0;  // (used where the token has a row)
        }
    };
    uint32_t total[kOwn], before[kOwn];
    const int own = threadIdx.x * kOwn;
    static_assert(kOwn == 4, "a thread's counts are one uint2");
    const auto add = [&](uint32_t (&sum)[kOwn], const uint2 &c, bool counts) {
        sum[0] += counts ? c.x & 0xFFFFu : 0;
        sum[1] += counts ? c.x >> 16 : 0;
        sum[2] += counts ? c.y & 0xFFFFu : 0;
        sum[3] += counts ? c.y >> 16 : 0;
    };
#pragma unroll
    for (int k = 0; k < kOwn; k++) total[k] = before[k] = 0;
    if constexpr (ONE) {
        uint16_t *run = reinterpret_cast<uint16_t *>(lds), *wave_counts = run + kMaxBuckets;
        for (int b = threadIdx.x; b < kMaxBuckets; b += kSortThreads) run[b] = 0;
        rank_batch(o, from, end, wave_counts, run, id, rank);
        add(total, *reinterpret_cast<const uint2 *>(run + own), true);
        __syncthreads();  // (the list takes the same LDS)
    } else {
        if (static_cast<int>(blockIdx.x) < lister) fetch(from);
        if (own < o.buckets) {
            constexpr int kRows = 16;  // rows of counts in flight
            for (int q = 0; q < o.blocks; q += kRows) {
                uint2 c[kRows];
#pragma unroll
                for (int r = 0; r < kRows; r++) {
                    const int64_t block = min(q + r, o.blocks - 1);
                    c[r] = *reinterpret_cast<const uint2 *>(o.counts + block * kMaxBuckets + own);
                }
#pragma unroll
                for (int r = 0; r < kRows; r++) {
                    add(total, c[r], q + r < o.blocks);
                    add(before, c[r], q + r < static_cast<int>(blockIdx.x));
                }
            }
        }
    }
    if (static_cast<int>(blockIdx.x) == lister) list_chunks(o, total, reinterpret_cast<Split *>(lds));
    if (!ONE && static_cast<int>(blockIdx.x) == lister) return;
    Counts<1> mine{}, all;
#pragma unroll
    for (int k = 0; k < kOwn; k++) mine.v[0] += total[k];
    uint32_t at = scan<1>(mine, wave_sums, all).v[0];
#pragma unroll
    for (int k = 0; k < kOwn; k++) {
        start[own + k] = at + before[k];
        at += total[k];
    }
    __syncthreads();
    for (int64_t batch = from; batch < end; batch += kBatch) {
        if (!ONE && batch > from) fetch(batch);
#pragma unroll
        for (int k = 0; k < kPer; k++)
            if (id[k] >= 0) {
                o.entry[start[id[k] >> o.shift] + rank[k]] = make_uint2(static_cast<uint32_t>(token(batch, k)), id[k]);
            }
    }
}

// ------------------------------------------------------------------ sums

// Zeros to the rows first ... first + rows - 1 of dtable whose bit is not set.
template <bool BF16, int LAYOUT, int L, int NV>
__device__ __forceinline__ void zero_rows(const Sums &a, int64_t first, int rows, const uint32_t *present) {
    using Cols = Columns<BF16, LAYOUT>;
    const int d = static_cast<int>(a.d), index = blockIdx.y * (64 * NV);
    for (int r = threadIdx.x / L; r < rows; r += kSumThreads / L)
        if (!(present[r >> 5] >> (r & 31) & 1))
#pragma unroll
            for (int i = 0; i < NV; i++) {
                const Cols col(index + i * L + static_cast<int>(threadIdx.x) % L, d);
                store_vec(a.dtable, (first + r) * d, col, d, true, raw4{0, 0, 0, 0});
            }
}

// E entries at most, ordered by id
template <int E, int L, int NV, int N>
struct Chunk {
    __align__(16) uint32_t key[E];
    uint32_t token[E], id[E];
    float carry[kSumThreads / L][NV][N][L];  // a group's first run, where it began in a group before
    unsigned long long open;                 // bit g: ... and it goes on behind group g
};

// Brings a thread's entries, tid, tid + kSumThreads ... of len, into the order of their keys (all different).
template <int Q, typename C>
__device__ __forceinline__ void order(C &c, int len, const uint32_t *key, const uint32_t *token, const uint32_t *id) {
    int at[Q];
#pragma unroll
    for (int q = 0; q < Q; q++) at[q] = 0;
#pragma unroll 4
    for (int i = 0; i < len; i += 4) {
        const uint4 other = *reinterpret_cast<const uint4 *>(&c.key[i]);
#pragma unroll
        for (int q = 0; q < Q; q++)
            at[q] += (other.x < key[q]) + (other.y < key[q]) + (other.z < key[q]) + (other.w < key[q]);
    }
#pragma unroll
    for (int q = 0; q < Q; q++)
        if (static_cast<int>(threadIdx.x) + q * kSumThreads < len) {
            c.token[at[q]] = token[q];
            c.id[at[q]] = id[q];
        }
    __syncthreads();
}

// Where a chunk of a split bucket leaves its rows: in the order of the ids that it has.
struct Slot {
    uint32_t row;
    uint32_t mask;
    const uint2 *present;  // nullptr: the chunk's rows go to dtable

    __device__ __forceinline__ uint32_t of(uint32_t id) const {
        const uint2 w = present[(id & mask) >> 5];
        return row + w.y + __popc(w.x & ((1u << (id & mask & 31)) - 1));
    }
};

// The sums of a chunk's runs: to dtable, or, of a split bucket, to the chunk's rows.
template <bool BF16, int LAYOUT, int L, int NV, typename C>
__device__ __forceinline__ void sum_chunk(const Sums &a, C &c, int len, const Slot &slot) {
    constexpr int N = Vec<BF16>::N, G = kSumThreads / L;
    constexpr int U = NV >= 3 ? 4 : 8;  // rows in flight
    using Cols = Columns<BF16, LAYOUT>;
    const int d = static_cast<int>(a.d), lane = threadIdx.x % L, group = threadIdx.x / L;
    const int per = (len + G - 1) / G;
    const int p0 = min(group * per, len), p1 = min(p0 + per, len);
    const int index = blockIdx.y * (64 * NV);  // first vector of this block of columns (L = 64 where there are several)
    float acc[NV][N];
    const auto clear = [&]() {
#pragma unroll
        for (int i = 0; i < NV; i++)
#pragma unroll
            for (int j = 0; j < N; j++) acc[i][j] = 0.f;
    };
    const auto finish = [&](uint32_t id) {
        const int64_t row = slot.present ? slot.of(id) : id;
#pragma unroll
        for (int i = 0; i < NV; i++) {
            const Cols col(index + i * L + lane, d);
            if (slot.present == nullptr) {
                float f[N];
#pragma unroll
                for (int j = 0; j < N; j++) f[j] = acc[i][j] * a.scale;
                store_vec(a.dtable, row * d, col, d, true, pack<BF16>(f));
            } else if (col.in) {
                float *to = a.partial + row * a.stride + col.c;
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
            for (int j = 0; j < N; j++) c.carry[group][i][j][lane] = acc[i][j];
    };
    clear();
    bool from_before = p0 < p1 && p0 > 0 && c.id[p0 - 1] == c.id[p0];
    uint32_t cur = p0 < p1 ? c.id[p0] : 0;
    for (int p = p0; p < p1; p += U) {
        raw4 v[U][NV];
#pragma unroll
        for (int u = 0; u < U; u++) {
            const bool there = p + u < p1;
            const int64_t row = there ? static_cast<int64_t>(c.token[p + u]) * d : 0;
#pragma unroll
            for (int i = 0; i < NV; i++) v[u][i] = load_vec(a.dy, row, Cols(index + i * L + lane, d), d, there);
        }
#pragma unroll
        for (int u = 0; u < U; u++) {
            if (p + u < p1) {
                if (c.id[p + u] != cur) {
                    if (from_before)
                        keep();
                    else
                        finish(cur);
                    from_before = false;
                    cur = c.id[p + u];
                    clear();
                }
#pragma unroll
                for (int i = 0; i < NV; i++)
#pragma unroll
                    for (int j = 0; j < N; j++) acc[i][j] += value<BF16>(v[u][i], j);
            }
        }
    }
    const bool goes_on = p0 < p1 && p1 < len && c.id[p1] == cur;
    if (p0 < p1) {
        if (from_before) {
            keep();
            if (lane == 0 && goes_on) atomicOr(&c.open, 1ull << group);
        } else if (!goes_on) {
            finish(cur);
        }
    }
    __syncthreads();
    if (p0 < p1 && !from_before && goes_on) {
        const int last = group + __ffsll(~(c.open >> (group + 1)));  // the group in which the run ends
#pragma unroll 4
        for (int g = group + 1; g <= last; g++)
#pragma unroll
            for (int i = 0; i < NV; i++)
#pragma unroll
                for (int j = 0; j < N; j++) acc[i][j] += c.carry[g][i][j][lane];
        finish(cur);
    }
}

// Chunks, then zeros, then positions.
template <bool BF16, int LAYOUT, int L, int NV>
__global__ __launch_bounds__(kSumThreads) void embedding_sum_kernel(Sums a) {
    __shared__ Chunk<kMaxEntries, L, NV, Vec<BF16>::N> c;
    __shared__ uint32_t present[kMaxWords];
    __shared__ uint2 places[kMaxWords];
    const int tid = threadIdx.x;
    if (blockIdx.x >= a.item_blocks + a.zero_blocks)
        return sum_positions<BF16, LAYOUT, L, NV, kSumThreads>(a, position_block(a.item_blocks + a.zero_blocks), &c.carry[0][0][0][0]);
    const uint32_t local_mask = (1u << a.shift) - 1;
    if (tid < kMaxWords) present[tid] = 0;
    if (blockIdx.x >= a.item_blocks) {
        // the rows of a bucket that do not occur (of a split one, the join knows)
        const int64_t b = blockIdx.x - a.item_blocks;
        const uint32_t first = a.bucket[b], size = a.bucket[b + 1] - first;
        if (size > 1u << a.entries_log) return;
        __syncthreads();
        for (uint32_t i = tid; i < size; i += kSumThreads) {
            const uint32_t local = a.entry[first + i].y & local_mask;
            atomicOr(&present[local >> 5], 1u << (local & 31));
        }
        __syncthreads();
        const int64_t row = b << a.shift, left = a.vocab - row, width = int64_t{1} << a.shift;
        return zero_rows<BF16, LAYOUT, L, NV>(a, row, static_cast<int>(left < width ? left : width), present);
    }
    const uint4 it = a.items[blockIdx.x];  // first entry, entries, slot
    if (blockIdx.x >= a.head[0]) return;
    const int len = it.y;
    // in the order of (id, place before); a chunk's ids lie within kOwn W <= 2^11 of each other
    constexpr int Q = kMaxEntries / kSumThreads;
    uint32_t token[Q], id[Q], key[Q];
    if (tid == 0) c.open = 0;
#pragma unroll
    for (int q = 0; q < Q; q++) {
        const int i = q * kSumThreads + tid;
        const uint2 e = i < len ? a.entry[it.x + i] : make_uint2(0, 0);
        token[q] = e.x;
        id[q] = e.y;
        key[q] = i < len ? (e.y & ((static_cast<uint32_t>(kOwn) << a.shift) - 1)) << 10 | i : 0xFFFFFFFFu;
        c.key[i] = key[q];
    }
    __syncthreads();
    if (it.z != kNoSlot)
#pragma unroll
        for (int q = 0; q < Q; q++)
            if (q * kSumThreads + tid < len) atomicOr(&present[(id[q] & local_mask) >> 5], 1u << (id[q] & local_mask & 31));
    if (a.shift == 0) {  // (a bucket is an id: the entries are in order)
#pragma unroll
        for (int q = 0; q < Q; q++)
            if (q * kSumThreads + tid < len) {
                c.token[q * kSumThreads + tid] = token[q];
                c.id[q * kSumThreads + tid] = id[q];
            }
        __syncthreads();
    } else if (len <= kSumThreads) {
        order<1>(c, len, key, token, id);
    } else {
        order<Q>(c, len, key, token, id);
    }
    Slot slot{0, local_mask, nullptr};
    if (it.z != kNoSlot) {
        if (tid < kMaxWords) {
            uint2 w = make_uint2(present[tid], 0);
            for (int i = 0; i < tid; i++) w.y += __popc(present[i]);
            places[tid] = w;
            if (blockIdx.y == 0) a.present[static_cast<int64_t>(it.z) * kMaxWords + tid] = w;
        }
        __syncthreads();
        slot = {a.slot_rows ? it.z * a.slot_rows : it.x, local_mask, places};
    }
    sum_chunk<BF16, LAYOUT, L, NV>(a, c, len, slot);
}

// Few tokens: a workgroup takes a.range ids, looks through all tokens for them, sums their rows and writes zeros to the
// rows of the others.  Then positions.
constexpr int kScanTokens = 512, kScanRange = 1024;

template <bool BF16, int LAYOUT, int L, int NV>
__global__ __launch_bounds__(kSumThreads) void embedding_scan_kernel(Sums a) {
    constexpr int Q = kScanTokens / kSumThreads, W = kSumThreads / 64;
    __shared__ Chunk<kScanTokens, L, NV, Vec<BF16>::N> c;
    __shared__ uint32_t present[kScanRange / 32];
    __shared__ int found[Q * W];
    if (blockIdx.x >= a.zero_blocks)
        return sum_positions<BF16, LAYOUT, L, NV, kSumThreads>(a, position_block(a.zero_blocks), &c.carry[0][0][0][0]);
    if (blockIdx.z) return;
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
    const int64_t lo = static_cast<int64_t>(blockIdx.x) * a.range, left = a.vocab - lo;
    const int rows = static_cast<int>(left < a.range ? left : a.range);
    if (tid < kScanRange / 32) present[tid] = 0;
    if (tid == 0) c.open = 0;
    int64_t id[Q];
    unsigned long long hits[Q];
#pragma unroll
    for (int q = 0; q < Q; q++) {
        const int64_t t = q * kSumThreads + tid;
        id[q] = t >= a.tokens ? -1 : a.wide ? static_cast<const int64_t *>(a.ids)[t] : static_cast<const int32_t *>(a.ids)[t];
        hits[q] = __ballot(id[q] >= lo && id[q] < lo + rows);
        if (lane == 0) found[q * W + wave] = __popcll(hits[q]);
    }
    __syncthreads();
    int len = 0;
    int first[Q];
#pragma unroll
    for (int i = 0; i < Q * W; i++) {
#pragma unroll
        for (int q = 0; q < Q; q++)
            if (i == q * W + wave) first[q] = len;
        len += found[i];
    }
#pragma unroll
    for (int q = 0; q < Q; q++)
        if (hits[q] >> lane & 1) {
            const int at = first[q] + __popcll(hits[q] & ((1ull << lane) - 1));
            const uint32_t local = static_cast<uint32_t>(id[q] - lo);
            c.key[at] = local << 16 | (q * kSumThreads + tid);
            atomicOr(&present[local >> 5], 1u << (local & 31));
        }
    if (tid < 4 && len + tid < kScanTokens) c.key[len + tid] = 0xFFFFFFFFu;
    __syncthreads();
    uint32_t key[Q], token[Q], row[Q];
#pragma unroll
    for (int q = 0; q < Q; q++) {
        key[q] = q * kSumThreads + tid < len ? c.key[q * kSumThreads + tid] : 0xFFFFFFFFu;
        token[q] = key[q] & 0xFFFF;
        row[q] = static_cast<uint32_t>(lo) + (key[q] >> 16);
    }
    order<Q>(c, len, key, token, row);
    zero_rows<BF16, LAYOUT, L, NV>(a, lo, rows, present);
    if (len) sum_chunk<BF16, LAYOUT, L, NV>(a, c, len, Slot{0, 0, nullptr});
}

// The rows of buckets of several chunks: a workgroup takes an id (of large buckets a sixteenth of the ids) and 256
// columns, each of its waves a share of the chunks.  Most ids of such a bucket do not occur, which one word a chunk
// says: a wave reads those of 64 chunks at once.
// The blocks behind `join_blocks` add the parts of the positions.
constexpr int kJoinThreads = 512, kJoinWaves = kJoinThreads / 64;

template <bool BF16>
__global__ __launch_bounds__(kJoinThreads) void embedding_join_kernel(Sums a, int join_blocks) {
    __shared__ float4 sums[kJoinWaves][64];
    __shared__ uint32_t any;
    if (static_cast<int>(blockIdx.x) >= join_blocks) {
        const int64_t values = a.n * a.d, step = static_cast<int64_t>(gridDim.x - join_blocks) * kJoinThreads;
        for (int64_t e = static_cast<int64_t>(blockIdx.x - join_blocks) * kJoinThreads + threadIdx.x; e < values; e += step) {
            float s = 0.f;
#pragma unroll 8
            for (int64_t q = 0; q < a.parts; q++) s += a.pos_partial[q * values + e];
            if constexpr (BF16)
                static_cast<__bf16 *>(a.dpos)[e] = static_cast<__bf16>(s);
            else
                static_cast<float *>(a.dpos)[e] = s;
        }
        return;
    }
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int column_blocks = static_cast<int>((a.d + 255) / 256);
    const int ids_log = a.shift > 4 ? a.shift - 4 : 0;  // ids of an item: 16 items a bucket
    const int64_t items = (static_cast<int64_t>(a.head[1]) << (a.shift - ids_log)) * column_blocks;
    for (int64_t i = blockIdx.x; i < items; i += join_blocks) {
        const int c = static_cast<int>(i % column_blocks) * 256 + lane * 4;
        const int64_t q = i / column_blocks;
        const uint32_t id0 = (static_cast<uint32_t>(q) & ((1u << (a.shift - ids_log)) - 1)) << ids_log;
        const uint4 m = a.multi[q >> (a.shift - ids_log)];  // bucket, first slot, chunks, first entry
        const int chunks = m.z, per = (chunks + kJoinWaves - 1) / kJoinWaves;
        const int from = wave * per, to = min(from + per, chunks);
        const auto words = [&](int k0) {  // of 64 chunks, for the 32 ids around id0
            const int64_t slot = static_cast<int64_t>(m.y) + k0 + lane;
            return k0 + lane < to ? a.present[slot * kMaxWords + (id0 >> 5)] : make_uint2(0, 0);
        };
        // the ids that any chunk has
        uint32_t mine = 0;
        for (int k0 = from; k0 < to; k0 += 64) mine |= words(k0).x;
        __syncthreads();  // (the sums below have been read)
        if (threadIdx.x == 0) any = 0;
        __syncthreads();
        if (mine) atomicOr(&any, mine);
        __syncthreads();
        for (uint32_t id = id0; id < id0 + (1u << ids_log); id++) {
            const int64_t row_id = (static_cast<int64_t>(m.x) << a.shift) + id;
            if (row_id >= a.vocab) break;
            float t[4] = {0.f, 0.f, 0.f, 0.f};
            if (any >> (id & 31) & 1) {
                float s[4] = {0.f, 0.f, 0.f, 0.f};
                for (int k0 = from; k0 < to; k0 += 64) {
                    const uint32_t at = m.y + k0 + lane, below = (1u << (id & 31)) - 1;
                    const uint2 w = words(k0);
                    const uint32_t row0 = a.slot_rows ? at * a.slot_rows : m.w + ((k0 + lane) << a.entries_log);
                    const uint32_t row = row0 + w.y + __popc(w.x & below);
                    unsigned long long has = __ballot((w.x >> (id & 31)) & 1);
                    while (has) {
                        constexpr int U = 8;  // rows in flight
                        float4 v[U];
                        int n = 0;
#pragma unroll
                        for (int u = 0; u < U; u++) {
                            v[u] = make_float4(0.f, 0.f, 0.f, 0.f);
                            if (has) {
                                const int k = __ffsll(has) - 1;
                                has &= has - 1;
                                const int64_t r = static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(row), k));
                                if (c < a.d) v[u] = *reinterpret_cast<const float4 *>(a.partial + r * a.stride + c);
                                n = u + 1;
                            }
                        }
#pragma unroll
                        for (int u = 0; u < U; u++)
                            if (u < n) {
                                s[0] += v[u].x; s[1] += v[u].y; s[2] += v[u].z; s[3] += v[u].w;
                            }
                    }
                }
                if (id > id0) __syncthreads();
                sums[wave][lane] = make_float4(s[0], s[1], s[2], s[3]);
                __syncthreads();
                if (wave == 0)
#pragma unroll
                    for (int w = 0; w < kJoinWaves; w++) {
                        const float4 v = sums[w][lane];
                        t[0] += v.x; t[1] += v.y; t[2] += v.z; t[3] += v.w;
                    }
            }
            if (wave == 0)
                for (int j = 0; j < 4 && c + j < a.d; j++) {
                    if constexpr (BF16)
                        static_cast<__bf16 *>(a.dtable)[row_id * a.d + c + j] = static_cast<__bf16>(t[j] * a.scale);
                    else
                        static_cast<float *>(a.dtable)[row_id * a.d + c + j] = t[j] * a.scale;
                }
        }
    }
}

// ------------------------------------------------------------------ host

int64_t up(int64_t a, int64_t b) { return (a + b - 1) / b; }

int shift_of(int64_t vocab) {
    int s = 0;
    while (((vocab - 1) >> s) + 1 > kMaxBuckets) s++;
    return s;
}

// Lanes and vectors for a row, or a block of its columns where a wave of four (16 bits: two) vectors a lane does
// not take it.
struct Form {
    int lanes, vectors, blocks;
};

// Where few tokens are scanned for, rows of more than 32 vectors are shared by workgroups with one vector a lane: a run
// of most tokens is then the work of several, 512 tokens x 768 fp32 of one id 42 us (with three vectors a lane 49).
Form form_of(bool bf16, int d, bool scan) {
    const int n = bf16 ? 8 : 4, nvec = (d + n - 1) / n, most = scan ? 1 : bf16 ? 2 : 4;
    int lanes = 4;
    while (lanes < 64 && nvec > (scan && lanes >= 32 ? 1 : 2) * lanes) lanes *= 2;
    const int blocks = static_cast<int>(up(nvec, 64 * most));
    return {lanes, static_cast<int>(up(nvec, static_cast<int64_t>(lanes) * blocks)), blocks};
}

// How the sum over a batch is shared: groups of lanes to a position (four sequences each at least), and, where the positions
// are so few that this gives less than 512 workgroups, parts of the batch (eight sequences a group at least).
struct PosPlan {
    int split;
    int64_t parts, blocks;  // blocks of one part
};

PosPlan pos_plan(bool bf16, int64_t tokens, int64_t n, int d) {
    PosPlan p{1, 1, 0};
    if (n == 0) return p;
    const int64_t batch = tokens / n;
    const int groups = (tokens > kBatch ? kSortThreads : kSumThreads) / form_of(bf16, d, tokens <= kScanTokens).lanes;
    while (p.split < groups && 8 * p.split <= batch) p.split *= 2;
    p.blocks = up(n, groups / p.split);
    const int64_t want = 512 / p.blocks, most = batch / (8 * p.split);
    p.parts = want < most ? want : most;
    if (p.parts < 1) p.parts = 1;
    return p;
}

struct Layout {
    size_t counts, rank, entry, items, multi, head, bucket, present, partial, pos, total;
    int64_t blocks, block_tokens, max_items, max_multi, stride;
    int64_t buckets;
    int shift, entries_log;
    uint32_t slot_rows;
};

Layout layout_of(bool bf16, int64_t tokens, int64_t n, int64_t vocab, int d) {
    Layout l{};
    l.shift = shift_of(vocab);
    l.buckets = ((vocab - 1) >> l.shift) + 1;
    const int64_t parts = pos_plan(bf16, tokens, n, d).parts;
    const size_t pos_bytes = parts > 1 ? static_cast<size_t>(parts) * n * d * 4 : 0;
    if (tokens <= kScanTokens) {
        l.total = pos_bytes;
        return l;
    }
    // 128 blocks of tokens, less where there are few; more where a block's tokens would pass the 16-bit ranks
    l.blocks = up(tokens, kBatch);
    const int64_t most = up(tokens, 65535);
    if (l.blocks > 128) l.blocks = most > 128 ? most : 128;
    l.block_tokens = up(tokens, l.blocks);
    // Entries of a chunk: about 1000 chunks for the 256 CUs.  65536 x 768 bf16: E = 128 59 us, 64 64 us (more rows left for
    // the join), 256 63 us (too few workgroups).  A bucket's share of very many tokens spread evenly still is one chunk
    // (786432 x 768 bf16 into 30000 rows: 419 a bucket; with E = 256 all were split, and the join took 200 us of 580, now
    // 335); narrow rows are summed faster than as many entries are ordered (2^24 x 16 fp32: E = 1024 1619 us, of which sums
    // 958; E = 256 1325, 558; near the threshold it is even: 2^21 x 64 fp32 184 and 189).
    l.stride = up(d, 8) * 8;
    l.entries_log = 5;
    const int most_entries = l.stride * (bf16 ? 2 : 4) >= 512 ? kMaxEntries : kMaxEntries / 4;
    while ((1 << l.entries_log) < most_entries && tokens >> l.entries_log >= 1024) l.entries_log++;
    // A chunk and the next one of the same thread hold more than E entries, but for the last part of a split bucket
    // (there are fewer than tokens / E such): at most 4 tokens / E chunks and one more a thread.
    const int64_t chunks = 4 * (tokens >> l.entries_log) + kSortThreads + 4;
    l.max_items = tokens < chunks ? tokens : chunks;
    l.max_multi = tokens / ((1 << l.entries_log) + 1);
    const int64_t slots = l.max_multi ? 2 * (tokens >> l.entries_log) : 0;
    size_t at = 0;
    const auto place = [&](size_t &off, size_t bytes) {
        off = at;
        at += (bytes + 255) / 256 * 256;
    };
    place(l.counts, l.blocks > 1 ? static_cast<size_t>(l.blocks) * kMaxBuckets * 2 : 0);
    place(l.rank, l.blocks > 1 ? static_cast<size_t>(tokens) * 2 : 0);
    place(l.entry, static_cast<size_t>(tokens) * 8);
    place(l.items, static_cast<size_t>(l.max_items) * 16);
    place(l.multi, static_cast<size_t>(l.max_multi) * 16);
    place(l.head, 16);
    place(l.bucket, (l.buckets + 1) * 4);
    place(l.present, static_cast<size_t>(slots) * kMaxWords * 8);
    // A chunk leaves a row an id, at most as many as it has entries: so many rows a slot, or, where all slots' would be more
    // than the entries, the rows of its entries' places.
    const int64_t width = int64_t{1} << (l.shift < l.entries_log ? l.shift : l.entries_log);
    l.slot_rows = slots * width <= tokens ? static_cast<uint32_t>(width) : 0;
    place(l.partial, static_cast<size_t>(l.slot_rows ? slots * width : slots ? tokens : 0) * l.stride * 4);
    place(l.pos, pos_bytes);
    l.total = at;
    return l;
}

// SCAN: the forms of rows that are scanned for
template <bool SCAN, bool BF16, int LAYOUT, typename F>
void with_form(int d, F f) {
    const Form form = form_of(BF16, d, SCAN);
#define YOSO_ROW_FORM(L_, NV_) \
    if (form.lanes == L_ && form.vectors == NV_) return f.template operator()<BF16, LAYOUT, L_, NV_>(form.blocks);
    YOSO_ROW_FORM(4, 1)
    if constexpr (LAYOUT != kTiny) {
        YOSO_ROW_FORM(4, 2) YOSO_ROW_FORM(8, 2) YOSO_ROW_FORM(16, 2)
        if constexpr (SCAN) {
            YOSO_ROW_FORM(64, 1)
        } else {
            YOSO_ROW_FORM(32, 2) YOSO_ROW_FORM(64, 2)
            if constexpr (!BF16) {
                YOSO_ROW_FORM(64, 3) YOSO_ROW_FORM(64, 4)
            }
        }
    }
#undef YOSO_ROW_FORM
}

template <bool SCAN, bool BF16, typename F>
void with_layout(int d, F f) {
    constexpr int N = Vec<BF16>::N;
    if (d % N == 0)
        with_form<SCAN, BF16, kAligned>(d, f);
    else if (d > N)
        with_form<SCAN, BF16, kOverlap>(d, f);
    else
        with_form<SCAN, BF16, kTiny>(d, f);
}

template <bool SCAN, typename F>
hipError_t with_layout(bool bf16, int d, F f) {
    bf16 ? with_layout<SCAN, true>(d, f) : with_layout<SCAN, false>(d, f);
    return hipGetLastError();
}

// The grid of `others` workgroups and those of the positions.  A grid's side must stay below 2^32 threads (a launch of more
// reports no error, and runs what is left modulo 2^32), so that more than 2^22 workgroups of positions, of up to 512 threads
// each, go on in the next layer.
dim3 pos_grid(Sums &a, int64_t others, int groups, int blocks) {
    constexpr int64_t kMost = int64_t{1} << 22;
    a.pos_blocks = up(a.n, groups / a.split) * a.parts;
    const int64_t layer = a.pos_blocks < kMost ? a.pos_blocks : kMost;
    return dim3(static_cast<unsigned>(others + layer), blocks, layer ? static_cast<unsigned>(up(a.pos_blocks, layer)) : 1);
}

struct Rank {
    const Order &o;
    Sums &a;
    hipStream_t stream;
    template <bool BF16, int LAYOUT, int L, int NV>
    void operator()(int blocks) const {
        const dim3 grid = pos_grid(a, o.blocks, kSortThreads / L, a.n ? blocks : 1);
        hipLaunchKernelGGL((embedding_rank_kernel<BF16, LAYOUT, L, NV>), grid, dim3(kSortThreads), kRankLds, stream, o, a);
    }
};

struct Sum {
    Sums &a;
    bool positions;
    hipStream_t stream;
    template <bool BF16, int LAYOUT, int L, int NV>
    void operator()(int blocks) const {
        const int64_t others = a.item_blocks + a.zero_blocks;
        const dim3 grid = positions ? pos_grid(a, others, kSumThreads / L, blocks) : dim3(static_cast<unsigned>(others), blocks);
        hipLaunchKernelGGL((embedding_sum_kernel<BF16, LAYOUT, L, NV>), grid, dim3(kSumThreads), 0, stream, a);
    }
};

struct Scan {
    Sums &a;
    hipStream_t stream;
    template <bool BF16, int LAYOUT, int L, int NV>
    void operator()(int blocks) const {
        const dim3 grid = pos_grid(a, a.zero_blocks, kSumThreads / L, blocks);
        hipLaunchKernelGGL((embedding_scan_kernel<BF16, LAYOUT, L, NV>), grid, dim3(kSumThreads), 0, stream, a);
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
    else if (nvec <= 128) YOSO_LOOKUP(32)
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

size_t embedding_backward_workspace(bool bf16, int64_t tokens, int64_t n, int64_t vocab, int d) {
    return layout_of(bf16, tokens, n, vocab, d).total;
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
    const Layout l = layout_of(bf16, a.tokens, a.n, a.vocab, a.d);
    const PosPlan plan = pos_plan(bf16, a.tokens, a.n, a.d);
    char *ws = static_cast<char *>(a.workspace);
    hipError_t e = hipSuccess;
    Sums s{};
    s.dy = a.dy;
    s.dtable = a.dtable;
    s.d = a.d;
    s.scale = a.scale;
    s.shift = l.shift;
    s.entries_log = l.entries_log;
    s.ids = a.ids;
    s.tokens = a.tokens;
    s.vocab = a.vocab;
    s.wide = wide;
    s.n = a.n;
    s.batch = a.n ? a.tokens / a.n : 0;
    s.parts = plan.parts;
    s.split = plan.split;
    s.dpos = a.dpos;
    s.pos_partial = reinterpret_cast<float *>(ws + l.pos);
    if (a.tokens <= kScanTokens) {
        s.range = static_cast<int>(up(a.vocab, 1024));  // (at most kScanRange)
        s.zero_blocks = up(a.vocab, s.range);
    } else {
        Order o{};
        o.ids = a.ids;
        o.wide = wide;
        o.tokens = a.tokens;
        o.vocab = a.vocab;
        o.shift = l.shift;
        o.buckets = static_cast<int>(l.buckets);
        o.blocks = static_cast<int>(l.blocks);
        o.entries_log = l.entries_log;
        o.block_tokens = l.block_tokens;
        o.counts = reinterpret_cast<uint16_t *>(ws + l.counts);
        o.rank = reinterpret_cast<uint16_t *>(ws + l.rank);
        o.entry = reinterpret_cast<uint2 *>(ws + l.entry);
        o.items = reinterpret_cast<uint4 *>(ws + l.items);
        o.multi = reinterpret_cast<uint4 *>(ws + l.multi);
        o.head = reinterpret_cast<uint32_t *>(ws + l.head);
        o.bucket = reinterpret_cast<uint32_t *>(ws + l.bucket);
        const bool one = l.blocks == 1;
        if (!one) {
            KernelTimer timer("embedding_rank_kernel", stream);
            const Rank run{o, s, stream};
            if ((e = with_layout<false>(bf16, a.d, run)) != hipSuccess) return e;
        }
        {
            KernelTimer timer("embedding_place_kernel", stream);
            auto *f = one ? embedding_place_kernel<true> : embedding_place_kernel<false>;
            const int64_t split = l.max_multi < kMaxBuckets ? l.max_multi : kMaxBuckets;
            const size_t lds = one ? kRankLds : static_cast<size_t>(split) * sizeof(Split);
            hipLaunchKernelGGL(f, dim3(static_cast<unsigned>(l.blocks + !one)), dim3(kSortThreads), lds, stream, o);
            if ((e = hipGetLastError()) != hipSuccess) return e;
        }
        s.entry = o.entry;
        s.items = o.items;
        s.multi = o.multi;
        s.head = o.head;
        s.bucket = o.bucket;
        s.present = reinterpret_cast<uint2 *>(ws + l.present);
        s.slot_rows = l.slot_rows;
        s.partial = reinterpret_cast<float *>(ws + l.partial);
        s.stride = l.stride;
        s.item_blocks = l.max_items;
        s.zero_blocks = l.buckets;
    }
    {
        KernelTimer timer("embedding_sum_kernel", stream);
        e = a.tokens <= kScanTokens ? with_layout<true>(bf16, a.d, Scan{s, stream})
                                    : with_layout<false>(bf16, a.d, Sum{s, l.blocks == 1, stream});
        if (e != hipSuccess) return e;
    }
    if (l.max_multi == 0 && s.parts == 1) return e;
    KernelTimer timer("embedding_join_kernel", stream);
    const int64_t items = (l.max_multi << (l.shift < 4 ? l.shift : 4)) * up(a.d, 256), join = items < 1024 ? items : 1024;
    const int64_t pos = s.parts > 1 ? up(a.n * a.d, kJoinThreads) : 0;
    auto *j = bf16 ? embedding_join_kernel<true> : embedding_join_kernel<false>;
    hipLaunchKernelGGL(j, dim3(static_cast<unsigned>(join + (pos < 512 ? pos : 512))), dim3(kJoinThreads), 0, stream, s,
                       static_cast<int>(join));
    return hipGetLastError();
}

}  // namespace yoso
