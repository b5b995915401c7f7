// The loss over a vocabulary at an encoder's output, and its gradient, without keeping the logits.
//
//   l[t][v] = scale (x_t . w_v + b_v),  lse_t = log sum_v exp l[t][v],  log q_k = l[t][i_k] - lse_t
//   loss_t  = sum_k p_k (log p_k - log q_k)
//
// with the ids i_k that token t is taught and their probabilities p: one id with p = 1 (cross entropy), or a
// teacher's top logits under a softmax (distillation).  Gradient: G[t][v] = dloss_t scale (q_v - sum_{i_k = v} p_k),
// dx = G W, dW = G^T X, db = sum_t G[t].
//
// Only tokens with a target take part: their numbers are listed first (list_kernel; count_kernel and rows_kernel), and
// everything after works on the listed rows, whose number only the device knows.  The products run on MFMA in
// 16 bits (loss_tiles.h).  x and the table are laid out first (lay_kernel) as fp16 planes, each row scaled by a power of
// two: for bf16 one plane holds a row exactly (values down to 2^-31 of its largest), for fp32 a pair of planes 22 bits (down to 2^-29).  The
// forward of up to some thousand bf16 tokens takes them as they lie (raw_rows), and few tokens have forms of their own.
//
// The backward makes the logits again, a piece of the vocabulary at a time, and keeps G of that piece as
// fp16 planes in the workspace, each value scaled as its row of x and of the table is:
//   Gs[t][v] = G[t][v] sx_t sw_v C,   x_t = sx_t xs_t,  w_v = sw_v ws_v,  C a power of two with |Gs| <= 2^14 (by a bound of |q - p|: largest_gradient)
// so that dx_t = (Gs ws) / (sx_t C) and dW_v = (Gs^T xs) / (sw_v C) come from the laid-out rows as they are.
#include <float.h>

#include "launch.h"
#include "loss_tiles.h"
#include "rows.h"
#include "timing.h"

namespace yoso {

namespace {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr int kThreads = 256;
constexpr int kCountTokens = 1024;  // tokens of a workgroup of count_kernel and rows_kernel
constexpr int kFewTokens = 64;      // up to so many tokens the forward reads the table where it lies
constexpr int kFewEntries = 1024;   // ids that a workgroup of the forms for few tokens holds
constexpr int kFewBlocks = 2048, kLayBlocks = 2048;
constexpr int kSlots = 512;         // workgroups of the logits that run at once (two on a CU)
constexpr int kGradSlots = 512;     // of the gradients' products
constexpr int kGradM = 128;         // columns of d of their tiles
constexpr int grad_n(bool bf16) { return bf16 ? 256 : 128; }
constexpr int kMaxTop = 1024;
constexpr int kSortedTop = 64;      // ids of a token that are sorted, for their logits to be taken from the tiles
constexpr int kNoId = 0x7FFFFFFF;
constexpr int kTileN = 128;         // tokens of a tile of the logits

// What the device tells later launches.  A maximum is spread over kMaxima values a cache line apart: thousands of
// atomics on one address take 12 ns each, one after the other.
constexpr int kMaxima = 64, kMaximaStride = 32;
enum : int { kMaxF = 0, kMaxDl = 1, kMaxSw = 2 };  // |dloss scale sx| times the bound of |q - p|, |dloss scale|, sw

struct Meta {
    int count;  // tokens that take part
    uint32_t maxima[kMaxima * kMaximaStride];  // bits of the three maxima, side by side

    __device__ __forceinline__ void raise(int which, float x) {
        atomicMax(&maxima[(blockIdx.x & (kMaxima - 1)) * kMaximaStride + which], __float_as_uint(x));
    }
    // every lane of the wave gets it
    __device__ __forceinline__ float largest(int which) const {
        static_assert(kMaxima == 64, "a lane each");
        return wave_max(__uint_as_float(maxima[(threadIdx.x & 63) * kMaximaStride + which]));
    }
};

// The scales that G carries.  A row of zeros has none of its own (sx, sw = 0): of the table it takes the largest, of x
// what brings its dloss up to the largest |dloss sx (q - p)|, so that its gradients are as exact as any row's.
struct Scales {
    float max_sw, max_f;
    __device__ __forceinline__ explicit Scales(const Meta *meta) {
        max_sw = meta->largest(kMaxSw);
        max_f = meta->largest(kMaxF);
        max_sw = max_sw > 0.f ? max_sw : 1.f;
        max_f = max_f > 0.f ? max_f : 1.f;
    }
    __device__ __forceinline__ float table(float sw) const { return sw != 0.f ? sw : max_sw; }
    __device__ __forceinline__ float row(float sx, float dl) const {
        if (sx != 0.f || dl == 0.f) return sx != 0.f ? sx : 1.f;
        int e = 0;
        frexpf(max_f / fabsf(dl), &e);  // 2^(e - 1) |dl| <= max_f
        return ldexpf(1.f, min(max(e - 1, -100), 100));
    }
    // Gs = G sx sw C with C = up() / max_sw
    __device__ __forceinline__ float up() const { return ldexpf(1.f, 14 - scale_exp(max_f)); }
    __device__ __forceinline__ float down() const { return ldexpf(1.f, scale_exp(max_f) - 14); }
};

// What a token is taught.
struct Taught {
    const void *ids;
    bool wide;
    int top;
    const float *teacher;  // NULL: cross entropy
    const float *dloss;    // NULL: forward
    int64_t tokens, vocab;

    __device__ __forceinline__ int64_t id(int64_t t, int k) const {
        const int64_t at = t * top + k;
        return wide ? static_cast<const int64_t *>(ids)[at] : static_cast<const int32_t *>(ids)[at];
    }
    __device__ __forceinline__ bool named(int64_t t, int k) const {
        const int64_t v = id(t, k);
        return v >= 0 && v < vocab && (teacher == nullptr || teacher[t * top + k] != -INFINITY);
    }
    __device__ __forceinline__ bool takes_part(int64_t t) const {
        if (t >= tokens || (dloss != nullptr && dloss[t] == 0.f)) return false;
        if (top == 1) return named(t, 0);
        for (int k = 0; k < top; k += 4) {  // (four loads together)
            bool in[4], any = false;
#pragma unroll
            for (int i = 0; i < 4; i++) {
                const int64_t v = id(t, k + i < top ? k + i : top - 1);
                in[i] = v >= 0 && v < vocab;
                any |= in[i];
            }
            if (any && teacher != nullptr) {
                float logit[4];
#pragma unroll
                for (int i = 0; i < 4; i++) logit[i] = teacher[t * top + (k + i < top ? k + i : top - 1)];
                any = false;
#pragma unroll
                for (int i = 0; i < 4; i++) any |= in[i] && logit[i] != -INFINITY;
            }
            if (any) return true;
        }
        return false;
    }
};

// xcd_remap for counts below 2^31
__device__ __forceinline__ int xcd_remap32(uint32_t id, int n) {
    const int q = n >> 3, r = n & 7, x = id & 7, i = id >> 3;
    return x * q + (x < r ? x : r) + i;
}

__device__ __forceinline__ float wave_sum(float x) { return group_sum(x, 64); }

__host__ __device__ constexpr int64_t up(int64_t n, int64_t to) { return (n + to - 1) / to * to; }

// ---------------------------------------------------------------- which tokens take part

__global__ __launch_bounds__(kThreads) void count_kernel(Taught a, int *counts, uint64_t *masks, Meta *meta) {
    __shared__ int part[4];
    const int wave = threadIdx.x >> 6;
    int n = 0;
    for (int j = 0; j < kCountTokens / kThreads; j++) {
        const int64_t t = static_cast<int64_t>(blockIdx.x) * kCountTokens + j * kThreads + threadIdx.x;
        const uint64_t m = __ballot(a.takes_part(t));
        n += __popcll(m);
        if ((threadIdx.x & 63) == 0) masks[t >> 6] = m;
    }
    if ((threadIdx.x & 63) == 0) part[wave] = n;
    __syncthreads();
    if (threadIdx.x == 0) {
        counts[blockIdx.x] = part[0] + part[1] + part[2] + part[3];
        if (blockIdx.x == 0) meta->count = 0;
    }
    if (blockIdx.x == 0)
        for (int i = threadIdx.x; i < kMaxima * kMaximaStride; i += kThreads) meta->maxima[i] = 0;
}

// count_kernel and rows_kernel in one launch of one workgroup, for few tokens
constexpr int kListThreads = 1024;
constexpr int64_t kListTokens = 8 * kListThreads;

__global__ __launch_bounds__(kListThreads) void list_kernel(Taught a, Meta *meta, int *rows, int *place, float *loss, float *lse,
                                                            float *logq) {
    __shared__ int wave_n[kListThreads / 64];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    for (int i = threadIdx.x; i < kMaxima * kMaximaStride; i += kListThreads) meta->maxima[i] = 0;
    // the first ids of the thread's tokens together, the others' one after the other
    constexpr int EACH = static_cast<int>(kListTokens / kListThreads);
    bool first[EACH];
#pragma unroll
    for (int i = 0; i < EACH; i++) {
        const int64_t t = i * kListThreads + threadIdx.x;
        first[i] = t < a.tokens && (a.dloss == nullptr || a.dloss[t] != 0.f) && a.named(t, 0);
    }
    int at = 0;
#pragma unroll
    for (int i = 0; i < EACH; i++) {
        const int64_t t = i * kListThreads + threadIdx.x;
        if (i * kListThreads >= a.tokens) break;
        const bool in = first[i] || (a.top > 1 && a.takes_part(t));
        const uint64_t m = __ballot(in);
        if (lane == 0) wave_n[wave] = __popcll(m);
        __syncthreads();
        int r = at + __popcll(m & ((uint64_t{1} << lane) - 1));
        for (int w = 0; w < kListThreads / 64; w++) {
            if (w < wave) r += wave_n[w];
            at += wave_n[w];
        }
        __syncthreads();
        if (in) rows[r] = static_cast<int>(t);
        if (t < a.tokens) {
            if (place) place[t] = in ? r : -1;
            if (!in && loss) {
                loss[t] = lse[t] = 0.f;
                if (logq)
                    for (int k = 0; k < a.top; k++) logq[t * a.top + k] = 0.f;
            }
        }
    }
    if (threadIdx.x == 0) meta->count = at;
}

// rows[r] = token of row r, in order; place[t] = row of token t or -1 (backward); the outputs of the others (forward).
__global__ __launch_bounds__(kThreads) void rows_kernel(Taught a, const int *counts, const uint64_t *masks, Meta *meta, int *rows, int *place, float *loss,
                                                        float *lse, float *logq) {
    __shared__ int part[4], wave_n[4];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    int before = 0;
    for (int b = threadIdx.x; b < static_cast<int>(blockIdx.x); b += kThreads) before += counts[b];
    for (int s = 32; s > 0; s >>= 1) before += __shfl_xor(before, s);
    if (lane == 0) part[wave] = before;
    __syncthreads();
    int at = part[0] + part[1] + part[2] + part[3];
    for (int j = 0; j < kCountTokens / kThreads; j++) {
        const int64_t t = static_cast<int64_t>(blockIdx.x) * kCountTokens + j * kThreads + threadIdx.x;
        const uint64_t m = masks[t >> 6];
        const bool in = m >> lane & 1;
        if (lane == 0) wave_n[wave] = __popcll(m);
        __syncthreads();
        int r = at + __popcll(m & ((uint64_t{1} << lane) - 1));
        for (int w = 0; w < wave; w++) r += wave_n[w];
        at += wave_n[0] + wave_n[1] + wave_n[2] + wave_n[3];
        __syncthreads();
        if (in) rows[r] = static_cast<int>(t);
        if (t < a.tokens) {
            if (place) place[t] = in ? r : -1;
            if (!in && loss) {
                loss[t] = lse[t] = 0.f;
                if (logq)
                    for (int k = 0; k < a.top; k++) logq[t * a.top + k] = 0.f;
            }
        }
    }
    if (blockIdx.x == gridDim.x - 1 && threadIdx.x == 0) meta->count = at;
}

// ---------------------------------------------------------------- rows as fp16 planes

// 8 values of a row from column c, 0 behind its end
template <bool BF16>
__device__ __forceinline__ void row8(const void *base, int64_t row, int c, int d, float (&v)[8]) {
    if (c + 8 <= d) {
        if constexpr (BF16) {
            const raw4 w = *reinterpret_cast<const raw4_any *>(static_cast<const uint16_t *>(base) + row + c);
#pragma unroll
            for (int j = 0; j < 8; j++) v[j] = value<true>(w, j);
        } else {
            const float *p = static_cast<const float *>(base) + row + c;
            const float4_any a = *reinterpret_cast<const float4_any *>(p), b = *reinterpret_cast<const float4_any *>(p + 4);
#pragma unroll
            for (int j = 0; j < 4; j++) v[j] = a[j], v[4 + j] = b[j];
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; j++) v[j] = c + j < d ? load1<BF16>(base, row + c + j) : 0.f;
    }
}

// db's sums of dloss scale p at the taught ids, in units of 2^-40 of the power of two above max_dl (integers, so that the
// order of the atomics does not matter), as some copies, for the waves to be spread over: atomics on one cache line take 11 ns
// each, one after the other (53012 x 6 ids of 97: pick_kernel 525 us with one copy, 27 with 64).
struct Picked {
    unsigned long long *sums;  // [copies][ld]; NULL: no db, or no teacher
    int64_t ld;
    int copies;  // a power of two
};
int64_t picked_ld(int64_t vocab) { return up(vocab, 16); }
// at most 64, in 2 MiB
int picked_copies(int64_t vocab) {
    int n = 64;
    while (n > 1 && n * picked_ld(vocab) > 1 << 18) n >>= 1;
    return n;
}

struct Lay {
    const void *src;
    int64_t n, padded;  // rows of the source (x: at most), rows written
    int d, ld;
    half8 *hi, *lo;     // planes of blocks of 32 columns, [ld / 32][padded][32]
    float *mult;        // source value = laid-out value times mult; 0: a row of zeros
    // x: the rows listed, and what the backward multiplies G by
    const int *rows;
    const float *dloss, *lse;
    const float *logq;  // cross entropy: the loss
    Taught taught;
    float scale;
    float *dls, *lse2;
    Meta *meta;
    bool table;
    Picked picked;  // table: cleared for pick_kernel

    __device__ __forceinline__ int64_t at(int64_t r, int c) const { return ((c >> 5) * padded + r) * 4 + ((c >> 3) & 3); }
};

// maximum over aligned groups of L lanes (16, 32 or 64)
template <int L>
__device__ __forceinline__ uint32_t group_max(uint32_t x) {
#pragma unroll
    for (int s = 1; s < L; s <<= 1) x = max(x, static_cast<uint32_t>(__shfl_xor(static_cast<int>(x), s)));
    return x;
}

template <int L>
__device__ __forceinline__ float group_max(float x) {
#pragma unroll
    for (int s = 1; s < L; s <<= 1) x = fmaxf(x, __shfl_xor(x, s));
    return x;
}

// A bound of |q - p| over the vocabulary (q the student's, p the teacher's probabilities) for token t, by L lanes: small where both are
// sure of one id.  With a the id of the largest q that is listed, every other entry has q <= 1 - q_a and p <= 1 - p_a, and q_a - p_a is the
// difference of those two.  1 - q_a comes from log q, 1 - p_a is a sum without a's entries, however often a is listed.
template <int L>
__device__ __forceinline__ float largest_gradient(const Taught &s, const float *logq, float scale, int64_t t, int lane) {
    float top = -INFINITY, best = -INFINITY;
    int a = -1;
    // (loads of several ids together)
#pragma unroll 4
    for (int k = lane; k < s.top; k += L) {
        const int64_t v = s.id(t, k);
        const float logit = s.teacher[t * s.top + k], lq = logq[t * s.top + k];
        const bool named = v >= 0 && v < s.vocab && logit != -INFINITY;
        top = named ? fmaxf(top, logit) : top;
        if (named && lq > best) best = lq, a = static_cast<int>(v);
    }
    top = group_max<L>(top);
#pragma unroll
    for (int step = 1; step < L; step <<= 1) {
        const float other = __shfl_xor(best, step);
        const int b = __shfl_xor(a, step);
        if (other > best || (other == best && b > a)) best = other, a = b;
    }
    float sum = 0.f, rest = 0.f;
#pragma unroll 4
    for (int k = lane; k < s.top; k += L) {
        const int64_t v = s.id(t, k);
        const float logit = s.teacher[t * s.top + k];
        const float e = v >= 0 && v < s.vocab && logit != -INFINITY ? exp2f((logit - top) * (scale * kLog2e)) : 0.f;
        sum += e;
        rest += v != a ? e : 0.f;
    }
    return fmaxf(-expm1f(best), group_sum(rest, L) / group_sum(sum, L));
}

// Bound by its bytes: 30000 x 768 fp32 read and written in 39 us (4.7 TB/s).  L lanes a row.  Values lie below 2^15.  Rows of up to 2048 values (L < 64: 8 L) stay in registers
// between their maximum and the planes.
template <bool BF16, int L>
__device__ __forceinline__ void lay_rows(const Lay &a, int block, int blocks) {
    constexpr int KEEP = L == 64 ? 4 : 1;
    __shared__ float most[4][3];
    const int lane = threadIdx.x & (L - 1), group = threadIdx.x / L;
    const int64_t n = a.table ? a.n : a.meta->count, rows = a.table ? a.padded : up(n, 128);
    float max_sw = 0.f, max_f = 0.f, max_dl = 0.f;
    for (int64_t r = static_cast<int64_t>(block) * (kThreads / L) + group; r < rows; r += static_cast<int64_t>(blocks) * (kThreads / L)) {
        const bool real = r < n;
        const int64_t t = !real ? 0 : a.rows ? a.rows[r] : r;
        const bool gives = !a.table && a.dloss != nullptr && real;  // a token of the backward
        const float dloss = gives ? a.dloss[t] : 0.f, lse = gives ? a.lse[t] : 0.f;
        const float loss = gives && a.taught.teacher == nullptr ? a.logq[t] : 0.f;
        float kept[KEEP][8];
        uint32_t bits = 0;  // of the row's largest magnitude; an infinity's or a NaN's are larger than any number's
#pragma unroll
        for (int i = 0; i < KEEP; i++) {
            const int c = lane * 8 + i * (8 * L);
            if (real && c < a.d) {
                row8<BF16>(a.src, t * a.d, c, a.d, kept[i]);
            } else {
#pragma unroll
                for (int j = 0; j < 8; j++) kept[i][j] = 0.f;
            }
        }
#pragma unroll
        for (int i = 0; i < KEEP; i++)
#pragma unroll
            for (int j = 0; j < 8; j++) bits = max(bits, __float_as_uint(kept[i][j]) & 0x7FFFFFFFu);
        if (real)
            for (int c = lane * 8 + KEEP * 8 * L; c < a.d; c += 8 * L) {
                float v[8];
                row8<BF16>(a.src, t * a.d, c, a.d, v);
#pragma unroll
                for (int j = 0; j < 8; j++) bits = max(bits, __float_as_uint(v[j]) & 0x7FFFFFFFu);
            }
        bits = group_max<L>(bits);
        const bool finite = bits < 0x7F800000u;
        const float big = finite ? __uint_as_float(bits) : FLT_MAX;
        const int e = scale_exp(big);
        const float up_by = ldexpf(1.f, 15 - e), mult = big > 0.f ? ldexpf(1.f, e - 15) : 0.f;
#pragma unroll
        for (int i = 0; i < KEEP; i++) {
            const int c = lane * 8 + i * (8 * L);
            if (c < a.ld) {
                half8 hi, lo;
                pairs(kept[i], up_by, hi, lo);
                a.hi[a.at(r, c)] = hi;
                if constexpr (!BF16) a.lo[a.at(r, c)] = lo;
            }
        }
        for (int c = lane * 8 + KEEP * 8 * L; c < a.ld; c += 8 * L) {
            float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
            if (real && c < a.d) row8<BF16>(a.src, t * a.d, c, a.d, v);
            half8 hi, lo;
            pairs(v, up_by, hi, lo);
            a.hi[a.at(r, c)] = hi;
            if constexpr (!BF16) a.lo[a.at(r, c)] = lo;
        }
        if (lane == 0) a.mult[r] = mult;
        if (a.table) {
            if (finite) max_sw = fmaxf(max_sw, mult);
            if (real && a.picked.sums)
                for (int c = lane; c < a.picked.copies; c += L) a.picked.sums[c * a.picked.ld + r] = 0;
        } else if (a.dloss) {
            const float dl = dloss * a.scale;
            // A bound of |q - p|, of which G is made: of cross entropy 1 - q of the target.  The forward's sum of exponentials
            // loses what is added to a sum near 1 in steps below 2^-25, 2^11 of them at most (a quarter of 2^20 / 128 tiles): 2^-12 is added.
            const float most = !real ? 0.f : a.taught.teacher ? largest_gradient<L>(a.taught, a.logq, a.scale, t, lane) : -expm1f(-loss);
            // (1 for what is no number)
            const float f = dl * mult * (most <= 1.f ? fminf(most + 0x1p-12f, 1.f) : 1.f);
            if (lane == 0) {
                a.dls[r] = dl;
                // (+inf is the mark of a padding row below: logits that reach it have no gradient)
                const float lse2 = lse * kLog2e;
                a.lse2[r] = lse2 == INFINITY ? NAN : lse2;
            }
            // (a row that holds no numbers, or whose logits are none, has no gradient: it must not scale the others' away)
            if (finite && fabsf(lse) <= FLT_MAX && fabsf(f) <= FLT_MAX) {
                max_f = fmaxf(max_f, fabsf(f));
                max_dl = fmaxf(max_dl, fabsf(dl));
            }
        }
    }
    if (!a.table && !a.dloss) return;
    max_f = wave_max(max_f), max_dl = wave_max(max_dl), max_sw = wave_max(max_sw);
    if ((threadIdx.x & 63) == 0) {
        float *w = most[threadIdx.x >> 6];
        w[kMaxF] = max_f, w[kMaxDl] = max_dl, w[kMaxSw] = max_sw;
    }
    __syncthreads();
    if (threadIdx.x < 3 && (threadIdx.x == kMaxSw) == a.table) {
        const float m = fmaxf(fmaxf(most[0][threadIdx.x], most[1][threadIdx.x]), fmaxf(most[2][threadIdx.x], most[3][threadIdx.x]));
        if (m > 0.f) a.meta->raise(threadIdx.x, m);
    }
}

// the table by the first workgroups, x by the others
template <bool BF16, int L>
__global__ __launch_bounds__(kThreads) void lay_kernel(Lay table, Lay x, int table_blocks) {
    const int block = blockIdx.x;
    if (block < table_blocks)
        lay_rows<BF16, L>(table, block, table_blocks);
    else
        lay_rows<BF16, L>(x, block - table_blocks, gridDim.x - table_blocks);
}

// ---------------------------------------------------------------- logits, a tile at a time

struct Logits {
    // table rows (M) and token rows (N), as planes of so many rows or as they lie
    const char *w[2], *x[2];
    int64_t w_rows, x_rows;
    const float *sw, *sx;  // NULL: as they lie
    const int *rows;       // token of a row
    int64_t ld;            // as they lie: bytes of a row
    int64_t d;
    const float *bias;
    float scale;
    int64_t vocab, v0, v1;  // the piece's first entry and its end
    const Meta *meta;
    float2 *part;  // forward: maximum and sum of each row over each part of the vocabulary, [part][token tiles TN]
    float *hit;    // forward of cross entropy: log2 e times the target's logit of each row
    // forward of distillation: each row's 64 id + k in order, ended by kNoId, and where log2 e times their logits go
    const int *sorted;
    int sorted_ld;
    float *picks;  // [tokens][top]
    // backward
    const float *dls, *lse2;
    Taught taught;
    const float *loss;  // cross entropy: the target's probability is exp(-loss); NULL: pick_kernel writes G at the taught ids
    _Float16 *g[2];  // planes, [piece / 32][x_rows][32]
    int64_t piece;
    float *db;  // the piece's sums over half a token tile, [2 token tiles][piece]
};

// Parts that the vocabulary's `tiles` tiles are cut into for `rows` token tiles: as few as make the rounds of kSlots
// workgroups, times the tiles of a part, least, but four (an XCD's 64 workgroups then read 16 token tiles and 4 table
// tiles at a time, which its L2 holds; with one part they read 64 token tiles).  Every lane of a wave gets it.
__device__ __forceinline__ int vocab_parts(int rows, int tiles) {
    const int from = tiles < 4 ? tiles : 4;
    uint32_t least = 0xFFFFFFFFu;
    for (int i = 0; i < 16 && (i == 0 || rows * (64 * i + 1) <= 2 * kSlots); i++) {
        const int s = (threadIdx.x & 63) + 1 + 64 * i;
        if (s >= from && s <= tiles && (s == from || rows * s <= 2 * kSlots)) {
            const uint32_t t = static_cast<uint32_t>((rows * s + kSlots - 1) / kSlots) * ((tiles + s - 1) / s) << 10 | (s - 1);
            least = t < least ? t : least;
        }
    }
#pragma unroll
    for (int s = 32; s > 0; s >>= 1) {
        const uint32_t o = __shfl_xor(least, s);
        least = o < least ? o : least;
    }
    return __builtin_amdgcn_readfirstlane(static_cast<int>(least & 1023)) + 1;
}

__device__ __forceinline__ float swap_halves(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return (threadIdx.x & 32) ? __uint_as_float(r[0]) : __uint_as_float(r[1]);
}

__device__ __forceinline__ float log2_of_power(float x) { return static_cast<float>(static_cast<int>(__float_as_uint(x) >> 23) - 127); }

// Lower half: its a and the upper half's a; upper half: the lower half's b and its b.
__device__ __forceinline__ uint4 exchange(uint2 a, uint2 b) {
    const auto x = __builtin_amdgcn_permlane32_swap(a.x, b.x, false, false);
    const auto y = __builtin_amdgcn_permlane32_swap(a.y, b.y, false, false);
    return make_uint4(x[0], y[0], x[1], y[1]);
}

// (m, l) of two disjoint sets: maximum, and sum of 2^(value - maximum) (0 where the maximum is -inf)
__device__ __forceinline__ void join(float &m, float &l, float m2, float l2) {
    const float top = fmaxf(m, m2), at = top == -INFINITY ? 0.f : top;
    l = l * exp2f(m - at) + l2 * exp2f(m2 - at);
    m = top;
}

// log q of the entry whose logit is x (times log2 e): against the maximum before the sum's logarithm, so that a token
// whose probability is near 1 keeps its loss (lse rounded first, it would be off by a step of lse)
__device__ __forceinline__ float log_q(float x, float m, float l) {
#pragma clang fp contract(off)
    const float above = x - m;
    return (above - log2f(l)) * kLn2;
}

// scale log2 e times entry v's bias; -inf takes the entry out whatever the sign of the scale
__device__ __forceinline__ float bias_of(const float *bias, int64_t v, float scale) {
    const float b = bias ? bias[v] : 0.f;
    return b == -INFINITY ? b : b * scale * kLog2e;
}

// The logit x of a taught id (times log2 e) where it may be a dot product of its own, beside m and l of the tiles.  Where
// the token is sure (l < 1.5: every entry but the largest lies below m - 1) an x this near m is the largest entry's, whose logit is m: x's own
// roundings, 1e-6 of its products, would be all that log q holds and give it either sign.  (Elsewhere |log q| > 0.4.)
__device__ __forceinline__ float settled(float x, float m, float l) { return l < 1.5f && x > m - 0.5f ? m : x; }

template <bool V>
struct Bool {
    static constexpr bool value = V;
};

// A workgroup has one token tile and, forward, a part of the vocabulary, whose tiles it goes through with each token's running
// maximum and sum in registers: a lane holds 16 entries of one token for each block, so both are taken within the
// lane and joined over two lanes and two waves at the end alone.  Bound by the matrix units (51% busy at 1.96 GHz) and the card's power: 16384 x 768
// into 30000, passes in a row, bf16 724 us forward (1.04 PFLOP/s; 40 less with the exponentials left out) and 839 with G, fp32 pairs 2110 with sorted
// ids and 2330 with G (1.08 and 0.97 of fp16 products).  (Behind a pause or other products the clock is lower for some tens of ms: bf16 up to 890.)
// MODE 0: maximum and sum; 3: and the logits of the sorted ids; 1: G; 2: G and its sums over the tile's tokens.  RAW:
// operands as they lie (bf16).
template <int PL, int MODE, bool RAW>
__global__ __launch_bounds__(kThreads, 2) void logits_kernel(Logits a) {
    constexpr bool FORWARD = MODE == 0 || MODE == 3, SORTED = MODE == 3;
    typedef Product<PL, PL == 1 ? 256 : 128, 128, false, false, RAW> P;
    constexpr int TM = P::TM, TN = P::TN, IM = P::IM, IN = P::IN;
    __shared__ __align__(1024) char stage[P::kLds];
    __shared__ float4 vocab_at[2][TM / 4];  // multiplier, bias
    const uint32_t lds = lds_address(stage);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wm = wave & 1, wn = wave >> 1;
    const int count = a.meta->count;
    const int row_tiles = (count + TN - 1) / TN, tiles = static_cast<int>((a.v1 - a.v0 + TM - 1) / TM);
    int tt, first, last, part = 0;
    if constexpr (FORWARD) {
        const int parts = vocab_parts(row_tiles, tiles), all = row_tiles * parts;
        if (static_cast<int>(blockIdx.x) >= all) return;
        // 16 token tiles (or all) of a part side by side, then the next part: an XCD's workgroups share their table tiles
        const int id = xcd_remap32(blockIdx.x, all), per = (tiles + parts - 1) / parts;
        const int wide = row_tiles < 16 ? row_tiles : 16, band = id / (wide * parts), in = id - band * wide * parts;
        const int high = row_tiles - band * wide < wide ? row_tiles - band * wide : wide;
        part = in / high;
        tt = band * wide + (in - part * high);
        first = part * per;
        last = first + per < tiles ? first + per : tiles;
    } else {
        // a workgroup a tile: one that ends does not wait for its stores, as the next tile's products would (loads and
        // stores share a counter).  Patches of eight token tiles: neighbours share table tiles in their L2
        const int all = row_tiles * tiles;
        if (static_cast<int>(blockIdx.x) >= all) return;
        const int id = xcd_remap32(blockIdx.x, all);
        const int band = id / (8 * tiles), in = id - band * 8 * tiles;
        const int high = row_tiles - band * 8 < 8 ? row_tiles - band * 8 : 8;
        first = in / high;
        tt = band * 8 + (in - first * high);
        last = first + 1;
    }

    typename P::A oa;
    typename P::B ob;
    const int64_t row0 = static_cast<int64_t>(tt) * TN;
    if constexpr (RAW) {
        ob.base[0] = a.x[0];
        ob.by_row([&](int r) {
            const int64_t at = row0 + r < count ? row0 + r : count - 1;
            return static_cast<uint32_t>(a.rows[at] * a.ld);
        });
    } else {
#pragma unroll
        for (int p = 0; p < PL; p++) ob.laid(p, a.x[p], a.x_rows, row0, 0);
    }
    const int64_t steps = (a.d + kStepK - 1) / kStepK;

    const Scales scales(a.meta);
    const float max_sw = scales.max_sw, cf = scales.up();
    float by_row[IN], m[IN], l[IN], f[IN], lse2[IN], dl[IN], less[IN];
    int64_t to[IN];
    int target[IN], left[IN];
    int4 coming[IN];  // the next ids of the lane's tokens
    const int4 *list[IN];
    float *row_picks[IN];
#pragma unroll
    for (int j = 0; j < IN; j++) {
        const int64_t r = row0 + wn * (TN / 2) + j * 32 + (lane & 31);
        by_row[j] = a.scale * kLog2e * (RAW ? 1.f : a.sx[r]);
        m[j] = -INFINITY;
        l[j] = 0.f;
    }

    if constexpr (!FORWARD)
#pragma unroll
        for (int j = 0; j < IN; j++) {
            const int64_t r = row0 + wn * (TN / 2) + j * 32 + (lane & 31);
            const bool real = r < count;
            f[j] = real ? a.dls[r] * scales.row(a.sx[r], a.dls[r]) * cf : 0.f;
            lse2[j] = real ? a.lse2[r] : INFINITY;
            dl[j] = MODE == 2 && real ? a.dls[r] : 0.f;
            to[j] = r * 32 + 8 * (lane >> 5);
            target[j] = -1;
            less[j] = 0.f;
            if (a.loss && real) {
                const int64_t t = a.rows[r];
                target[j] = static_cast<int>(a.taught.id(t, 0));
                less[j] = expm1f(-a.loss[t]) / max_sw;  // q - 1 there, times 1 / max_sw
            }
        }
    if constexpr (FORWARD)
#pragma unroll
        for (int j = 0; j < IN; j++) {
            const int64_t r = row0 + wn * (TN / 2) + j * 32 + (lane & 31);
            target[j] = a.hit && r < count ? static_cast<int>(a.taught.id(a.rows[r], 0)) : -1;
            coming[j] = make_int4(kNoId, kNoId, kNoId, kNoId);
            left[j] = 4;
            if (SORTED && r < count) {
                list[j] = reinterpret_cast<const int4 *>(a.sorted + r * a.sorted_ld);
                coming[j] = *list[j];
                row_picks[j] = a.picks + static_cast<int64_t>(a.rows[r]) * a.taught.top;
            }
        }
    const auto table_tile = [&](int tile) {
        const int64_t v0 = a.v0 + static_cast<int64_t>(tile) * TM;
        if constexpr (RAW) {
            oa.base[0] = a.w[0] + v0 * a.ld;
            oa.by_row([&](int r) {
                const int64_t at = v0 + r < a.vocab ? r : static_cast<int>(a.vocab - 1 - v0);
                return static_cast<uint32_t>(at * a.ld);
            });
        } else {
#pragma unroll
            for (int p = 0; p < PL; p++) oa.laid(p, a.w[p], a.w_rows, v0, 0);
        }
    };
    if (first < last) {
        table_tile(first);
        P::begin(oa, ob, steps, lds);
    }
    for (int tile = first; tile < last; tile++) {
        const int64_t v0 = a.v0 + static_cast<int64_t>(tile) * TM;
        // the tile's entries: multiplier and bias (they arrive during the products)
        const int64_t ve = v0 + threadIdx.x;
        const bool in = ve < a.vocab && threadIdx.x < TM;
        float e_sw = !RAW && in ? a.sw[ve] : 0.f;
        if (!FORWARD && in) e_sw = scales.table(e_sw);
        const float e_bias = !in ? -INFINITY : bias_of(a.bias, ve, a.scale);
        floatx16 acc[IM][IN];
#pragma unroll
        for (int i = 0; i < IM; i++)
#pragma unroll
            for (int j = 0; j < IN; j++)
#pragma unroll
                for (int k = 0; k < 16; k++) acc[i][j][k] = 0.f;
        P::run(oa, ob, steps, lds, acc);
        if (threadIdx.x < TM) {
            float *at = reinterpret_cast<float *>(vocab_at);
            if constexpr (!RAW) at[threadIdx.x] = e_sw;
            // (backward: 2^x comes out times sw / max_sw, a power of two)
            at[TM + threadIdx.x] = !FORWARD && in ? e_bias + log2_of_power(e_sw / max_sw) : e_bias;
        }
        __syncthreads();
        // every wave has read the last step: the next tile's first steps come in while this one is finished
        if (tile + 1 < last) {
            table_tile(tile + 1);
            P::begin(oa, ob, steps, lds);
        }

        // the lane's token is a column of the tile, its entries 8 (k / 4) + 4 (lane / 32) + k % 4 of each block
        const int v_first = wm * (TM / 2) + 4 * (lane >> 5);
        if constexpr (FORWARD) {
            float top[IN];
#pragma unroll
            for (int j = 0; j < IN; j++) top[j] = -INFINITY;
#pragma unroll
            for (int i = 0; i < IM; i++) {
#pragma unroll
                for (int q = 0; q < 4; q++) {
                    const int at = (v_first + i * 32 + q * 8) >> 2;
                    const float4 b = vocab_at[1][at], s = RAW ? b : vocab_at[0][at];
                    const float bs[4] = {b.x, b.y, b.z, b.w}, ss[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
                    for (int j = 0; j < IN; j++)
#pragma unroll
                        for (int k = 0; k < 4; k++) {
                            float x = acc[i][j][q * 4 + k];
                            x = RAW ? fmaf(x, by_row[j], bs[k]) : fmaf(x * by_row[j], ss[k], bs[k]);
                            acc[i][j][q * 4 + k] = x;
                            top[j] = fmaxf(top[j], x);
                        }
                }
                if (!SORTED && a.hit) {
                    const int at_block = static_cast<int>(v0) + wm * (TM / 2) + i * 32;
                    bool mine = false;
#pragma unroll
                    for (int j = 0; j < IN; j++) mine |= static_cast<unsigned>(target[j] - at_block) < 32u;
                    if (__ballot(mine) != 0) {
#pragma unroll
                        for (int j = 0; j < IN; j++)
#pragma unroll
                            for (int k = 0; k < 16; k++)
                                if (target[j] == static_cast<int>(v0) + v_first + i * 32 + (k >> 2) * 8 + (k & 3))
                                    a.hit[row0 + wn * (TN / 2) + j * 32 + (lane & 31)] = acc[i][j][k];
                    }
                }
                if constexpr (SORTED) {
                    const int at_block = static_cast<int>(v0) + wm * (TM / 2) + i * 32;
#pragma unroll
                    for (int j = 0; j < IN; j++)
                        while (__ballot((coming[j].x >> 6) < at_block + 32) != 0) {
                            const int id = coming[j].x >> 6, o = id - at_block;
                            if (o < 32) {
                                if (o >= 0 && (o >> 2 & 1) == lane >> 5) {
                                    const int e = (o >> 3) * 4 + (o & 3);
                                    float x = acc[i][j][0];
#pragma unroll
                                    for (int k = 1; k < 16; k++) x = e == k ? acc[i][j][k] : x;
                                    row_picks[j][coming[j].x & 63] = x;
                                }
                                coming[j].x = coming[j].y, coming[j].y = coming[j].z, coming[j].z = coming[j].w;
                                if (--left[j] == 0) {
                                    coming[j] = *++list[j];
                                    left[j] = 4;
                                }
                            }
                        }
                }
                __builtin_amdgcn_sched_barrier(0);  // (reads of later blocks ahead of these would cost registers)
            }
#pragma unroll
            for (int j = 0; j < IN; j++) {
                const float at = top[j] == -INFINITY ? 0.f : top[j];
                float sum = 0.f;
#pragma unroll
                for (int i = 0; i < IM; i++)
#pragma unroll
                    for (int k = 0; k < 16; k++) sum += __builtin_amdgcn_exp2f(acc[i][j][k] - at);
                join(m[j], l[j], top[j], sum);
            }
        } else {
#pragma unroll
            for (int i = 0; i < IM; i++) {
                const int64_t block = ((v0 - a.v0 + wm * (TM / 2) + i * 32) >> 5) * a.x_rows * 32;
                const int at_block = static_cast<int>(v0) + wm * (TM / 2) + i * 32;
                bool mine = false;
#pragma unroll
                for (int j = 0; j < IN; j++) mine |= static_cast<unsigned>(target[j] - at_block) < 32u;
                const bool some = __ballot(mine) != 0;  // a target of these tokens lies in the block
                float sums[16];
                const auto values = [&](auto targets) {
#pragma unroll
                    for (int q2 = 0; q2 < 2; q2++) {
                        uint2 hi[2][IN], lo[2][IN];
#pragma unroll
                        for (int h = 0; h < 2; h++) {
                            const int q = q2 * 2 + h, at = (v_first + i * 32 + q * 8) >> 2;
                            const float4 b = vocab_at[1][at], s = vocab_at[0][at];
                            const float bs[4] = {b.x, b.y, b.z, b.w}, ss[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
                            for (int j = 0; j < IN; j++) {
                                half4 h4, l4;
                                float g[4];
#pragma unroll
                                for (int k = 0; k < 4; k++) {
                                    const float x = fmaf(acc[i][j][q * 4 + k] * by_row[j], ss[k], bs[k]);
                                    float p = __builtin_amdgcn_exp2f(x - lse2[j]);  // (a padding row's lse is +inf: 0)
                                    if constexpr (decltype(targets)::value)
                                        if (target[j] == static_cast<int>(v0) + at * 4 + k) p = less[j] * ss[k];
                                    if constexpr (MODE == 2) sums[q * 4 + k] = j == 0 ? p * dl[j] : fmaf(p, dl[j], sums[q * 4 + k]);
                                    g[k] = p * f[j];  // (of a sure token's taught ids past fp16: pick_kernel writes those anew)
                                }
                                pairs(g, 1.f, h4, l4);
                                hi[h][j] = __builtin_bit_cast(uint2, h4);
                                if constexpr (PL == 2) lo[h][j] = __builtin_bit_cast(uint2, l4);
                            }
                        }
                        // a lane has entries 0-3 and 8-11 (upper half: 4-7, 12-15) of 16: the halves exchange, 16 bytes a lane
#pragma unroll
                        for (int j = 0; j < IN; j++) {
                            const int64_t at = block + to[j] + q2 * 16;
                            *reinterpret_cast<uint4 *>(a.g[0] + at) = exchange(hi[0][j], hi[1][j]);
                            if constexpr (PL == 2) *reinterpret_cast<uint4 *>(a.g[1] + at) = exchange(lo[0][j], lo[1][j]);
                        }
                        __builtin_amdgcn_sched_barrier(0);
                    }
                };
                if (some)
                    values(Bool<true>{});
                else
                    values(Bool<false>{});
                if constexpr (MODE == 2) {
                    // sums over the 32 lanes of a half: each step halves the values and adds those of the other lanes
                    int n = 16, e = 0;
#pragma unroll
                    for (int mask = 16; mask > 1; mask >>= 1) {
                        n >>= 1;
                        const bool upper = lane & mask;
#pragma unroll
                        for (int k = 0; k < 8; k++)
                            if (k < n) {
                                const float keep = upper ? sums[k + n] : sums[k], give = upper ? sums[k] : sums[k + n];
                                sums[k] = keep + __shfl_xor(give, mask);
                            }
                        e += upper ? n : 0;
                    }
                    sums[0] += __shfl_xor(sums[0], 1);
                    const int ve = v_first + i * 32 + ((e >> 2) & 3) * 8 + (e & 3);
                    const float sw = reinterpret_cast<const float *>(vocab_at)[ve];  // (0 behind the vocabulary's end)
                    if ((lane & 1) == 0) a.db[(tt * 2 + wn) * a.piece + (v0 - a.v0) + ve] = sums[0] * (max_sw / sw);
                }
            }
        }
    }
    if constexpr (FORWARD) {
        float2 *both = reinterpret_cast<float2 *>(stage);
        __syncthreads();  // (the last tile began no other)
#pragma unroll
        for (int j = 0; j < IN; j++) {
            const float m2 = swap_halves(m[j]), l2 = swap_halves(l[j]);
            join(m[j], l[j], m2, l2);
            const int r = wn * (TN / 2) + j * 32 + (lane & 31);
            if (wm == 1 && lane < 32) both[r] = make_float2(m[j], l[j]);
        }
        __syncthreads();
#pragma unroll
        for (int j = 0; j < IN; j++) {
            const int r = wn * (TN / 2) + j * 32 + (lane & 31);
            if (wm == 0 && lane < 32) {
                join(m[j], l[j], both[r].x, both[r].y);
                a.part[static_cast<int64_t>(part) * row_tiles * TN + row0 + r] = make_float2(m[j], l[j]);
            }
        }
    }
}

// ---------------------------------------------------------------- logits of few tokens

struct Few {
    const void *x, *table;
    const float *bias;
    int64_t tokens, vocab;
    int d;
    float scale;
    float2 *part;  // [gridDim.x][kFewTokens]
    Taught taught;
    float *hit;    // cross entropy: log2 e times the target's logit of each token; or NULL
    float *picks;  // distillation from up to kFewEntries ids: log2 e times their logits, [tokens][top]; or NULL
};

// 4 (fp32) or 8 (bf16) values of a row from column c as MFMA operands, 0 behind the row's end
template <bool BF16>
__device__ __forceinline__ raw4 row16(const void *base, int64_t row, int c, int d) {
    constexpr int N = Vec<BF16>::N;
    const char *p = static_cast<const char *>(base) + (row + c) * (BF16 ? 2 : 4);
    if (c + N <= d) return *reinterpret_cast<const raw4_any *>(p);
    raw4 v = {0, 0, 0, 0};
#pragma unroll
    for (int j = 0; j < N - 1; j++)
        if (c + j < d) {
            if constexpr (BF16)
                v[j >> 1] |= static_cast<uint32_t>(reinterpret_cast<const uint16_t *>(p)[j]) << (16 * (j & 1));
            else
                v[j] = reinterpret_cast<const uint32_t *>(p)[j];
        }
    return v;
}

// 16 entries of the table by 16 NT tokens; the four waves share the columns.  Bound by the table's bytes (one token, 30000 x 768 fp32:
// 18 us, 5.1 TB/s; without four loads under way 22): operands go
// from memory into registers in the order that MFMA takes them (a lane's 16 bytes are its k of four
// fp32 products or of one bf16 product), no LDS, no copy of the table.
template <bool BF16, int NT>
__global__ __launch_bounds__(kThreads) void few_kernel(Few a) {
    constexpr int N = Vec<BF16>::N, S = 4 * N;  // columns of a step
    __shared__ floatx4 sums[3][NT][64];
    __shared__ int ids[kFewEntries];     // -1: not named
    __shared__ float tile[16 * NT][17];  // the first wave's
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, row = lane & 15, k0 = (lane >> 4) * N;
    const int steps = (a.d + S - 1) / S, per = (steps + 3) / 4, from = wave * per, to = from + per < steps ? from + per : steps;
    float m[NT], l[NT];
#pragma unroll
    for (int j = 0; j < NT; j++) m[j] = -INFINITY, l[j] = 0.f;
    const int entries = a.picks ? static_cast<int>(a.tokens) * a.taught.top : 0;
    for (int e = threadIdx.x; e < entries; e += kThreads) {
        const int t = e / a.taught.top, k = e - t * a.taught.top;
        ids[e] = a.taught.named(t, k) ? static_cast<int>(a.taught.id(t, k)) : -1;
    }
    int64_t target[NT];
#pragma unroll
    for (int j = 0; j < NT; j++) target[j] = a.hit && j * 16 + row < a.tokens ? a.taught.id(j * 16 + row, 0) : -1;
    const char *xp[NT];
#pragma unroll
    for (int j = 0; j < NT; j++)
        xp[j] = static_cast<const char *>(a.x) + ((j * 16 + row < a.tokens ? j * 16 + row : a.tokens - 1) * a.d + k0) * (BF16 ? 2 : 4);
    const int64_t groups = (a.vocab + 15) / 16;
    for (int64_t g = blockIdx.x; g < groups; g += gridDim.x) {
        const int64_t v = g * 16 + row < a.vocab ? g * 16 + row : a.vocab - 1;
        floatx4 acc[NT];
#pragma unroll
        for (int j = 0; j < NT; j++) acc[j] = floatx4{0.f, 0.f, 0.f, 0.f};
        const auto multiply = [&](const raw4 &w, const raw4 &x, floatx4 &sum) {
            if constexpr (BF16) {
                sum = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, w), __builtin_bit_cast(bf16x8, x), sum, 0, 0, 0);
            } else {
#pragma unroll
                for (int k = 0; k < 4; k++)
                    sum = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(w[k]), __uint_as_float(x[k]), sum, 0, 0, 0);
            }
        };
        // steps within the rows four at a time, their loads under way together; then those at the end
        const int whole = a.d / S < to ? a.d / S : to;
        const char *wp = static_cast<const char *>(a.table) + (v * a.d + k0) * (BF16 ? 2 : 4);
        int s = from;
        for (; s + 4 <= whole; s += 4) {
            raw4 w[4], x[NT][4];
#pragma unroll
            for (int i = 0; i < 4; i++) w[i] = *reinterpret_cast<const raw4_any *>(wp + (s + i) * 64);
#pragma unroll
            for (int j = 0; j < NT; j++)
#pragma unroll
                for (int i = 0; i < 4; i++) x[j][i] = *reinterpret_cast<const raw4_any *>(xp[j] + (s + i) * 64);
#pragma unroll
            for (int i = 0; i < 4; i++)
#pragma unroll
                for (int j = 0; j < NT; j++) multiply(w[i], x[j][i], acc[j]);
        }
        for (; s < to; s++) {
            const raw4 w = row16<BF16>(a.table, v * a.d, s * S + k0, a.d);
#pragma unroll
            for (int j = 0; j < NT; j++) {
                const int64_t t = j * 16 + row < a.tokens ? j * 16 + row : a.tokens - 1;
                multiply(w, row16<BF16>(a.x, t * a.d, s * S + k0, a.d), acc[j]);
            }
        }
        __syncthreads();
        if (wave > 0)
#pragma unroll
            for (int j = 0; j < NT; j++) sums[wave - 1][j][lane] = acc[j];
        __syncthreads();
        if (wave == 0) {
            // the lane's entries 4 (lane / 16) + k of its token lane % 16
            float b[4];
#pragma unroll
            for (int k = 0; k < 4; k++) {
                const int64_t e = g * 16 + 4 * (lane >> 4) + k;
                b[k] = e >= a.vocab ? -INFINITY : bias_of(a.bias, e, a.scale);
            }
#pragma unroll
            for (int j = 0; j < NT; j++) {
                float x[4], top = -INFINITY, sum = 0.f;
#pragma unroll
                for (int k = 0; k < 4; k++) {
                    const float s = acc[j][k] + sums[0][j][lane][k] + sums[1][j][lane][k] + sums[2][j][lane][k];
                    x[k] = fmaf(s, a.scale * kLog2e, b[k]);
                    if (target[j] == g * 16 + 4 * (lane >> 4) + k && target[j] < a.vocab) a.hit[j * 16 + row] = x[k];
                    if (a.picks) tile[j * 16 + row][4 * (lane >> 4) + k] = x[k];
                    top = fmaxf(top, x[k]);
                }
                const float at = top == -INFINITY ? 0.f : top;
#pragma unroll
                for (int k = 0; k < 4; k++) sum += __builtin_amdgcn_exp2f(x[k] - at);
                join(m[j], l[j], top, sum);
            }
            wave_meet();
            for (int e = lane; e < entries; e += 64) {
                const int64_t in = ids[e] - g * 16;
                if (ids[e] >= 0 && in >= 0 && in < 16) a.picks[e] = tile[e / a.taught.top][in];
            }
            wave_meet();
        }
    }
    if (wave == 0)
#pragma unroll
        for (int j = 0; j < NT; j++) {
#pragma unroll
            for (int s = 16; s < 64; s <<= 1) join(m[j], l[j], __shfl_xor(m[j], s), __shfl_xor(l[j], s));
            if (lane < 16) a.part[static_cast<int64_t>(blockIdx.x) * kFewTokens + j * 16 + lane] = make_float2(m[j], l[j]);
        }
}

// The softmax of a row's teacher logits, computed by the wave: probability of entry k is exp2((logit - top) c) / sum.  (The difference
// first: of large logits the product's rounding is no longer small.)
struct Teacher {
    float c, top, sum;
    __device__ __forceinline__ Teacher(const Taught &a, int64_t t, float scale) {
        const int lane = threadIdx.x & 63;
        c = scale * kLog2e;
        top = -INFINITY;
        for (int k = lane; k < a.top; k += 64)
            if (a.named(t, k)) top = fmaxf(top, a.teacher[t * a.top + k]);
        top = wave_max(top);
        sum = 0.f;
        for (int k = lane; k < a.top; k += 64)
            if (a.named(t, k)) sum += exp2f((a.teacher[t * a.top + k] - top) * c);
        sum = wave_sum(sum);
    }
    __device__ __forceinline__ float log2_of(float logit) const { return (logit - top) * c - log2f(sum); }
    __device__ __forceinline__ float of(float logit) const { return exp2f((logit - top) * c) / sum; }
};

typedef uint32_t raw2_any __attribute__((ext_vector_type(2), aligned(2)));

// four values of a row from column c, as many as it has
template <bool BF16>
__device__ __forceinline__ void store4(void *base, int64_t row, int64_t c, int64_t d, const float (&v)[4]) {
    if constexpr (BF16) {
        uint16_t *p = static_cast<uint16_t *>(base) + row + c;
        raw2_any w;
#pragma unroll
        for (int j = 0; j < 2; j++) {
            const floatx2 f = {v[2 * j], v[2 * j + 1]};
            w[j] = __builtin_bit_cast(uint32_t, __builtin_convertvector(f, bf16x2));
        }
        if (c + 4 <= d)
            *reinterpret_cast<raw2_any *>(p) = w;
        else
#pragma unroll
            for (int j = 0; j < 3; j++)
                if (c + j < d) p[j] = static_cast<uint16_t>(w[j >> 1] >> (16 * (j & 1)));
    } else {
        float *p = static_cast<float *>(base) + row + c;
        if (c + 4 <= d)
            *reinterpret_cast<float4_any *>(p) = float4_any{v[0], v[1], v[2], v[3]};
        else
#pragma unroll
            for (int j = 0; j < 3; j++)
                if (c + j < d) p[j] = v[j];
    }
}

// ---------------------------------------------------------------- gradients of few tokens

struct FewBackward {
    Taught taught;
    const void *x, *table;
    const float *bias, *logq, *lse;  // logq: cross entropy's loss where taught.teacher is NULL
    int64_t tokens, vocab;
    int d;
    float scale;
    void *dw;
    float *db, *px;  // px [gridDim.x][16 NT][d]
};

constexpr int kFewBackward = 32;          // tokens at most
constexpr int kFewColumns = 1024;         // columns at most, of up to 16 tokens twice as many
constexpr int kFewBackwardBlocks = 512;

// four values of a row from column c, 0 behind its end or where `in` is false
template <bool BF16>
__device__ __forceinline__ void load4(const void *base, int64_t row, int c, int d, bool in, float (&v)[4]) {
#pragma unroll
    for (int k = 0; k < 4; k++) v[k] = 0.f;
    if (!in) return;
    if (c + 4 <= d) {
        if constexpr (BF16) {
            const raw2_any w = *reinterpret_cast<const raw2_any *>(static_cast<const uint16_t *>(base) + row + c);
#pragma unroll
            for (int k = 0; k < 4; k++) v[k] = __uint_as_float(k & 1 ? w[k >> 1] & 0xFFFF0000u : w[k >> 1] << 16);
        } else {
            const float4_any w = *reinterpret_cast<const float4_any *>(static_cast<const float *>(base) + row + c);
#pragma unroll
            for (int k = 0; k < 4; k++) v[k] = w[k];
        }
    } else {
#pragma unroll
        for (int k = 0; k < 3; k++)
            if (c + k < d) v[k] = load1<BF16>(base, row + c + k);
    }
}

// All gradients of 16 entries of the table at a time, in fp32 throughout: their logits (as few_kernel), G, their rows of dW, their
// part of dx, which stays in registers until the workgroup's last entries.  The table is read from memory once and dW
// written once; what the general form does with planes would read and write the table three times more.  16 tokens, 30000 x 768
// fp32: 60 us, bound by the latency of four dependent stages for each 16 entries at two waves a SIMD (more waves: 75 to 80).
template <bool BF16, int NT, int CT>  // 16 NT tokens; CT stretches of 64 columns a wave
__global__ __launch_bounds__(kThreads, 2) void few_backward_kernel(FewBackward a) {
    constexpr int N = Vec<BF16>::N, S = 4 * N, T = 16 * NT;
    __shared__ floatx4 sums[3][NT][64];
    __shared__ float g[T][17];
    __shared__ int ids[kFewEntries];  // the first of equal ids of a token; -1: none
    __shared__ float taught_p[kFewEntries], taught_q[kFewEntries];
    __shared__ float dls[T];  // dloss scale, 0 where the token takes no part
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, row = lane & 15, quad = lane >> 4, k0 = quad * N;
    const int tokens = static_cast<int>(a.tokens), top = a.taught.top;

    for (int t = wave; t < T; t += 4) {
        bool any = false;
        if (t < tokens)
            for (int k = lane; k < top; k += 64) any |= a.taught.named(t, k);
        const float dl = t < tokens ? a.taught.dloss[t] : 0.f;
        any = __ballot(any) != 0 && dl != 0.f;
        if (lane == 0) dls[t] = any ? dl * a.scale : 0.f;
        if (t >= tokens) continue;
        if (a.taught.teacher) {
            const Teacher p(a.taught, t, a.scale);
            for (int k = lane; k < top; k += 64) {
                const bool named = any && a.taught.named(t, k);
                ids[t * top + k] = named ? static_cast<int>(a.taught.id(t, k)) : -1;
                taught_p[t * top + k] = named ? p.of(a.taught.teacher[static_cast<int64_t>(t) * top + k]) : 0.f;
                taught_q[t * top + k] = a.logq[static_cast<int64_t>(t) * top + k];
            }
        } else if (lane == 0) {
            ids[t] = any ? static_cast<int>(a.taught.id(t, 0)) : -1;
            taught_p[t] = 1.f;
            taught_q[t] = -a.logq[t];
        }
    }
    __syncthreads();
    if (a.taught.teacher) {
        // equal ids: the first gets the sum
        constexpr int EACH = kFewEntries / kThreads;
        float p[EACH];
        bool later[EACH];
#pragma unroll
        for (int i = 0; i < EACH; i++) {
            const int e = i * kThreads + threadIdx.x;
            p[i] = 0.f;
            later[i] = false;
            if (e < tokens * top && ids[e] >= 0) {
                const int t0 = e / top * top;
                for (int o = t0; o < t0 + top; o++)
                    if (ids[o] == ids[e]) {
                        p[i] += taught_p[o];
                        later[i] |= o < e;
                    }
            }
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < EACH; i++) {
            const int e = i * kThreads + threadIdx.x;
            if (e < tokens * top) {
                taught_p[e] = p[i];
                if (later[i]) ids[e] = -1;
            }
        }
        __syncthreads();
    }

    // a lane's token of the logits' tiles, and its rows of x
    float lse2[NT], dl[NT];
    const char *xp[NT];
#pragma unroll
    for (int j = 0; j < NT; j++) {
        const int t = j * 16 + row;
        dl[j] = dls[t];
        lse2[j] = t < tokens ? a.lse[t] * kLog2e : 0.f;
        xp[j] = static_cast<const char *>(a.x) + (static_cast<int64_t>(t < tokens ? t : tokens - 1) * a.d + k0) * (BF16 ? 2 : 4);
    }
    const int steps = (a.d + S - 1) / S, per = (steps + 3) / 4, from = wave * per, to = from + per < steps ? from + per : steps;
    const int whole = a.d / S < to ? a.d / S : to;
    // columns 64 (wave + 4 c) + 4 row + k: one 16-byte load is an operand of four products, k = 0 ... 3
    floatx4 dx[NT][CT][4];
    uint32_t takes = 0;  // tokens 16 j + 4 i + quad
#pragma unroll
    for (int j = 0; j < NT; j++)
#pragma unroll
        for (int i = 0; i < 4; i++) takes |= dls[j * 16 + 4 * i + quad] != 0.f ? 1u << (j * 4 + i) : 0u;
#pragma unroll
    for (int j = 0; j < NT; j++)
#pragma unroll
        for (int c = 0; c < CT; c++)
#pragma unroll
            for (int k = 0; k < 4; k++) dx[j][c][k] = floatx4{0.f, 0.f, 0.f, 0.f};

    const int64_t groups = (a.vocab + 15) / 16;
    for (int64_t group = blockIdx.x; group < groups; group += gridDim.x) {
        const int64_t v0 = group * 16, v = v0 + row < a.vocab ? v0 + row : a.vocab - 1;
        floatx4 acc[NT];
#pragma unroll
        for (int j = 0; j < NT; j++) acc[j] = floatx4{0.f, 0.f, 0.f, 0.f};
        const auto multiply = [&](const raw4 &w, const raw4 &x, floatx4 &sum) {
            if constexpr (BF16) {
                sum = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, w), __builtin_bit_cast(bf16x8, x), sum, 0, 0, 0);
            } else {
#pragma unroll
                for (int k = 0; k < 4; k++)
                    sum = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(w[k]), __uint_as_float(x[k]), sum, 0, 0, 0);
            }
        };
        const char *wp = static_cast<const char *>(a.table) + (v * a.d + k0) * (BF16 ? 2 : 4);
        int s = from;
        for (; s + 4 <= whole; s += 4) {
            raw4 w[4], x[NT][4];
#pragma unroll
            for (int i = 0; i < 4; i++) w[i] = *reinterpret_cast<const raw4_any *>(wp + (s + i) * 64);
#pragma unroll
            for (int j = 0; j < NT; j++)
#pragma unroll
                for (int i = 0; i < 4; i++) x[j][i] = *reinterpret_cast<const raw4_any *>(xp[j] + (s + i) * 64);
#pragma unroll
            for (int i = 0; i < 4; i++)
#pragma unroll
                for (int j = 0; j < NT; j++) multiply(w[i], x[j][i], acc[j]);
        }
        for (; s < to; s++) {
            const raw4 w = row16<BF16>(a.table, v * a.d, s * S + k0, a.d);
#pragma unroll
            for (int j = 0; j < NT; j++) {
                const int64_t t = j * 16 + row < tokens ? j * 16 + row : tokens - 1;
                multiply(w, row16<BF16>(a.x, t * a.d, s * S + k0, a.d), acc[j]);
            }
        }
        if (wave > 0)
#pragma unroll
            for (int j = 0; j < NT; j++) sums[wave - 1][j][lane] = acc[j];
        __syncthreads();  // (every wave has done with g of the entries before, too)
        if (wave == 0)
#pragma unroll
            for (int j = 0; j < NT; j++)
#pragma unroll
                for (int k = 0; k < 4; k++) {
                    // the lane's entries 4 quad + k of its token
                    const int64_t e = v0 + 4 * quad + k;
                    const float b = e >= a.vocab ? -INFINITY : bias_of(a.bias, e, a.scale);
                    const float l = acc[j][k] + sums[0][j][lane][k] + sums[1][j][lane][k] + sums[2][j][lane][k];
                    const float p = __builtin_amdgcn_exp2f(fmaf(l, a.scale * kLog2e, b) - lse2[j]);
                    g[j * 16 + row][4 * quad + k] = dl[j] == 0.f ? 0.f : e >= a.vocab ? 0.f : p * dl[j];
                }
        __syncthreads();
        for (int e = threadIdx.x; e < tokens * top; e += kThreads) {
            const int64_t in = ids[e] - v0;
            if (ids[e] >= 0 && in >= 0 && in < 16) {
                const int t = e / top;
                const float p = taught_p[e], q = taught_q[e];
                g[t][in] = (p == 1.f ? expm1f(q) : expf(q) - p) * dls[t];
            }
        }
        __syncthreads();
        if (a.db && threadIdx.x < 16 && v0 + threadIdx.x < a.vocab) {
            float sum = 0.f;
#pragma unroll
            for (int t = 0; t < T; t++) sum += g[t][threadIdx.x];
            a.db[v0 + threadIdx.x] = sum;
        }
        // operands of the products over tokens and over entries: k = 4 i + quad of four MFMA
        float gv[NT][4], gt[NT][4];
#pragma unroll
        for (int j = 0; j < NT; j++)
#pragma unroll
            for (int i = 0; i < 4; i++) {
                gv[j][i] = g[j * 16 + 4 * i + quad][row];  // entry `row`, token 4 i + quad
                gt[j][i] = g[j * 16 + row][4 * i + quad];  // token `row`, entry 4 i + quad
            }
#pragma unroll
        for (int c = 0; c < CT; c++) {
            const int first = 64 * (wave + 4 * c), col = first + 4 * row;
            if (first >= a.d) break;
            floatx4 dw[4];
            float w[4][4], x[NT][4][4];
#pragma unroll
            for (int i = 0; i < 4; i++) {
                const int64_t e = v0 + 4 * i + quad;
                load4<BF16>(a.table, (e < a.vocab ? e : a.vocab - 1) * a.d, col, a.d, true, w[i]);
            }
#pragma unroll
            for (int j = 0; j < NT; j++)
#pragma unroll
                for (int i = 0; i < 4; i++)
                    load4<BF16>(a.x, static_cast<int64_t>(j * 16 + 4 * i + quad) * a.d, col, a.d, takes >> (j * 4 + i) & 1, x[j][i]);
#pragma unroll
            for (int k = 0; k < 4; k++) {
                dw[k] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int j = 0; j < NT; j++)
#pragma unroll
                    for (int i = 0; i < 4; i++) {
                        dw[k] = __builtin_amdgcn_mfma_f32_16x16x4f32(gv[j][i], x[j][i][k], dw[k], 0, 0, 0);
                        dx[j][c][k] = __builtin_amdgcn_mfma_f32_16x16x4f32(gt[j][i], w[i][k], dx[j][c][k], 0, 0, 0);
                    }
            }
            // rows 4 quad + e, four columns each
#pragma unroll
            for (int e = 0; e < 4; e++) {
                const float v4[4] = {dw[0][e], dw[1][e], dw[2][e], dw[3][e]};
                if (col < a.d && v0 + 4 * quad + e < a.vocab) store4<BF16>(a.dw, (v0 + 4 * quad + e) * a.d, col, a.d, v4);
            }
            __builtin_amdgcn_sched_barrier(0);  // (loads of the next columns ahead would cost registers)
        }
    }
#pragma unroll
    for (int c = 0; c < CT; c++) {
        const int col = 64 * (wave + 4 * c) + 4 * row;
        if (col < a.d)
#pragma unroll
            for (int j = 0; j < NT; j++)
#pragma unroll
                for (int e = 0; e < 4; e++) {
                    const float v4[4] = {dx[j][c][0][e], dx[j][c][1][e], dx[j][c][2][e], dx[j][c][3][e]};
                    store4<false>(a.px, (static_cast<int64_t>(blockIdx.x) * T + j * 16 + 4 * quad + e) * a.d, col, a.d, v4);
                }
    }
}

// dx of a token's 64 columns: 16 threads a vector of four, each a sixteenth of the workgroups' parts, joined in order.
template <bool BF16>
__global__ __launch_bounds__(kThreads) void few_finish_kernel(FewBackward a, int parts, int rows) {
    __shared__ float4 sums[16][16];
    const int in = threadIdx.x & 15, slice = threadIdx.x >> 4;
    const int t = blockIdx.y, c = blockIdx.x * 64 + in * 4;
    float v[4] = {0.f, 0.f, 0.f, 0.f};
    if (c < a.d) {
        const int n = parts > slice ? (parts - slice + 15) / 16 : 0;
        const float *p = a.px + (static_cast<int64_t>(slice) * rows + t) * a.d + c;
        const int64_t stride = static_cast<int64_t>(16) * rows * a.d;
        if (c + 4 <= a.d) {
#pragma unroll 8
            for (int i = 0; i < n; i++) {
                const float4_any s = *reinterpret_cast<const float4_any *>(p + i * stride);
#pragma unroll
                for (int k = 0; k < 4; k++) v[k] += s[k];
            }
        } else {
            for (int i = 0; i < n; i++)
#pragma unroll
                for (int k = 0; k < 3; k++)
                    if (c + k < a.d) v[k] += p[i * stride + k];
        }
    }
    sums[slice][in] = make_float4(v[0], v[1], v[2], v[3]);
    __syncthreads();
    if (slice != 0 || c >= a.d) return;
    const bool part = a.taught.takes_part(t);
    for (int k = 0; k < 4; k++) v[k] = 0.f;
#pragma unroll
    for (int i = 0; i < 16; i++) {
        const float4 s = sums[i][in];
        v[0] += s.x, v[1] += s.y, v[2] += s.z, v[3] += s.w;
    }
    // (a token that takes no part has zeros, whatever the table holds)
#pragma unroll
    for (int k = 0; k < 4; k++) v[k] = part ? v[k] : 0.f;
    store4<BF16>(a.dw, static_cast<int64_t>(t) * a.d, c, a.d, v);
}

// ---------------------------------------------------------------- the loss

struct Loss {
    Taught taught;
    const void *x, *table;
    const float *bias;
    int d;
    float scale;
    const int *rows;  // NULL: row r is token r (few tokens)
    const Meta *meta;
    const float2 *part;
    int parts;  // few tokens
    int tile_m;
    float *loss, *lse, *logq;
    const float *hit;  // cross entropy: the tiles' logits of the targets (times log2 e)
    bool left;         // distillation: the tiles left the taught ids' logits in logq (times log2 e)
};

// x_t . table_v of four entries (wave-uniform; an entry below 0 is skipped)
template <bool BF16>
__device__ __forceinline__ void dots(const void *x, int64_t xr, const void *w, const int (&v)[4], int d, float (&s)[4]) {
#pragma unroll
    for (int k = 0; k < 4; k++) s[k] = 0.f;
    for (int c = (threadIdx.x & 63) * 8; c < d; c += 512) {
        float a[8], b[4][8];
        row8<BF16>(x, xr, c, d, a);
#pragma unroll
        for (int k = 0; k < 4; k++)
            if (v[k] >= 0) row8<BF16>(w, static_cast<int64_t>(v[k]) * d, c, d, b[k]);
#pragma unroll
        for (int k = 0; k < 4; k++)
            if (v[k] >= 0)
#pragma unroll
                for (int j = 0; j < 8; j++) s[k] = fmaf(a[j], b[k][j], s[k]);
    }
#pragma unroll
    for (int k = 0; k < 4; k++) s[k] = wave_sum(s[k]);
}

// Cross entropy and distillation of few tokens, whose tiles left the taught ids' logits, and distillation where they are made
// here, as fp32 dot products.  A wave a row (R = 4), or where there are few rows the workgroup a row (R = 1).  With dot products
// bound by the rows of the table that are gathered (16384 x 32 of 768 fp32: 270 us, 6 TB/s), else by its launch (5 us).
template <bool BF16, int R>
__global__ __launch_bounds__(kThreads) void loss_kernel(Loss a) {
    __shared__ float picked[R][kMaxTop];
    __shared__ float2 joined[4];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t count = a.rows ? a.meta->count : a.taught.tokens;
    const int64_t r = static_cast<int64_t>(blockIdx.x) * R + (R == 1 ? 0 : wave);
    if (r >= count) return;  // (R == 4: no barrier follows)
    const int64_t t = a.rows ? a.rows[r] : r;
    float *at = picked[R == 1 ? 0 : wave];
    bool any = false;
    if (a.hit) {  // (few tokens)
        any = a.taught.named(t, 0);
        if (lane == 0) at[0] = a.hit[t];
    }
    if (a.left)  // (few tokens)
        for (int k = lane; k < up(a.taught.top, 64); k += 64) {
            const bool named = k < a.taught.top && a.taught.named(t, k);
            any |= __ballot(named) != 0;
            if (named) at[k] = a.logq[t * a.taught.top + k];
        }
    for (int k0 = 0; k0 < a.taught.top && !a.hit && !a.left; k0 += 64) {
        // a lane an id, then four at a time
        const int k = k0 + lane;
        const bool named = k < a.taught.top && a.taught.named(t, k);
        const int id = named ? static_cast<int>(a.taught.id(t, k)) : -1;
        const uint64_t some = __ballot(named);
        any |= some != 0;
        const int n = a.taught.top - k0 < 64 ? a.taught.top - k0 : 64;
        for (int e = R == 1 ? 4 * wave : 0; e < n; e += R == 1 ? 16 : 4) {
            int v[4];
            float s[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int j = 0; j < 4; j++) v[j] = __builtin_amdgcn_readlane(id, (e + j) & 63);
#pragma unroll
            for (int j = 0; j < 4; j++) v[j] = e + j < n ? v[j] : -1;
            if ((some >> e & 15) != 0) dots<BF16>(a.x, t * a.d, a.table, v, a.d, s);
#pragma unroll
            for (int j = 0; j < 4; j++)
                if (lane == 0 && e + j < n) at[k0 + e + j] = v[j] < 0 ? 0.f : a.scale * kLog2e * (s[j] + (a.bias ? a.bias[v[j]] : 0.f));
        }
    }
    wave_meet();
    float m = -INFINITY, l = 0.f;
    {
        int parts = a.parts;
        int64_t ld = kFewTokens;
        if (a.rows) {
            const int row_tiles = static_cast<int>((count + kTileN - 1) / kTileN);
            parts = vocab_parts(row_tiles, static_cast<int>((a.taught.vocab + a.tile_m - 1) / a.tile_m));
            ld = static_cast<int64_t>(row_tiles) * kTileN;
        }
#pragma unroll 4
        for (int i = R == 1 ? static_cast<int>(threadIdx.x) : lane; i < parts; i += R == 1 ? kThreads : 64) {
            const float2 s = a.part[i * ld + r];
            join(m, l, s.x, s.y);
        }
#pragma unroll
        for (int s = 1; s < 64; s <<= 1) {
            const float m2 = __shfl_xor(m, s), l2 = __shfl_xor(l, s);
            join(m, l, m2, l2);
        }
        if constexpr (R == 1) {
            if (lane == 0) joined[wave] = make_float2(m, l);
            __syncthreads();
            if (wave != 0) return;
            for (int w = 1; w < 4; w++) join(m, l, joined[w].x, joined[w].y);
        }
    }
    const float lse = (m + log2f(l)) * kLn2;
    float loss = 0.f;
    if (any && a.taught.teacher) {
        const Teacher p(a.taught, t, a.scale);
        for (int k = lane; k < a.taught.top; k += 64)
            if (a.taught.named(t, k)) {
                const float logit = a.taught.teacher[t * a.taught.top + k], prob = p.of(logit);
                if (prob != 0.f) loss += prob * (p.log2_of(logit) * kLn2 - log_q(settled(at[k], m, l), m, l));
            }
        loss = wave_sum(loss);
    } else if (any) {
        loss = -log_q(at[0], m, l);
    }
    if (a.logq)
        for (int k = lane; k < a.taught.top; k += 64) a.logq[t * a.taught.top + k] = a.taught.named(t, k) ? log_q(settled(at[k], m, l), m, l) : 0.f;
    if (lane == 0) {
        a.loss[t] = loss;
        a.lse[t] = any ? lse : 0.f;
    }
}

// Distillation where the tiles left the ids' logits (times log2 e) in logq: a wave a row, a lane an id.
__global__ __launch_bounds__(kThreads) void picked_loss_kernel(Loss a) {
    const int lane = threadIdx.x & 63;
    const int64_t count = a.meta->count, r = static_cast<int64_t>(blockIdx.x) * 4 + (threadIdx.x >> 6);
    if (r >= count) return;
    const int64_t t = a.rows[r];
    const int row_tiles = static_cast<int>((count + kTileN - 1) / kTileN);
    const int parts = vocab_parts(row_tiles, static_cast<int>((a.taught.vocab + a.tile_m - 1) / a.tile_m));
    const int64_t ld = static_cast<int64_t>(row_tiles) * kTileN;
    const bool in = lane < a.taught.top;
    const int64_t id = in ? a.taught.id(t, lane) : -1;
    const float logit = in ? a.taught.teacher[t * a.taught.top + lane] : -INFINITY, x = in ? a.logq[t * a.taught.top + lane] : 0.f;
    const bool named = id >= 0 && id < a.taught.vocab && logit != -INFINITY;
    float m = -INFINITY, l = 0.f;
    for (int i = lane; i < parts; i += 64) {
        const float2 s = a.part[i * ld + r];
        join(m, l, s.x, s.y);
    }
    for (int s = 1; s < 64 && s < parts; s <<= 1) {
        const float m2 = __shfl_xor(m, s), l2 = __shfl_xor(l, s);
        join(m, l, m2, l2);
    }
    m = __shfl(m, 0), l = __shfl(l, 0);
    const float lse = (m + log2f(l)) * kLn2, logq = named ? log_q(x, m, l) : 0.f;
    const float c = a.scale * kLog2e, top = wave_max(named ? logit : -INFINITY);
    const float e = named ? exp2f((logit - top) * c) : 0.f, sum = wave_sum(e), p = e / sum;
    const float loss = wave_sum(named && p != 0.f ? p * (((logit - top) * c - log2f(sum)) * kLn2 - logq) : 0.f);
    if (in) a.logq[t * a.taught.top + lane] = logq;
    if (lane == 0) {
        a.loss[t] = loss;
        a.lse[t] = lse;
    }
}

// The named ids of each row in ascending order, as 64 id + k: a wave a row, one id a lane, sorted by exchanges.
__global__ __launch_bounds__(kThreads) void sort_ids_kernel(Taught a, const int *rows, const Meta *meta, int *sorted, int ld) {
    const int lane = threadIdx.x & 63;
    for (int r = blockIdx.x * 4 + (threadIdx.x >> 6); r < meta->count; r += gridDim.x * 4) {
        const int64_t t = rows[r];
        int key = kNoId;
        if (lane < a.top && a.named(t, lane)) key = static_cast<int>(a.id(t, lane)) * 64 + lane;
#pragma unroll
        for (int size = 2; size <= 64; size <<= 1)
#pragma unroll
            for (int step = size >> 1; step > 0; step >>= 1) {
                const int other = __shfl_xor(key, step);
                const bool low = ((lane & step) == 0) == ((lane & size) == 0);
                key = low ? min(key, other) : max(key, other);
            }
        if (lane < ld) sorted[static_cast<int64_t>(r) * ld + lane] = key;
        if (lane + 64 < ld) sorted[static_cast<int64_t>(r) * ld + 64 + lane] = kNoId;
    }
}

// Cross entropy where the tiles left the targets' logits: R rows of a workgroup, 256 / R threads share a row's parts.
template <int R>
__global__ __launch_bounds__(kThreads) void target_loss_kernel(Loss a) {
    __shared__ float2 from[kThreads];
    const int64_t count = a.meta->count, r = static_cast<int64_t>(blockIdx.x) * R + threadIdx.x % R;
    if (static_cast<int64_t>(blockIdx.x) * R >= count) return;
    const int row_tiles = static_cast<int>((count + kTileN - 1) / kTileN);
    const int parts = vocab_parts(row_tiles, static_cast<int>((a.taught.vocab + a.tile_m - 1) / a.tile_m));
    const int64_t ld = static_cast<int64_t>(row_tiles) * kTileN;  // (whole multiples of R: r is within)
    float m = -INFINITY, l = 0.f;
#pragma unroll 4
    for (int i = threadIdx.x / R; i < parts; i += kThreads / R) {
        const float2 s = a.part[i * ld + r];
        join(m, l, s.x, s.y);
    }
    from[threadIdx.x] = make_float2(m, l);
    for (int n = kThreads / R / 2; n > 0; n >>= 1) {
        __syncthreads();
        if (threadIdx.x < n * R) {
            const float2 s = from[threadIdx.x + n * R];
            join(m, l, s.x, s.y);
            from[threadIdx.x] = make_float2(m, l);
        }
    }
    if (threadIdx.x >= R || r >= count) return;
    const int64_t t = a.rows[r];
    a.loss[t] = -log_q(a.hit[r], m, l);
    a.lse[t] = (m + log2f(l)) * kLn2;
}

// ---------------------------------------------------------------- G at the ids that are taught

struct Pick {
    Taught taught;
    const float *logq;  // log q of each id
    float scale;
    const int *rows;
    const Meta *meta;
    const float *sx, *dls, *sw;
    int64_t v0, v1;
    _Float16 *g[2];
    int64_t g_rows;
    Picked picked;
    float *db;  // with picked: Logits::db, which a probability that is no number goes to
    int64_t piece;

    // dloss scale p to db's entry v, by row r
    __device__ __forceinline__ void add(int64_t r, int64_t v, float p, float unit) const {
        if (p != p) db[r / (kTileN / 2) * piece + (v - v0)] = p;
        const int copy = (blockIdx.x * 4 + (threadIdx.x >> 6)) & (picked.copies - 1);
        atomicAdd(&picked.sums[copy * picked.ld + v], static_cast<unsigned long long>(llrintf(p != p ? 0.f : dls[r] * p * unit * 1048576.f)));
    }

    // G[r][v] = (q - p) by, as planes
    template <int PL>
    __device__ __forceinline__ void put(int64_t r, int64_t v, float logq, float p, float by) const {
        const float x = (p == 1.f ? expm1f(logq) : expf(logq) - p) * by;
        _Float16 hi, lo;
        pair(x, 1.f, hi, lo);
        const int64_t at = (((v - v0) >> 5) * g_rows + r) * 32 + ((v - v0) & 31);
        g[0][at] = hi;
        if constexpr (PL == 2) g[1][at] = lo;
    }
};

// q - p is formed from the forward's log q in fp32, so that nothing of it is lost where q is near p (cross
// entropy: so does logits_kernel).  A wave a row, a lane an id.
typedef int intx4 __attribute__((ext_vector_type(4)));

template <int PL, bool MANY>  // MANY: more than 64 ids a token
__global__ __launch_bounds__(kThreads) void pick_kernel(Pick a) {
    __shared__ __align__(16) int ids[4][MANY ? kMaxTop : 1];
    __shared__ __align__(16) float probs[4][MANY ? kMaxTop : 1];
    const int lane = threadIdx.x & 63;
    const Taught &s = a.taught;
    const Scales scales(a.meta);
    const float by_sw = 1.f / scales.max_sw;
    const float unit = ldexpf(1.f, 40 - scale_exp(a.meta->largest(kMaxDl)) - 20);
    const int count = a.meta->count;
    for (int r = blockIdx.x * 4 + (threadIdx.x >> 6); r < count; r += gridDim.x * 4) {
        const int64_t t = a.rows[r];
        const float f = a.dls[r] * scales.row(a.sx[r], a.dls[r]) * scales.up();
        if constexpr (!MANY) {
            const bool in = lane < s.top;
            const int64_t v64 = in ? s.id(t, lane) : -1;
            const float logit = in ? s.teacher[t * s.top + lane] : -INFINITY;
            const bool named = v64 >= 0 && v64 < s.vocab && logit != -INFINITY;
            const int v = named ? static_cast<int>(v64) : -1;
            const bool here = named && v >= a.v0 && v < a.v1;
            if (__ballot(here) == 0) continue;
            const float c = a.scale * kLog2e, top = wave_max(named ? logit : -INFINITY);
            const float e = named ? exp2f((logit - top) * c) : 0.f;
            const float mine = e / wave_sum(e);
            if (here && a.picked.sums) a.add(r, v, mine, unit);
            // the same id again (looked for first): the first writes the sum
            float sum = mine;
            bool first = true;
            uint64_t again = 0;
            for (int k = 0; k < s.top; k++) again |= __ballot(v == __builtin_amdgcn_readlane(v, k)) & ~(uint64_t{1} << k);
            if ((again & __ballot(here)) != 0) {
                sum = 0.f;
                for (int k = 0; k < s.top; k++) {
                    const int o = __builtin_amdgcn_readlane(v, k);
                    const float po = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(mine), k));
                    if (o == v) {
                        sum += po;
                        first = first && k >= lane;
                    }
                }
            }
            if (here && first) a.template put<PL>(r, v, a.logq[t * s.top + lane], sum, f * (scales.table(a.sw[v]) * by_sw));
        } else {
            // more ids than lanes: the row's list in LDS, a lane's up to 16 ids compared with four of it at a time
            constexpr int EACH = kMaxTop / 64;
            const Teacher p(s, t, a.scale);
            const int wave = threadIdx.x >> 6, quads = (s.top + 3) / 4;
            for (int k = lane; k < 4 * quads; k += 64) {
                const bool named = k < s.top && s.named(t, k);
                ids[wave][k] = named ? static_cast<int>(s.id(t, k)) : -1;
                probs[wave][k] = named ? p.of(s.teacher[t * s.top + k]) : 0.f;
            }
            wave_meet();
            int v[EACH];
            float sum[EACH];
            uint32_t again = 0;  // the lane's ids that came before in the list
#pragma unroll
            for (int i = 0; i < EACH; i++) {
                const int k = i * 64 + lane;
                const int id = k < s.top ? ids[wave][k] : -1;
                const bool here = id >= a.v0 && id < a.v1;
                v[i] = here ? id : -2;
                sum[i] = 0.f;
                if (here && a.picked.sums) a.add(r, id, probs[wave][k], unit);
            }
            for (int e = 0; e < quads; e++) {
                const intx4 os = *reinterpret_cast<const intx4 *>(&ids[wave][4 * e]);
                const floatx4 ps = *reinterpret_cast<const floatx4 *>(&probs[wave][4 * e]);
#pragma unroll
                for (int i = 0; i < EACH; i++) {
                    if (i * 64 >= s.top) break;
#pragma unroll
                    for (int c = 0; c < 4; c++)
                        if (os[c] == v[i]) {
                            sum[i] += ps[c];
                            if (e * 4 + c < i * 64 + lane) again |= 1u << i;
                        }
                }
            }
#pragma unroll
            for (int i = 0; i < EACH; i++)
                if (v[i] >= 0 && !(again >> i & 1))
                    a.template put<PL>(r, v[i], a.logq[t * s.top + i * 64 + lane], sum[i], f * (scales.table(a.sw[v[i]]) * by_sw));
            wave_meet();
        }
    }
}

// ---------------------------------------------------------------- dx and dW of a piece

struct Gradients {
    const char *x[2], *w[2], *g[2];  // planes of rows (x, g) and w_rows rows
    int64_t rows, w_rows;
    int64_t ld, piece;  // columns of the planes of x and w, of g
    int64_t d, v0, vocab, width;     // width: entries of the piece, its end cut at the vocabulary's
    const Meta *meta;
    const float *sw;
    float *px, *pw;  // fp32 parts [part][rows][ld]
    bool add;        // a later piece: px holds the ones before
    bool single;     // one piece: sums that are not cut go to dx at once
    const int *listed;
    const float *sx, *dls;
    void *dx;        // [tokens][d]
    void *dw;        // [vocab][d]
};

// Parts that a sum over `steps` steps is cut into for `tiles` tiles: enough workgroups for the card, a part of 16 steps at least.
__host__ __device__ inline int sum_parts(int tiles, int steps) {
    const int room = kGradSlots / (tiles > 0 ? tiles : 1), most = steps / 16;
    const int n = room < most ? room : most;
    return n < 1 ? 1 : n;
}

// Sums over the vocabulary (dx) and over the tokens (dW) of one piece in one launch, the table's and x's columns as the tiles' rows (a
// lane then holds four columns of a row of the result side by side).  Bound by the matrix units and the card's power:
// 16384 x 768 into 30000, passes in a row, bf16 1420 us (1.06 PFLOP/s), fp32 pairs 3985 (1.14).
template <bool BF16>
__global__ __launch_bounds__(kThreads, 2) void gradients_kernel(Gradients a) {
    constexpr int PL = BF16 ? 1 : 2, TM = kGradM, TN = grad_n(BF16);
    typedef Product<PL, TM, TN, true, false, false> PX;
    typedef Product<PL, TM, TN, true, true, false> PW;
    constexpr int IM = PX::IM, IN = PX::IN;
    __shared__ __align__(1024) char stage[PX::kLds > PW::kLds ? PX::kLds : PW::kLds];
    const uint32_t lds = lds_address(stage);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wm = wave & 1, wn = wave >> 1;
    const int count = a.meta->count, row_tiles = (count + TN - 1) / TN, tiles_d = (static_cast<int>(a.d) + TM - 1) / TM;
    const int width = static_cast<int>(a.width), w_tiles = (width + TN - 1) / TN;
    const int x_steps = (width + kStepK - 1) / kStepK, w_steps = (count + kStepK - 1) / kStepK;
    const int x_parts = sum_parts(row_tiles * tiles_d, x_steps), w_parts = sum_parts(w_tiles * tiles_d, w_steps);
    const int x_all = row_tiles * tiles_d * x_parts, w_all = w_tiles * tiles_d * w_parts;
    // the longer sums first, so that the short ones fill the end
    const bool x_first = x_steps / x_parts >= w_steps / w_parts;
    const int block = blockIdx.x, ahead = x_first ? x_all : w_all;
    if (block >= x_all + w_all) return;
    const bool dx = (block < ahead) == x_first;
    const int mine = block < ahead ? block : block - ahead;
    const int n_tiles = dx ? row_tiles : w_tiles, steps = dx ? x_steps : w_steps, parts = dx ? x_parts : w_parts, tiles = n_tiles * tiles_d;
    // the tiles of one stretch of G's rows (or columns) side by side: they share it in their L2
    const int id = xcd_remap32(mine, tiles * parts);
    const int rest = id / tiles_d;
    const int64_t td = id - rest * tiles_d, part = rest / n_tiles, tn = rest - static_cast<int>(part) * n_tiles;
    const int64_t per = (steps + parts - 1) / parts, from = part * per, to = from + per < steps ? from + per : steps;
    const int64_t n = to > from ? to - from : 0;
    floatx16 acc[IM][IN];
#pragma unroll
    for (int i = 0; i < IM; i++)
#pragma unroll
        for (int j = 0; j < IN; j++)
#pragma unroll
            for (int k = 0; k < 16; k++) acc[i][j][k] = 0.f;
    if (dx) {
        typename PX::A oa;
        typename PX::B ob;
#pragma unroll
        for (int p = 0; p < PL; p++) {
            oa.laid(p, a.w[p], a.w_rows, a.v0 + from * kStepK, td * TM);
            ob.laid(p, a.g[p], a.rows, tn * TN, from * kStepK);
        }
        PX::begin(oa, ob, n, lds);
        PX::run(oa, ob, n, lds, acc);
    } else {
        typename PW::A oa;
        typename PW::B ob;
#pragma unroll
        for (int p = 0; p < PL; p++) {
            oa.laid(p, a.x[p], a.rows, from * kStepK, td * TM);
            ob.laid(p, a.g[p], a.rows, from * kStepK, tn * TN);
        }
        PW::begin(oa, ob, n, lds);
        PW::run(oa, ob, n, lds, acc);
    }
    // the lane's row of the result is a column of the tile; four columns of d in each group of registers
    const int64_t c0 = td * TM + wm * (TM / 2) + 4 * (lane >> 5);
    const Scales scales(a.meta);
    const float max_sw = scales.max_sw, cf = scales.down();
#pragma unroll
    for (int j = 0; j < IN; j++) {
        const int64_t r = tn * TN + wn * (TN / 2) + j * 32 + (lane & 31);
        const bool out = parts == 1 && (!dx || a.single);
        if (dx ? r >= count : r >= width) continue;
        const float by = !out ? 1.f : dx ? cf / scales.row(a.sx[r], a.dls[r]) : cf * (max_sw / scales.table(a.sw[a.v0 + r]));
        const float and_by = dx && out ? max_sw : 1.f;
        const int64_t to_row = !out ? 0 : dx ? a.listed[r] : a.v0 + r;
        float *at = dx ? a.px + (part * row_tiles * TN + r) * a.ld : a.pw + (part * a.piece + r) * a.ld;
#pragma unroll
        for (int i = 0; i < IM; i++)
#pragma unroll
            for (int q = 0; q < 4; q++) {
                const int64_t c = c0 + i * 32 + q * 8;
                float v[4];
#pragma unroll
                for (int k = 0; k < 4; k++) v[k] = acc[i][j][q * 4 + k] * and_by * by;
                if (out) {
                    if (c < a.d) store4<BF16>(dx ? a.dx : a.dw, to_row * a.d, c, a.d, v);
                } else {
                    float4 *p = reinterpret_cast<float4 *>(at + c);
                    float4 s = make_float4(v[0], v[1], v[2], v[3]);
                    if (dx && a.add) {
                        const float4 o = *p;
                        s.x += o.x, s.y += o.y, s.z += o.z, s.w += o.w;
                    }
                    *p = s;
                }
            }
    }
}

struct Finish {
    const Meta *meta;
    const int *place;
    const float *px, *pw, *sx, *sw, *dls;
    int64_t ld, d, tokens, v0, width, piece, x_width;  // x_width: entries of the first piece
    int tile_n;
    void *dx, *dw;
    int x_rows, w_rows;  // rows of a workgroup
    bool single;         // dx of one piece: written already where the sums were not cut
    // db
    const float *db_part;
    Picked picked;  // NULL: taken off already
    float *db;
    int x_blocks, w_blocks;  // workgroups of dx, then of dW, then of db
};

// four columns of the sum of `parts` rows, `stride` floats apart; loads of eight are under way at once
__device__ __forceinline__ void sum_rows(const float *p, int parts, int64_t stride, float (&v)[4]) {
    int i = 0;
    for (; i + 8 <= parts; i += 8) {
        float4 s[8];
#pragma unroll
        for (int k = 0; k < 8; k++) s[k] = *reinterpret_cast<const float4 *>(p + (i + k) * stride);
#pragma unroll
        for (int k = 0; k < 8; k++) v[0] += s[k].x, v[1] += s[k].y, v[2] += s[k].z, v[3] += s[k].w;
    }
    for (; i < parts; i++) {
        const float4 s = *reinterpret_cast<const float4 *>(p + i * stride);
        v[0] += s.x, v[1] += s.y, v[2] += s.z, v[3] += s.w;
    }
}

// dx of every token: its row's parts, or 0.  A workgroup takes x_rows tokens, 4 columns a lane.
template <bool BF16>
__device__ __forceinline__ void finish_x(const Finish &a, int block) {
    const int row_tiles = (a.meta->count + a.tile_n - 1) / a.tile_n;
    // (every piece is cut as the first is: it sums as many steps, the last fewer)
    const int parts = sum_parts(row_tiles * ((static_cast<int>(a.d) + kGradM - 1) / kGradM), static_cast<int>((a.x_width + kStepK - 1) / kStepK));
    const Scales scales(a.meta);
    const float max_sw = scales.max_sw, cf = scales.down();
    const unsigned vecs = (static_cast<unsigned>(a.d) + 3) / 4;
    const int64_t first = static_cast<int64_t>(block) * a.x_rows;
    const unsigned n = static_cast<unsigned>(a.tokens - first < a.x_rows ? a.tokens - first : a.x_rows) * vecs;
    for (unsigned i = threadIdx.x; i < n; i += kThreads) {
        const unsigned in = i / vecs, c = (i - in * vecs) * 4;
        const int64_t t = first + in;
        const int r = a.place[t];
        if (r >= 0 && parts == 1 && a.single) continue;
        float v[4] = {0.f, 0.f, 0.f, 0.f};
        if (r >= 0) {
            sum_rows(a.px + r * a.ld + c, parts, static_cast<int64_t>(row_tiles) * a.tile_n * a.ld, v);
            const float by = cf / scales.row(a.sx[r], a.dls[r]);
#pragma unroll
            for (int k = 0; k < 4; k++) v[k] = v[k] * max_sw * by;
        }
        store4<BF16>(a.dx, t * a.d, c, a.d, v);
    }
}

// dW of a piece whose sums were cut
template <bool BF16>
__device__ __forceinline__ void finish_w(const Finish &a, int block) {
    const int tiles = static_cast<int>((a.width + a.tile_n - 1) / a.tile_n * ((a.d + kGradM - 1) / kGradM));
    const int parts = sum_parts(tiles, (a.meta->count + kStepK - 1) / kStepK);
    if (parts == 1) return;
    const Scales scales(a.meta);
    const float max_sw = scales.max_sw, cf = scales.down();
    const unsigned vecs = (static_cast<unsigned>(a.d) + 3) / 4;
    const int64_t first = static_cast<int64_t>(block) * a.w_rows;
    const unsigned n = static_cast<unsigned>(a.width - first < a.w_rows ? a.width - first : a.w_rows) * vecs;
    for (unsigned i = threadIdx.x; i < n; i += kThreads) {
        const unsigned in = i / vecs, c = (i - in * vecs) * 4;
        const int64_t r = first + in;
        float v[4] = {0.f, 0.f, 0.f, 0.f};
        sum_rows(a.pw + r * a.ld + c, parts, a.piece * a.ld, v);
        const float by = cf * (max_sw / scales.table(a.sw[a.v0 + r]));
#pragma unroll
        for (int k = 0; k < 4; k++) v[k] *= by;
        store4<BF16>(a.dw, (a.v0 + r) * a.d, c, a.d, v);
    }
}

// db of a piece: sums of q over the token tiles, less the taught probabilities.  32 entries a workgroup, eight threads an
// entry (one: 65 us for 829 sums of 97 entries, eight 20).
constexpr int kDbEntries = 32;
__device__ __forceinline__ void finish_b(const Finish &a, int block) {
    constexpr int SLICES = kThreads / kDbEntries;
    __shared__ double sums[SLICES][kDbEntries];
    __shared__ unsigned long long taken[SLICES][kDbEntries];
    const int in = threadIdx.x % kDbEntries, slice = threadIdx.x / kDbEntries;
    const int64_t v = static_cast<int64_t>(block) * kDbEntries + in;
    const double unit = ldexp(1.0, scale_exp(a.meta->largest(kMaxDl)) - 40);  // (by all lanes)
    const int n = (a.meta->count + kTileN - 1) / kTileN * 2;
    double s[4] = {0.0, 0.0, 0.0, 0.0};  // (up to 65536 tiles' sums)
    unsigned long long less = 0;
    if (v < a.width) {
        int i = slice;
        for (; i + 3 * SLICES < n; i += 4 * SLICES)
#pragma unroll
            for (int k = 0; k < 4; k++) s[k] += a.db_part[(i + k * SLICES) * a.piece + v];
        for (; i < n; i += SLICES) s[0] += a.db_part[i * a.piece + v];
        if (a.picked.sums)
            for (int c = slice; c < a.picked.copies; c += SLICES) less += a.picked.sums[c * a.picked.ld + a.v0 + v];
    }
    sums[slice][in] = (s[0] + s[1]) + (s[2] + s[3]);
    taken[slice][in] = less;
    __syncthreads();
    if (slice != 0 || v >= a.width) return;
    double sum = 0.0;
    less = 0;
#pragma unroll
    for (int i = 0; i < SLICES; i++) sum += sums[i][in], less += taken[i][in];
    a.db[a.v0 + v] = static_cast<float>(sum - static_cast<double>(static_cast<long long>(less)) * unit);
}

template <bool BF16>
__global__ __launch_bounds__(kThreads) void finish_kernel(Finish a) {
    const int block = blockIdx.x;
    if (block < a.x_blocks)
        finish_x<BF16>(a, block);
    else if (block < a.x_blocks + a.w_blocks)
        finish_w<BF16>(a, block - a.x_blocks);
    else
        finish_b(a, block - a.x_blocks - a.w_blocks);
}

// ---------------------------------------------------------------- workspace

class Layout {
   public:
    size_t take(int64_t bytes) {
        const size_t at = total;
        total += static_cast<size_t>(up(bytes, 256));
        return at;
    }
    size_t total = 0;
};

constexpr int kRowPad = 256, kVocabPad = 256;
constexpr int64_t kPieceBytes = int64_t{1} << 30;  // of G at once (256 entries of the vocabulary at least)

bool few(int64_t tokens) { return tokens <= kFewTokens; }

// bf16 rows of whole steps are read as they lie, through 32-bit offsets, where that is faster: half cache lines make the
// products of tokens V d slower (16384 x 768 into 30000: 900 against 750 us), laying out costs (tokens + V) d (45 us).
bool raw_rows(bool bf16, int64_t tokens, int64_t vocab, int d) {
    return bf16 && d % kStepK == 0 && tokens * d * 2 < (int64_t{1} << 32) && tokens * vocab < 4096 * (tokens + vocab);
}

int64_t row_ld(int d) { return up(d, kGradM); }

// workgroups of logits_kernel at most: token tiles times parts
int64_t logits_grid(int64_t tokens) {
    const int64_t four = 4 * ((tokens + kTileN - 1) / kTileN);
    return four > 2 * kSlots ? four : 2 * kSlots;
}

// ids of a row, at least one kNoId behind them, in whole 16 bytes
int sorted_row(int top) { return (top + 4) / 4 * 4; }

// Whether the taught ids' logits are taken from the tiles, by order, instead of made as dot products: those read top rows of the table
// a token (16384 x 32 of 768 fp32: 2250 against 2370 us), the order is a launch more (200 x 20 of 384: 55 against 43) and a search in
// every tile (3559 x 46 of 64 columns: 85 against 56).
bool sorts(int64_t tokens, int top, int d) { return top > 0 && top <= kSortedTop && tokens * top * d >= int64_t{1} << 24; }

struct ForwardPlan {
    size_t counts, masks, meta, rows, part, hit, sorted, sx, sw, x[2], w[2];
    size_t total;
    int64_t few_blocks;
    ForwardPlan(bool bf16, int64_t tokens, int top, int64_t vocab, int d) {  // top = 0: cross entropy
        Layout l;
        counts = masks = meta = rows = hit = sorted = sx = sw = x[0] = x[1] = w[0] = w[1] = 0;
        const int64_t groups = (vocab + 15) / 16;
        few_blocks = groups < kFewBlocks ? groups : kFewBlocks;
        if (few(tokens)) {
            part = l.take(few_blocks * kFewTokens * 8);
            hit = l.take(top == 0 ? kFewTokens * 4 : 0);
        } else {
            counts = l.take((tokens + kCountTokens - 1) / kCountTokens * 4);
            masks = l.take(up(tokens, kCountTokens) / 8);
            meta = l.take(sizeof(Meta));
            rows = l.take(tokens * 4);
            part = l.take(logits_grid(tokens) * kTileN * 8);
            hit = l.take(top == 0 ? tokens * 4 : 0);
            sorted = l.take(sorts(tokens, top, d) ? tokens * sorted_row(top) * 4 : 0);
            if (!raw_rows(bf16, tokens, vocab, d)) {
                const int64_t tp = up(tokens, kTileN), vp = up(vocab, kVocabPad);
                sx = l.take(tp * 4);
                sw = l.take(vp * 4);
                for (int p = 0; p < (bf16 ? 1 : 2); p++) {
                    x[p] = l.take(tp * row_ld(d) * 2);
                    w[p] = l.take(vp * row_ld(d) * 2);
                }
            }
        }
        total = l.total;
    }
};

// Up to 16 tokens: 30000 x 768 fp32 71 against 127 us of the general form, 2000 x 768 27 against 62, 30000 x 2048 fp32 242 against
// 308 (bf16 170 against 185), one token into 2000 x 2048 35 against 77.  17 to 32 tokens hold twice the
// registers and read x twice as often: 39 against 63 us at 2000 x 768, but 135 (bf16 119) against 127 (92) at 30000 x 768.
bool few_backward(int64_t tokens, int top, int64_t vocab, int d) {
    if (tokens == 0 || tokens * top > kFewEntries) return false;
    return tokens <= 16 ? d <= 2 * kFewColumns : tokens <= kFewBackward && d <= kFewColumns && vocab * d <= int64_t{1} << 23;
}
size_t few_backward_bytes(int64_t tokens, int64_t vocab, int d) {
    const int64_t groups = (vocab + 15) / 16;
    return static_cast<size_t>(groups < kFewBackwardBlocks ? groups : kFewBackwardBlocks) * (tokens <= 16 ? 16 : 32) * d * 4;
}

struct BackwardPlan {
    size_t counts, masks, meta, rows, place, sx, dls, lse2, sw, x[2], w[2], g[2], px, pw, db, picked;
    size_t total;
    int64_t piece, pieces, ld;
    int tile_n;  // of the gradients' products
    BackwardPlan(bool bf16, int64_t tokens, int64_t vocab, int d) {
        Layout l;
        const int planes = bf16 ? 1 : 2;
        tile_n = grad_n(bf16);
        ld = row_ld(d);
        const int64_t tp = up(tokens, kRowPad), vp = up(vocab, kVocabPad);
        const int64_t room = kPieceBytes / (2 * planes * (tp > 0 ? tp : kRowPad)) / kVocabPad * kVocabPad;
        piece = room < kVocabPad ? kVocabPad : room > vp ? vp : room;
        pieces = (vocab + piece - 1) / piece;
        piece = up((vocab + pieces - 1) / pieces, kVocabPad);
        pieces = (vocab + piece - 1) / piece;
        counts = l.take((tokens / kCountTokens + 1) * 4);
        masks = l.take(up(tokens, kCountTokens) / 8);
        meta = l.take(sizeof(Meta));
        rows = l.take(tokens * 4);
        place = l.take(tokens * 4);
        sx = l.take(tp * 4);
        dls = l.take(tp * 4);
        lse2 = l.take(tp * 4);
        sw = l.take(vp * 4);
        x[1] = w[1] = g[1] = 0;
        for (int p = 0; p < planes; p++) {
            x[p] = l.take(tp * ld * 2);
            w[p] = l.take(vp * ld * 2);
            g[p] = l.take(tp * piece * 2);
        }
        // parts of dx: as many rows as the tokens have, or as the card's slots take if that is more and the sum is long enough
        const int64_t tiles = (tokens + tile_n - 1) / tile_n, most = (piece + kStepK - 1) / kStepK / 16;
        int64_t cut = kGradSlots / (ld / kGradM);
        if (cut > tiles * most) cut = tiles * most;
        px = l.take((cut > tiles ? cut : tiles) * tile_n * ld * 4);
        const int parts = sum_parts((piece + tile_n - 1) / tile_n * (ld / kGradM), (tokens + kStepK - 1) / kStepK);
        const int64_t last = vocab - (pieces - 1) * piece;
        const int parts_last = sum_parts((last + tile_n - 1) / tile_n * (ld / kGradM), (tokens + kStepK - 1) / kStepK);
        const int parts_most = parts > parts_last ? parts : parts_last;
        pw = l.take(parts_most > 1 ? parts_most * piece * ld * 4 : 0);
        db = l.take((tokens + kTileN - 1) / kTileN * 2 * piece * 4);
        picked = l.take(picked_copies(vocab) * picked_ld(vocab) * 8);
        total = l.total;
    }
};

template <typename T>
T *at(void *ws, size_t offset) {
    return reinterpret_cast<T *>(static_cast<char *>(ws) + offset);
}

template <typename... K, typename... A>
void run(void (*kernel)(K...), int64_t blocks, hipStream_t stream, A... args) {
    hipLaunchKernelGGL(kernel, dim3(static_cast<unsigned>(blocks)), dim3(kThreads), 0, stream, static_cast<K>(args)...);
}

// rows of a workgroup of the finishing kernels: about 2048 workgroups, where each has a vector for every thread
int finish_rows(int64_t rows, int d) {
    const int least = (4 * kThreads + d - 1) / d;
    const int64_t n = (rows + 2047) / 2048;
    return n < least ? least : n > 1024 ? 1024 : static_cast<int>(n);
}

#define YOSO_HIP(expr)                        \
    do {                                      \
        const hipError_t _e = (expr);         \
        if (_e != hipSuccess) return _e;      \
    } while (0)

// Calls f with the form of few_backward_kernel for so many tokens (16 or 32) and columns.
template <bool BF16, typename F>
void with_few_columns(int rows, int d, F f) {
    if (rows == 16)
        d <= 256    ? f(few_backward_kernel<BF16, 1, 1>)
        : d <= 1024 ? f(few_backward_kernel<BF16, 1, 4>)
                    : f(few_backward_kernel<BF16, 1, 8>);
    else
        d <= 256 ? f(few_backward_kernel<BF16, 2, 1>) : f(few_backward_kernel<BF16, 2, 4>);
}
template <typename F>
void with_few_form(bool bf16, int rows, int d, F f) {
    bf16 ? with_few_columns<true>(rows, d, f) : with_few_columns<false>(rows, d, f);
}

hipError_t launch_list(const Taught &a, int *counts, uint64_t *masks, Meta *meta, int *rows, int *place, float *loss, float *lse, float *logq,
                       hipStream_t stream) {
    KernelTimer timer("loss_rows_kernel", stream);
    // (one CU reads a cache line for each token of a teacher's lists: 4000 of them take 13 us)
    if (a.tokens <= (a.teacher ? kListThreads : kListTokens)) {
        hipLaunchKernelGGL(list_kernel, dim3(1), dim3(kListThreads), 0, stream, a, meta, rows, place, loss, lse, logq);
        return hipGetLastError();
    }
    const int64_t grid = (a.tokens + kCountTokens - 1) / kCountTokens;
    run(count_kernel, grid, stream, a, counts, masks, meta);
    YOSO_HIP(hipGetLastError());
    run(rows_kernel, grid, stream, a, counts, masks, meta, rows, place, loss, lse, logq);
    return hipGetLastError();
}

hipError_t launch_lay(const Lay &table, const Lay &x, bool bf16, hipStream_t stream) {
    KernelTimer timer("loss_lay_kernel", stream);
    const int lanes = x.ld <= 128 ? 16 : x.ld <= 256 ? 32 : 64;
    const auto blocks = [&](const Lay &a) {
        const int64_t need = (a.padded * lanes + kThreads - 1) / kThreads;
        return static_cast<int>(need < kLayBlocks ? need : kLayBlocks);
    };
    const int first = blocks(table), all = first + blocks(x);
    if (lanes == 16) bf16 ? run(lay_kernel<true, 16>, all, stream, table, x, first) : run(lay_kernel<false, 16>, all, stream, table, x, first);
    if (lanes == 32) bf16 ? run(lay_kernel<true, 32>, all, stream, table, x, first) : run(lay_kernel<false, 32>, all, stream, table, x, first);
    if (lanes == 64) bf16 ? run(lay_kernel<true, 64>, all, stream, table, x, first) : run(lay_kernel<false, 64>, all, stream, table, x, first);
    return hipGetLastError();
}

}  // namespace

size_t vocab_loss_workspace(bool bf16, int64_t tokens, int top, int64_t vocab, int d) {
    return tokens > 0 ? ForwardPlan(bf16, tokens, top, vocab, d).total : 0;
}

size_t vocab_loss_backward_workspace(bool bf16, int64_t tokens, int top, int64_t vocab, int d) {
    return few_backward(tokens, top, vocab, d) ? few_backward_bytes(tokens, vocab, d) : BackwardPlan(bf16, tokens, vocab, d).total;
}

size_t vocab_loss_backward_workspace_any(bool bf16, int64_t tokens, int64_t vocab, int d) {
    const size_t few = vocab_loss_backward_workspace(bf16, tokens, 1, vocab, d), many = vocab_loss_backward_workspace(bf16, tokens, kMaxTop, vocab, d);
    return few > many ? few : many;
}

hipError_t launch_vocab_loss(const VocabLoss &a, bool bf16, bool wide, hipStream_t stream) {
    if (a.tokens == 0) return hipSuccess;
    const ForwardPlan p(bf16, a.tokens, a.teacher ? a.top : 0, a.vocab, a.d);
    const Taught taught{a.ids, wide, a.top, a.teacher, nullptr, a.tokens, a.vocab};
    Loss out{taught, a.x, a.table, a.bias, a.d, a.scale, nullptr, nullptr, at<float2>(a.workspace, p.part), static_cast<int>(p.few_blocks),
             0, a.loss, a.lse, a.logq, nullptr, false};
    if (few(a.tokens)) {
        out.hit = a.teacher ? nullptr : at<float>(a.workspace, p.hit);
        out.left = a.teacher && a.tokens * a.top <= kFewEntries;
        const Few f{a.x, a.table, a.bias, a.tokens, a.vocab, a.d, a.scale, at<float2>(a.workspace, p.part), taught,
                    a.teacher ? nullptr : at<float>(a.workspace, p.hit), out.left ? a.logq : nullptr};
        {
            KernelTimer timer("loss_few_kernel", stream);
            const int64_t grid = p.few_blocks;
            const int nt = a.tokens <= 16 ? 1 : a.tokens <= 32 ? 2 : 4;
            if (bf16) {
                if (nt == 1) run(few_kernel<true, 1>, grid, stream, f);
                if (nt == 2) run(few_kernel<true, 2>, grid, stream, f);
                if (nt == 4) run(few_kernel<true, 4>, grid, stream, f);
            } else {
                if (nt == 1) run(few_kernel<false, 1>, grid, stream, f);
                if (nt == 2) run(few_kernel<false, 2>, grid, stream, f);
                if (nt == 4) run(few_kernel<false, 4>, grid, stream, f);
            }
            YOSO_HIP(hipGetLastError());
        }
        KernelTimer timer("loss_kernel", stream);
        bf16 ? run(loss_kernel<true, 1>, a.tokens, stream, out)
             : run(loss_kernel<false, 1>, a.tokens, stream, out);
        return hipGetLastError();
    }
    int *rows = at<int>(a.workspace, p.rows);
    Meta *meta = at<Meta>(a.workspace, p.meta);
    YOSO_HIP(launch_list(taught, at<int>(a.workspace, p.counts), at<uint64_t>(a.workspace, p.masks), meta, rows, nullptr, a.loss, a.lse, a.logq, stream));
    const bool raw = raw_rows(bf16, a.tokens, a.vocab, a.d);
    const int tile_m = bf16 ? 256 : 128;
    Logits l{};
    l.rows = rows;
    l.d = a.d;
    l.bias = a.bias;
    l.scale = a.scale;
    l.vocab = l.v1 = a.vocab;
    l.meta = meta;
    l.part = at<float2>(a.workspace, p.part);
    l.taught = taught;
    l.hit = a.teacher ? nullptr : at<float>(a.workspace, p.hit);
    if (a.teacher && sorts(a.tokens, a.top, a.d)) {
        KernelTimer timer("loss_sort_kernel", stream);
        l.sorted = at<int>(a.workspace, p.sorted);
        l.sorted_ld = sorted_row(a.top);
        l.picks = a.logq;
        const int64_t need = (a.tokens + 3) / 4;
        run(sort_ids_kernel, need < 2048 ? need : 2048, stream, taught, rows, meta, at<int>(a.workspace, p.sorted), l.sorted_ld);
        YOSO_HIP(hipGetLastError());
    }
    if (raw) {
        l.w[0] = static_cast<const char *>(a.table);
        l.x[0] = static_cast<const char *>(a.x);
        l.ld = 2 * static_cast<int64_t>(a.d);
    } else {
        const int64_t ld = row_ld(a.d);
        Lay w{a.table, a.vocab, up(a.vocab, kVocabPad), a.d, static_cast<int>(ld), at<half8>(a.workspace, p.w[0]),
              at<half8>(a.workspace, p.w[1]), at<float>(a.workspace, p.sw), nullptr, nullptr, nullptr, nullptr, {}, a.scale, nullptr, nullptr,
              meta, true, {}};
        Lay x{a.x, a.tokens, up(a.tokens, kTileN), a.d, static_cast<int>(ld), at<half8>(a.workspace, p.x[0]),
              at<half8>(a.workspace, p.x[1]), at<float>(a.workspace, p.sx), rows, nullptr, nullptr, nullptr, {}, a.scale, nullptr, nullptr,
              meta, false, {}};
        YOSO_HIP(launch_lay(w, x, bf16, stream));
        for (int i = 0; i < 2; i++) {
            l.w[i] = at<char>(a.workspace, p.w[i]);
            l.x[i] = at<char>(a.workspace, p.x[i]);
        }
        l.sw = w.mult;
        l.sx = x.mult;
        l.w_rows = w.padded;
        l.x_rows = x.padded;
    }
    {
        KernelTimer timer("loss_logits_kernel", stream);
        const int64_t grid = logits_grid(a.tokens);
        if (raw)
            l.sorted ? run(logits_kernel<1, 3, true>, grid, stream, l) : run(logits_kernel<1, 0, true>, grid, stream, l);
        else if (bf16)
            l.sorted ? run(logits_kernel<1, 3, false>, grid, stream, l) : run(logits_kernel<1, 0, false>, grid, stream, l);
        else
            l.sorted ? run(logits_kernel<2, 3, false>, grid, stream, l) : run(logits_kernel<2, 0, false>, grid, stream, l);
        YOSO_HIP(hipGetLastError());
    }
    out.rows = rows;
    out.meta = meta;
    out.tile_m = tile_m;
    KernelTimer timer("loss_kernel", stream);
    out.hit = l.hit;
    if (l.hit) {
        if (a.tokens <= 4096)
            run(target_loss_kernel<16>, (a.tokens + 15) / 16, stream, out);
        else
            run(target_loss_kernel<64>, (a.tokens + 63) / 64, stream, out);
        return hipGetLastError();
    }
    if (l.sorted) {
        run(picked_loss_kernel, (a.tokens + 3) / 4, stream, out);
        return hipGetLastError();
    }
    // (a workgroup a row as long as the card is not full of waves otherwise)
    if (a.tokens <= 4096)
        bf16 ? run(loss_kernel<true, 1>, a.tokens, stream, out) : run(loss_kernel<false, 1>, a.tokens, stream, out);
    else
        bf16 ? run(loss_kernel<true, 4>, (a.tokens + 3) / 4, stream, out) : run(loss_kernel<false, 4>, (a.tokens + 3) / 4, stream, out);
    return hipGetLastError();
}

hipError_t launch_vocab_loss_backward(const VocabLossBackward &a, bool bf16, bool wide, hipStream_t stream) {
    void *ws = a.workspace;
    const Taught taught{a.ids, wide, a.top, a.teacher, a.dloss, a.tokens, a.vocab};
    if (few_backward(a.tokens, a.top, a.vocab, a.d)) {
        FewBackward f{taught, a.x, a.table, a.bias, a.logq, a.lse, a.tokens, a.vocab, a.d, a.scale, a.dtable, a.dbias, static_cast<float *>(ws)};
        const int64_t groups = (a.vocab + 15) / 16;
        const int parts = static_cast<int>(groups < kFewBackwardBlocks ? groups : kFewBackwardBlocks), rows = a.tokens <= 16 ? 16 : 32;
        {
            KernelTimer timer("loss_few_backward_kernel", stream);
            with_few_form(bf16, rows, a.d, [&](auto kernel) { run(kernel, parts, stream, f); });
            YOSO_HIP(hipGetLastError());
        }
        KernelTimer timer("loss_finish_kernel", stream);
        f.dw = a.dx;
        const dim3 grid(static_cast<unsigned>((a.d + 63) / 64), static_cast<unsigned>(a.tokens));
        if (bf16)
            hipLaunchKernelGGL(few_finish_kernel<true>, grid, dim3(kThreads), 0, stream, f, parts, rows);
        else
            hipLaunchKernelGGL(few_finish_kernel<false>, grid, dim3(kThreads), 0, stream, f, parts, rows);
        return hipGetLastError();
    }
    const BackwardPlan p(bf16, a.tokens, a.vocab, a.d);
    Meta *meta = at<Meta>(ws, p.meta);
    int *rows = at<int>(ws, p.rows), *place = at<int>(ws, p.place);
    const Picked picked{a.dbias && a.teacher ? at<unsigned long long>(ws, p.picked) : nullptr, picked_ld(a.vocab), picked_copies(a.vocab)};
    YOSO_HIP(launch_list(taught, at<int>(ws, p.counts), at<uint64_t>(ws, p.masks), meta, rows, place, nullptr, nullptr, nullptr, stream));
    const int64_t ld = p.ld, tp = up(a.tokens, kRowPad);
    Lay w{a.table, a.vocab, up(a.vocab, kVocabPad), a.d, static_cast<int>(ld), at<half8>(ws, p.w[0]), at<half8>(ws, p.w[1]),
          at<float>(ws, p.sw), nullptr, nullptr, nullptr, nullptr, {}, a.scale, nullptr, nullptr, meta, true, picked};
    Lay x{a.x, a.tokens, tp, a.d, static_cast<int>(ld), at<half8>(ws, p.x[0]), at<half8>(ws, p.x[1]), at<float>(ws, p.sx), rows, a.dloss,
          a.lse, a.logq, taught, a.scale, at<float>(ws, p.dls), at<float>(ws, p.lse2), meta, false, {}};
    YOSO_HIP(launch_lay(w, x, bf16, stream));
    const int64_t row_tiles = (a.tokens + kTileN - 1) / kTileN, tiles_d = ld / kGradM;
    const int tile_m = bf16 ? 256 : 128;
    for (int64_t i = 0; i < p.pieces; i++) {
        const int64_t v0 = i * p.piece, v1 = v0 + p.piece < a.vocab ? v0 + p.piece : a.vocab, width = v1 - v0;
        Logits l{};
        Gradients g{};
        Pick pick{taught, a.logq, a.scale, rows, meta, x.mult, x.dls, w.mult, v0, v1, {}, tp, picked, at<float>(ws, p.db), p.piece};
        for (int k = 0; k < 2; k++) {
            l.w[k] = at<char>(ws, p.w[k]);
            l.x[k] = at<char>(ws, p.x[k]);
            l.g[k] = pick.g[k] = at<_Float16>(ws, p.g[k]);
            g.x[k] = l.x[k];
            g.w[k] = l.w[k];
            g.g[k] = at<char>(ws, p.g[k]);
        }
        if (a.tokens > 0) {
            l.sw = w.mult;
            l.sx = x.mult;
            l.w_rows = up(a.vocab, kVocabPad);
            l.x_rows = tp;
            l.d = a.d;
            l.bias = a.bias;
            l.scale = a.scale;
            l.vocab = a.vocab;
            l.v0 = v0;
            l.v1 = v1;
            l.meta = meta;
            l.dls = x.dls;
            l.lse2 = x.lse2;
            l.taught = taught;
            l.loss = a.teacher ? nullptr : a.logq;
            l.rows = rows;
            l.piece = p.piece;
            l.db = at<float>(ws, p.db);
            const int64_t n = row_tiles * ((width + tile_m - 1) / tile_m);
            {
                KernelTimer timer("loss_grad_logits_kernel", stream);
                if (bf16 && a.dbias) run(logits_kernel<1, 2, false>, n, stream, l);
                if (bf16 && !a.dbias) run(logits_kernel<1, 1, false>, n, stream, l);
                if (!bf16 && a.dbias) run(logits_kernel<2, 2, false>, n, stream, l);
                if (!bf16 && !a.dbias) run(logits_kernel<2, 1, false>, n, stream, l);
                YOSO_HIP(hipGetLastError());
            }
            if (a.teacher) {
                KernelTimer timer("loss_pick_kernel", stream);
                const int64_t need = (a.tokens + 3) / 4, grid = need < 2048 ? need : 2048;
                if (a.top <= 64)
                    bf16 ? run(pick_kernel<1, false>, grid, stream, pick) : run(pick_kernel<2, false>, grid, stream, pick);
                else
                    bf16 ? run(pick_kernel<1, true>, grid, stream, pick) : run(pick_kernel<2, true>, grid, stream, pick);
                YOSO_HIP(hipGetLastError());
            }
        }
        g.ld = ld;
        g.piece = p.piece;
        g.rows = tp;
        g.w_rows = up(a.vocab, kVocabPad);
        g.d = a.d;
        g.v0 = v0;
        g.vocab = a.vocab;
        g.width = width;
        g.meta = meta;
        g.sw = w.mult;
        g.px = at<float>(ws, p.px);
        g.pw = at<float>(ws, p.pw);
        g.add = i > 0;
        g.dw = a.dtable;
        g.single = p.pieces == 1;
        g.listed = rows;
        g.sx = x.mult;
        g.dls = x.dls;
        g.dx = a.dx;
        const int64_t tx = (a.tokens + p.tile_n - 1) / p.tile_n * tiles_d, tw = (width + p.tile_n - 1) / p.tile_n * tiles_d;
        const int64_t n = (tx > kGradSlots ? tx : a.tokens == 0 ? 0 : kGradSlots) + (tw > kGradSlots ? tw : kGradSlots);
        {
            KernelTimer timer("loss_gradients_kernel", stream);
            bf16 ? run(gradients_kernel<true>, n, stream, g)
                 : run(gradients_kernel<false>, n, stream, g);
            YOSO_HIP(hipGetLastError());
        }
        // (both sums may have been cut; the host knows only how many tokens there are at most)
        Finish f{};
        f.meta = meta;
        f.place = place;
        f.px = g.px;
        f.pw = g.pw;
        f.sx = x.mult;
        f.sw = w.mult;
        f.dls = x.dls;
        f.ld = ld;
        f.d = a.d;
        f.tokens = a.tokens;
        f.v0 = v0;
        f.width = width;
        f.piece = p.piece;
        f.x_width = p.pieces > 1 ? p.piece : a.vocab;
        f.tile_n = p.tile_n;
        f.dx = a.dx;
        f.dw = a.dtable;
        f.x_rows = finish_rows(a.tokens, a.d);
        f.w_rows = finish_rows(width, a.d);
        f.single = p.pieces == 1;
        f.db_part = l.db;
        f.picked = picked;
        f.db = a.dbias;
        f.x_blocks = i + 1 < p.pieces ? 0 : static_cast<int>((a.tokens + f.x_rows - 1) / f.x_rows);
        f.w_blocks = sum_parts(static_cast<int>(tw), static_cast<int>((a.tokens + kStepK - 1) / kStepK)) > 1
                         ? static_cast<int>((width + f.w_rows - 1) / f.w_rows)
                         : 0;
        const int64_t finishing = f.x_blocks + f.w_blocks + (a.dbias ? (width + kDbEntries - 1) / kDbEntries : 0);
        if (finishing > 0) {
            KernelTimer timer("loss_finish_kernel", stream);
            bf16 ? run(finish_kernel<true>, finishing, stream, f) : run(finish_kernel<false>, finishing, stream, f);
            YOSO_HIP(hipGetLastError());
        }
    }
    return hipSuccess;
}

}  // namespace yoso
