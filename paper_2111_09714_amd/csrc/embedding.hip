// Embedding lookup with positions, and its gradient (gfx950).
//
//   y[t] = scale table[ids[t]] + pos[t mod n];  ids outside [0, vocab) have no row (0)
//   dtable[v] = scale sum_{t : ids[t] = v} dy[t],   dpos[p] = sum_b dy[b n + p]
#include "common.h"
#include "launch.h"
#include "timing.h"

namespace yoso {

namespace {

constexpr int kThreads = 256;

template <bool BF16>
__device__ __forceinline__ void store1(void *base, int64_t off, float v) {
    if constexpr (BF16)
        static_cast<__bf16 *>(base)[off] = static_cast<__bf16>(v);
    else
        static_cast<float *>(base)[off] = v;
}

template <bool BF16, typename ID>
__global__ __launch_bounds__(kThreads) void embedding_kernel(const ID *ids, const void *table, const void *pos,
                                                             int64_t tokens, int64_t n, int64_t vocab, int d,
                                                             float scale, void *y) {
    for (int64_t t = blockIdx.x; t < tokens; t += gridDim.x) {
        const int64_t id = ids[t];
        const bool named = id >= 0 && id < vocab;
        for (int c = threadIdx.x; c < d; c += kThreads) {
            const float p = pos ? load1<BF16>(pos, (t % n) * d + c) : 0.f;
            store1<BF16>(y, t * d + c, named ? fmaf(scale, load1<BF16>(table, id * d + c), p) : p);
        }
    }
}

// one row of the table per workgroup: it looks through all ids for its own
template <bool BF16, typename ID>
__global__ __launch_bounds__(kThreads) void embedding_bwd_kernel(const ID *ids, const void *dy, int64_t tokens,
                                                                 int64_t vocab, int d, float scale, void *dtable) {
    __shared__ unsigned long long hits[kThreads / 64];
    for (int64_t v = blockIdx.x; v < vocab; v += gridDim.x) {
        for (int c0 = 0; c0 < d; c0 += kThreads) {
            const int c = c0 + threadIdx.x;
            float a = 0.f;
            for (int64_t t0 = 0; t0 < tokens; t0 += kThreads) {
                const int64_t t = t0 + threadIdx.x;
                const unsigned long long m = __ballot(t < tokens && static_cast<int64_t>(ids[t]) == v);
                __syncthreads();
                if ((threadIdx.x & 63) == 0) hits[threadIdx.x >> 6] = m;
                __syncthreads();
                for (int w = 0; w < kThreads / 64; w++)
                    for (unsigned long long h = hits[w]; h; h &= h - 1)
                        if (c < d) a += load1<BF16>(dy, (t0 + 64 * w + __ffsll(h) - 1) * d + c);
            }
            if (c < d) store1<BF16>(dtable, v * d + c, a * scale);
        }
    }
}

template <bool BF16>
__global__ __launch_bounds__(kThreads) void embedding_pos_kernel(const void *dy, int64_t tokens, int64_t n, int d,
                                                                 void *dpos) {
    for (int64_t p = blockIdx.x; p < n; p += gridDim.x)
        for (int c = threadIdx.x; c < d; c += kThreads) {
            float a = 0.f;
            for (int64_t t = p; t < tokens; t += n) a += load1<BF16>(dy, t * d + c);
            store1<BF16>(dpos, p * d + c, a);
        }
}

unsigned row_grid(int64_t rows) { return static_cast<unsigned>(rows < 65536 ? rows : 65536); }

}  // namespace

size_t embedding_backward_workspace(bool bf16, int64_t tokens, int64_t n, int64_t vocab, int d) { return 0; }

hipError_t launch_embedding(const Embedding &a, bool bf16, bool wide, hipStream_t stream) {
    if (a.tokens == 0) return hipSuccess;
    KernelTimer timer("embedding_kernel", stream);
    const dim3 grid(row_grid(a.tokens)), block(kThreads);
    if (wide) {
        auto *f = bf16 ? embedding_kernel<true, int64_t> : embedding_kernel<false, int64_t>;
        hipLaunchKernelGGL(f, grid, block, 0, stream, static_cast<const int64_t *>(a.ids), a.table, a.pos, a.tokens, a.n,
                           a.vocab, a.d, a.scale, a.y);
    } else {
        auto *f = bf16 ? embedding_kernel<true, int32_t> : embedding_kernel<false, int32_t>;
        hipLaunchKernelGGL(f, grid, block, 0, stream, static_cast<const int32_t *>(a.ids), a.table, a.pos, a.tokens, a.n,
                           a.vocab, a.d, a.scale, a.y);
    }
    return hipGetLastError();
}

hipError_t launch_embedding_backward(const EmbeddingBackward &a, bool bf16, bool wide, hipStream_t stream) {
    {
        KernelTimer timer("embedding_bwd_kernel", stream);
        const dim3 grid(row_grid(a.vocab)), block(kThreads);
        if (wide) {
            auto *f = bf16 ? embedding_bwd_kernel<true, int64_t> : embedding_bwd_kernel<false, int64_t>;
            hipLaunchKernelGGL(f, grid, block, 0, stream, static_cast<const int64_t *>(a.ids), a.dy, a.tokens, a.vocab,
                               a.d, a.scale, a.dtable);
        } else {
            auto *f = bf16 ? embedding_bwd_kernel<true, int32_t> : embedding_bwd_kernel<false, int32_t>;
            hipLaunchKernelGGL(f, grid, block, 0, stream, static_cast<const int32_t *>(a.ids), a.dy, a.tokens, a.vocab,
                               a.d, a.scale, a.dtable);
        }
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess || a.n == 0) return e;
    }
    KernelTimer timer("embedding_pos_kernel", stream);
    auto *f = bf16 ? embedding_pos_kernel<true> : embedding_pos_kernel<false>;
    hipLaunchKernelGGL(f, dim3(row_grid(a.n)), dim3(kThreads), 0, stream, a.dy, a.tokens, a.n, a.d, a.dpos);
    return hipGetLastError();
}

}  // namespace yoso
