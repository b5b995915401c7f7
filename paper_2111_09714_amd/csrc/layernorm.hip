// Layer norm of rows of any width, with the residual added on the way in, and its backward (gfx950).
//
//   z = x + residual;  mu = mean_c z;  s = 1 / sqrt(mean_c (z - mu)^2 + eps)
//   y = (z - mu) s w + b
//   g = dy w;  dx = s (g - mean_c g - xh mean_c (g xh)) + dsum,   xh = (z - mu) s
//   dw = sum_r dy xh;  db = sum_r dy
//
// The mean is taken in two steps, mu = m0 + mean(z - m0) with m0 the fp32 mean, and the variance
// around m0 less the square of the second step: rows far from zero keep the accuracy of their
// deviations.
#include "common.h"
#include "launch.h"
#include "timing.h"

namespace yoso {

namespace {

constexpr int kThreads = 256;

__device__ __forceinline__ float block_sum(float v) {
    __shared__ float part[kThreads / 64];
    v = group_sum(v, 64);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
    __syncthreads();
    return (part[0] + part[1]) + (part[2] + part[3]);
}

template <bool BF16>
__device__ __forceinline__ void store1(void *base, int64_t off, float v) {
    if constexpr (BF16)
        static_cast<__bf16 *>(base)[off] = static_cast<__bf16>(v);
    else
        static_cast<float *>(base)[off] = v;
}

// the mean m0 + m1 (kept apart: their sum would round the second step away) and 1/std of one row of
// x (+ residual), by the whole workgroup
template <bool BF16>
__device__ __forceinline__ void row_stats(const void *x, const void *res, int64_t off, int d, float eps, float &m0,
                                          float &m1, float &rstd) {
    float a = 0.f;
    for (int c = threadIdx.x; c < d; c += kThreads) a += load1<BF16>(x, off + c) + (res ? load1<BF16>(res, off + c) : 0.f);
    m0 = block_sum(a) / d;
    float s1 = 0.f, s2 = 0.f;
    for (int c = threadIdx.x; c < d; c += kThreads) {
        const float t = load1<BF16>(x, off + c) + (res ? load1<BF16>(res, off + c) : 0.f) - m0;
        s1 += t;
        s2 += t * t;
    }
    s1 = block_sum(s1) / d;
    s2 = block_sum(s2) / d;
    m1 = s1;
    rstd = 1.f / sqrtf(fmaxf(s2 - s1 * s1, 0.f) + eps);
}

template <bool BF16>
__global__ __launch_bounds__(kThreads) void layer_norm_kernel(const void *x, const void *res, const float *w,
                                                              const float *b, int64_t rows, int d, float eps,
                                                              void *sum, void *y) {
    for (int64_t r = blockIdx.x; r < rows; r += gridDim.x) {
        const int64_t off = r * d;
        float m0, m1, rstd;
        row_stats<BF16>(x, res, off, d, eps, m0, m1, rstd);
        for (int c = threadIdx.x; c < d; c += kThreads) {
            const float z = load1<BF16>(x, off + c) + (res ? load1<BF16>(res, off + c) : 0.f);
            if (sum) store1<BF16>(sum, off + c, z);
            store1<BF16>(y, off + c, (z - m0 - m1) * rstd * (w ? w[c] : 1.f) + (b ? b[c] : 0.f));
        }
    }
}

template <bool BF16>
__global__ __launch_bounds__(kThreads) void layer_norm_bwd_kernel(const void *z, const float *w, const void *dy,
                                                                  const void *dsum, int64_t rows, int d, float eps,
                                                                  void *dx, float4 *stats) {
    for (int64_t r = blockIdx.x; r < rows; r += gridDim.x) {
        const int64_t off = r * d;
        float m0, m1, rstd;
        row_stats<BF16>(z, nullptr, off, d, eps, m0, m1, rstd);
        float a = 0.f, c2 = 0.f;
        for (int c = threadIdx.x; c < d; c += kThreads) {
            const float g = load1<BF16>(dy, off + c) * (w ? w[c] : 1.f);
            a += g;
            c2 += g * (load1<BF16>(z, off + c) - m0 - m1) * rstd;
        }
        a = block_sum(a) / d;
        c2 = block_sum(c2) / d;
        for (int c = threadIdx.x; c < d; c += kThreads) {
            const float g = load1<BF16>(dy, off + c) * (w ? w[c] : 1.f);
            const float xh = (load1<BF16>(z, off + c) - m0 - m1) * rstd;
            const float t = dsum ? load1<BF16>(dsum, off + c) : 0.f;
            store1<BF16>(dx, off + c, rstd * (g - a - xh * c2) + t);
        }
        if (stats && threadIdx.x == 0) stats[r] = make_float4(m0, m1, rstd, 0.f);
    }
}

template <bool BF16>
__global__ __launch_bounds__(kThreads) void layer_norm_params_kernel(const void *z, const void *dy,
                                                                     const float4 *stats, int64_t rows, int d,
                                                                     float *dw, float *db) {
    const int c = blockIdx.x * kThreads + threadIdx.x;
    if (c >= d) return;
    float a = 0.f, b = 0.f;
    for (int64_t r = 0; r < rows; r++) {
        const float g = load1<BF16>(dy, r * d + c);
        a += g * (load1<BF16>(z, r * d + c) - stats[r].x - stats[r].y) * stats[r].z;
        b += g;
    }
    dw[c] = a;
    db[c] = b;
}

unsigned row_grid(int64_t rows) { return static_cast<unsigned>(rows < 65536 ? rows : 65536); }

}  // namespace

size_t layer_norm_backward_workspace(bool bf16, int64_t rows, int d) { return static_cast<size_t>(rows) * 16; }

hipError_t launch_layer_norm(const LayerNorm &a, bool bf16, hipStream_t stream) {
    if (a.rows == 0) return hipSuccess;
    KernelTimer timer("layer_norm_kernel", stream);
    auto *f = bf16 ? layer_norm_kernel<true> : layer_norm_kernel<false>;
    hipLaunchKernelGGL(f, dim3(row_grid(a.rows)), dim3(kThreads), 0, stream, a.x, a.residual, a.weight, a.bias, a.rows,
                       a.d, a.eps, a.sum, a.y);
    return hipGetLastError();
}

hipError_t launch_layer_norm_backward(const LayerNormBackward &a, bool bf16, hipStream_t stream) {
    if (a.rows > 0) {
        KernelTimer timer("layer_norm_bwd_kernel", stream);
        auto *f = bf16 ? layer_norm_bwd_kernel<true> : layer_norm_bwd_kernel<false>;
        hipLaunchKernelGGL(f, dim3(row_grid(a.rows)), dim3(kThreads), 0, stream, a.z, a.weight, a.dy, a.dsum, a.rows,
                           a.d, a.eps, a.dx, a.dweight ? static_cast<float4 *>(a.workspace) : nullptr);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    if (!a.dweight) return hipSuccess;
    KernelTimer timer("layer_norm_params_kernel", stream);
    auto *f = bf16 ? layer_norm_params_kernel<true> : layer_norm_params_kernel<false>;
    hipLaunchKernelGGL(f, dim3((a.d + kThreads - 1) / kThreads), dim3(kThreads), 0, stream, a.z, a.dy,
                       static_cast<const float4 *>(a.workspace), a.rows, a.d, a.dweight, a.dbias);
    return hipGetLastError();
}

}  // namespace yoso
