// Layer norm of rows of any width, with the residual added on the way in, and its backward (gfx950).
//
//   z = x + residual;  mu = mean_c z;  s = 1 / sqrt(mean_c (z - mu)^2 + eps)
//   y = (z - mu) s w + b
//   g = dy w;  dx = s (g - mean_c g - xh mean_c (g xh)) + dsum,   xh = (z - mu) s
//   dw = sum_r dy xh;  db = sum_r dy
//
// The mean is taken in two steps, mu = m0 + m1 with m0 the fp32 mean and m1 = mean(z - m0), kept
// apart (their fp32 sum would round m1 away), and the variance is that around m0 less m1^2: rows far
// from zero keep the accuracy of their deviations.  Sums are fp32 whatever the storage type.
//
// Both are streams: a row stays in registers between its one load and its one store, L lanes to a
// row (a part of a wave, a wave, or several), so every value crosses the memory bus once.  The backward
// sums dw and db of its rows in registers, each workgroup writes one partial row pair, and a second
// launch adds those in order: no atomics, the same bits every time.
#include "common.h"
#include "launch.h"
#include "rows.h"
#include "timing.h"

namespace yoso {

namespace {

// Lanes to a row: the fewest of 16, 32, ... 1024 that take it in at most 16 columns each.
constexpr int kMaxColumns = 16;

template <bool BF16, bool ALIGNED, int L, int NV, int T>
__global__ __launch_bounds__(T) void layer_norm_kernel(LayerNorm a) {
    constexpr int N = Vec<BF16>::N, G = T / L;
    __shared__ float part[2][2 * (T / 64)];
    const int lane = threadIdx.x % L, group = threadIdx.x / L, d = a.d;
    float w[NV][N], b[NV][N];
#pragma unroll
    for (int i = 0; i < NV; i++) {
        load_param<N, ALIGNED>(a.weight, (i * L + lane) * N, d, 1.f, w[i]);
        load_param<N, ALIGNED>(a.bias, (i * L + lane) * N, d, 0.f, b[i]);
    }
    for (int64_t r0 = static_cast<int64_t>(blockIdx.x) * G; r0 < a.rows; r0 += static_cast<int64_t>(gridDim.x) * G) {
        const bool active = r0 + group < a.rows;  // the others follow through the barriers, without columns
        const int64_t row = (r0 + group) * d;
        const int end = active ? d : 0;
        float z[NV][N];
        raw4 v[NV], u[NV];
#pragma unroll
        for (int i = 0; i < NV; i++) v[i] = load_vec<BF16, ALIGNED>(a.x, row, (i * L + lane) * N, end);
        if (a.residual) {
#pragma unroll
            for (int i = 0; i < NV; i++) u[i] = load_vec<BF16, ALIGNED>(a.residual, row, (i * L + lane) * N, end);
#pragma unroll
            for (int i = 0; i < NV; i++)
#pragma unroll
                for (int j = 0; j < N; j++) z[i][j] = value<BF16>(v[i], j) + value<BF16>(u[i], j);
        } else {
#pragma unroll
            for (int i = 0; i < NV; i++)
#pragma unroll
                for (int j = 0; j < N; j++) z[i][j] = value<BF16>(v[i], j);
        }
        if (a.sum) {
#pragma unroll
            for (int i = 0; i < NV; i++)
                store_vec<BF16, ALIGNED>(a.sum, row, (i * L + lane) * N, end, pack<BF16>(z[i]));
        }
        float s[1] = {0.f};
#pragma unroll
        for (int i = 0; i < NV; i++)
#pragma unroll
            for (int j = 0; j < N; j++) s[0] += z[i][j];
        row_sums<1, L, T>(s, part[0]);
        const float m0 = s[0] / d;
        float q[2] = {0.f, 0.f};
#pragma unroll
        for (int i = 0; i < NV; i++)
#pragma unroll
            for (int j = 0; j < N; j++) {
                z[i][j] -= m0;
                // (only a lane's last vector can lie behind the row's end)
                const float t = i < NV - 1 || (i * L + lane) * N + (ALIGNED ? 0 : j) < d ? z[i][j] : 0.f;
                q[0] += t;
                q[1] = fmaf(t, t, q[1]);
            }
        row_sums<2, L, T>(q, part[1]);
        const float m1 = q[0] / d;
        const float rstd = 1.f / sqrtf(fmaxf(q[1] / d - m1 * m1, 0.f) + a.eps);
#pragma unroll
        for (int i = 0; i < NV; i++) {
#pragma unroll
            for (int j = 0; j < N; j++) z[i][j] = fmaf((z[i][j] - m1) * rstd, w[i][j], b[i][j]);
            store_vec<BF16, ALIGNED>(a.y, row, (i * L + lane) * N, end, pack<BF16>(z[i]));
        }
    }
}

// dx of the workgroup's rows; `part`, [gridDim.x][2][d] (or, of one workgroup, dw and db themselves),
// takes the workgroup's sums of dy xh and of dy.
template <bool BF16, bool ALIGNED, int L, int NV, int T>
__global__ __launch_bounds__(T) void layer_norm_bwd_kernel(LayerNormBackward a, float *part_w, float *part_b,
                                                           int64_t part_stride) {
    constexpr int N = Vec<BF16>::N, G = T / L;
    constexpr int W = T / 64;  // waves
    // 1024 threads have 128 registers each: the weights of the widest rows come from the cache again
    constexpr bool KEEP = L < 1024;
    __shared__ float sums[2][3 * W];
    const int lane = threadIdx.x % L, group = threadIdx.x / L, d = a.d;
    float dw[NV][N], db[NV][N], held[KEEP ? NV : 1][N];
#pragma unroll
    for (int i = 0; i < NV; i++) {
        if constexpr (KEEP) load_param<N, ALIGNED>(a.weight, (i * L + lane) * N, d, 1.f, held[i]);
#pragma unroll
        for (int j = 0; j < N; j++) dw[i][j] = db[i][j] = 0.f;
    }
    const auto weight = [&](int i, float (&w)[N]) {
        if constexpr (KEEP) {
#pragma unroll
            for (int j = 0; j < N; j++) w[j] = held[i][j];
        } else {
            const float *p = a.weight;
            asm volatile("" : "+s"(p));  // else the loads are moved out of the loop, back into registers
            load_param<N, ALIGNED>(p, (i * L + lane) * N, d, 1.f, w);
        }
    };
    for (int64_t r0 = static_cast<int64_t>(blockIdx.x) * G; r0 < a.rows; r0 += static_cast<int64_t>(gridDim.x) * G) {
        const int64_t row = (r0 + group) * d;
        const int end = r0 + group < a.rows ? d : 0;
        raw4 zv[NV], gv[NV], sv[NV];
#pragma unroll
        for (int i = 0; i < NV; i++) zv[i] = load_vec<BF16, ALIGNED>(a.z, row, (i * L + lane) * N, end);
#pragma unroll
        for (int i = 0; i < NV; i++) gv[i] = load_vec<BF16, ALIGNED>(a.dy, row, (i * L + lane) * N, end);
        if (a.dsum) {
#pragma unroll
            for (int i = 0; i < NV; i++) sv[i] = load_vec<BF16, ALIGNED>(a.dsum, row, (i * L + lane) * N, end);
        }
        float s[2] = {0.f, 0.f};
#pragma unroll
        for (int i = 0; i < NV; i++) {
            float w[N];
            weight(i, w);
#pragma unroll
            for (int j = 0; j < N; j++) {
                s[0] += value<BF16>(zv[i], j);
                s[1] = fmaf(value<BF16>(gv[i], j), w[j], s[1]);
            }
        }
        row_sums<2, L, T>(s, sums[0]);
        const float m0 = s[0] / d;
        float q[3] = {0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < NV; i++) {
            float w[N];
            weight(i, w);
#pragma unroll
            for (int j = 0; j < N; j++) {
                const float zc = value<BF16>(zv[i], j) - m0;
                const float t = i < NV - 1 || (i * L + lane) * N + (ALIGNED ? 0 : j) < d ? zc : 0.f;
                q[0] += t;
                q[1] = fmaf(t, t, q[1]);
                q[2] = fmaf(value<BF16>(gv[i], j) * w[j], t, q[2]);
            }
        }
        row_sums<3, L, T>(q, sums[1]);
        const float m1 = q[0] / d;
        const float rstd = 1.f / sqrtf(fmaxf(q[1] / d - m1 * m1, 0.f) + a.eps);
        const float mg = s[1] / d;                        // mean of g
        const float mx = rstd * ((q[2] - m1 * s[1]) / d);  // mean of g xh
#pragma unroll
        for (int i = 0; i < NV; i++) {
            float o[N], w[N];
            weight(i, w);
#pragma unroll
            for (int j = 0; j < N; j++) {
                const float g = value<BF16>(gv[i], j);
                const float xh = (value<BF16>(zv[i], j) - m0 - m1) * rstd;
                dw[i][j] = fmaf(g, xh, dw[i][j]);
                db[i][j] += g;
                o[j] = rstd * (fmaf(g, w[j], -mg) - xh * mx);
            }
            if (a.dsum) {
#pragma unroll
                for (int j = 0; j < N; j++) o[j] += value<BF16>(sv[i], j);
            }
            store_vec<BF16, ALIGNED>(a.dx, row, (i * L + lane) * N, end, pack<BF16>(o));
        }
    }
    if (part_w == nullptr) return;
    // one pair of rows per workgroup: rows of one wave by lane exchanges, then the waves through LDS
    constexpr int R = L < 64 ? W : G;  // rows left after the exchanges
    constexpr int C = L * N;           // columns of a vector index
    __shared__ float join[R > 1 ? 2 * R * C : 1];
    part_w += blockIdx.x * part_stride;
    part_b += blockIdx.x * part_stride;
#pragma unroll
    for (int i = 0; i < NV; i++) {
        if constexpr (L < 64) {
#pragma unroll
            for (int j = 0; j < N; j++) {
                if constexpr (L == 16) {
                    const auto p = __builtin_amdgcn_permlane16_swap(__float_as_uint(dw[i][j]), __float_as_uint(dw[i][j]), false, false);
                    dw[i][j] = __uint_as_float(p[0]) + __uint_as_float(p[1]);
                    const auto q = __builtin_amdgcn_permlane16_swap(__float_as_uint(db[i][j]), __float_as_uint(db[i][j]), false, false);
                    db[i][j] = __uint_as_float(q[0]) + __uint_as_float(q[1]);
                }
                const auto p = __builtin_amdgcn_permlane32_swap(__float_as_uint(dw[i][j]), __float_as_uint(dw[i][j]), false, false);
                dw[i][j] = __uint_as_float(p[0]) + __uint_as_float(p[1]);
                const auto q = __builtin_amdgcn_permlane32_swap(__float_as_uint(db[i][j]), __float_as_uint(db[i][j]), false, false);
                db[i][j] = __uint_as_float(q[0]) + __uint_as_float(q[1]);
            }
        }
        if constexpr (R > 1) {
            const int r = L < 64 ? threadIdx.x >> 6 : group;
            __syncthreads();
            if (L >= 64 || (threadIdx.x & 63) < L)
#pragma unroll
                for (int j = 0; j < N; j += 4) {
                    *reinterpret_cast<float4 *>(&join[r * C + lane * N + j]) = make_float4(dw[i][j], dw[i][j + 1], dw[i][j + 2], dw[i][j + 3]);
                    *reinterpret_cast<float4 *>(&join[(R + r) * C + lane * N + j]) = make_float4(db[i][j], db[i][j + 1], db[i][j + 2], db[i][j + 3]);
                }
            __syncthreads();
            for (int k = threadIdx.x; k < 2 * C; k += T) {
                const float *col = join + (k < C ? k : R * C + k - C);
                float s = 0.f;
#pragma unroll
                for (int q = 0; q < R; q++) s += col[q * C];
                const int c = i * C + (k < C ? k : k - C);
                if (c < d) (k < C ? part_w : part_b)[c] = s;
            }
        } else {
#pragma unroll
            for (int j = 0; j < N; j++) {
                const int c = (i * L + lane) * N + j;
                if (c < d) {
                    part_w[c] = dw[i][j];
                    part_b[c] = db[i][j];
                }
            }
        }
    }
}

// dw and db from the partial rows [parts][2 d]: 64 columns to a workgroup, the parts over its 4 waves
constexpr int kParamThreads = 256;
__global__ __launch_bounds__(kParamThreads) void layer_norm_params_kernel(const float *part, int parts, int d,
                                                                          float *dw, float *db) {
    __shared__ float join[kParamThreads];
    const int c = blockIdx.x * 64 + (threadIdx.x & 63), wave = threadIdx.x >> 6;
    const int64_t stride = 2 * static_cast<int64_t>(d);
    float s = 0.f;
    if (c < stride)
#pragma unroll 8
        for (int p = wave; p < parts; p += kParamThreads / 64) s += part[p * stride + c];
    join[threadIdx.x] = s;
    __syncthreads();
    if (wave == 0 && c < stride) {
        s = (join[c % 64 + 0] + join[c % 64 + 64]) + (join[c % 64 + 128] + join[c % 64 + 192]);
        (c < d ? dw : db)[c < d ? c : c - d] = s;
    }
}

__global__ void layer_norm_no_rows_kernel(int d, float *dw, float *db) {
    for (int c = threadIdx.x; c < d; c += blockDim.x) dw[c] = db[c] = 0.f;
}

// Workgroups of the backward and with them partial rows: 512 threads, two workgroups to a CU.
constexpr int kBwdThreads = 512;
constexpr int64_t kBwdGroups = 512;

int row_lanes(bool bf16, int d) {
    const int nvec = (d + (bf16 ? 7 : 3)) / (bf16 ? 8 : 4);
    int lanes = 16;
    while (nvec > kMaxColumns / (bf16 ? 8 : 4) * lanes) lanes *= 2;
    return lanes;
}

int64_t backward_groups(bool bf16, int64_t rows, int d) {
    const int lanes = row_lanes(bf16, d);
    const int64_t per = lanes > kBwdThreads ? 1 : kBwdThreads / lanes;
    const int64_t need = (rows + per - 1) / per;
    return need < kBwdGroups ? need : kBwdGroups;
}

// Calls f.template operator()<BF16, ALIGNED, L, NV>() for the form that takes rows of d values.
template <bool BF16, bool ALIGNED, typename F>
void with_form(int d, F f) {
    constexpr int N = Vec<BF16>::N;
    const int nvec = (d + N - 1) / N, lanes = row_lanes(BF16, d), nv = (nvec + lanes - 1) / lanes;
#define YOSO_ROW_FORM(L_, NV_) \
    if (lanes == L_ && nv == NV_) return f.template operator()<BF16, ALIGNED, L_, NV_>();
    YOSO_ROW_FORM(16, 1) YOSO_ROW_FORM(16, 2)
    YOSO_ROW_FORM(32, 2) YOSO_ROW_FORM(64, 2) YOSO_ROW_FORM(128, 2) YOSO_ROW_FORM(256, 2) YOSO_ROW_FORM(512, 2)
    YOSO_ROW_FORM(1024, 2)
    if constexpr (!BF16) {
        YOSO_ROW_FORM(16, 3) YOSO_ROW_FORM(32, 3) YOSO_ROW_FORM(64, 3) YOSO_ROW_FORM(128, 3) YOSO_ROW_FORM(256, 3)
        YOSO_ROW_FORM(512, 3) YOSO_ROW_FORM(1024, 3)
        YOSO_ROW_FORM(16, 4) YOSO_ROW_FORM(32, 4) YOSO_ROW_FORM(64, 4) YOSO_ROW_FORM(128, 4) YOSO_ROW_FORM(256, 4)
        YOSO_ROW_FORM(512, 4) YOSO_ROW_FORM(1024, 4)
    }
#undef YOSO_ROW_FORM
}

template <typename F>
void with_form(bool bf16, int d, F f) {
    if (bf16)
        d % 8 == 0 ? with_form<true, true>(d, f) : with_form<true, false>(d, f);
    else
        d % 4 == 0 ? with_form<false, true>(d, f) : with_form<false, false>(d, f);
}

struct Forward {
    const LayerNorm &a;
    hipStream_t stream;
    template <bool BF16, bool ALIGNED, int L, int NV>
    void operator()() const {
        constexpr int T = L > 256 ? L : 256;
        const int64_t need = (a.rows + T / L - 1) / (T / L), most = L > 256 ? 512 : 2048;
        hipLaunchKernelGGL((layer_norm_kernel<BF16, ALIGNED, L, NV, T>), dim3(static_cast<unsigned>(need < most ? need : most)),
                           dim3(T), 0, stream, a);
    }
};

struct Backward {
    const LayerNormBackward &a;
    int64_t groups;
    hipStream_t stream;
    template <bool BF16, bool ALIGNED, int L, int NV>
    void operator()() const {
        constexpr int T = L > kBwdThreads ? L : kBwdThreads;
        float *part = static_cast<float *>(a.workspace);
        float *pw = groups == 1 ? a.dweight : part, *pb = groups == 1 ? a.dbias : part + a.d;
        if (!a.dweight) pw = pb = nullptr;
        hipLaunchKernelGGL((layer_norm_bwd_kernel<BF16, ALIGNED, L, NV, T>), dim3(static_cast<unsigned>(groups)), dim3(T), 0,
                           stream, a, pw, pb, 2 * static_cast<int64_t>(a.d));
    }
};

}  // namespace

size_t layer_norm_backward_workspace(bool bf16, int64_t rows, int d) {
    const int64_t groups = backward_groups(bf16, rows, d);
    return groups > 1 ? static_cast<size_t>(groups) * 2 * d * sizeof(float) : 0;
}

hipError_t launch_layer_norm(const LayerNorm &a, bool bf16, hipStream_t stream) {
    if (a.rows == 0) return hipSuccess;
    KernelTimer timer("layer_norm_kernel", stream);
    with_form(bf16, a.d, Forward{a, stream});
    return hipGetLastError();
}

hipError_t launch_layer_norm_backward(const LayerNormBackward &a, bool bf16, hipStream_t stream) {
    if (a.rows == 0) {
        if (!a.dweight) return hipSuccess;
        KernelTimer timer("layer_norm_params_kernel", stream);
        hipLaunchKernelGGL(layer_norm_no_rows_kernel, dim3(1), dim3(kParamThreads), 0, stream, a.d, a.dweight, a.dbias);
        return hipGetLastError();
    }
    const int64_t groups = backward_groups(bf16, a.rows, a.d);
    {
        KernelTimer timer("layer_norm_bwd_kernel", stream);
        with_form(bf16, a.d, Backward{a, groups, stream});
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess || groups == 1 || !a.dweight) return e;
    }
    KernelTimer timer("layer_norm_params_kernel", stream);
    hipLaunchKernelGGL(layer_norm_params_kernel, dim3(static_cast<unsigned>((2 * a.d + 63) / 64)), dim3(kParamThreads), 0,
                       stream, static_cast<const float *>(a.workspace), static_cast<int>(groups), a.d, a.dweight, a.dbias);
    return hipGetLastError();
}

}  // namespace yoso
