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
// Both are streams bound by memory: a row stays in registers between its one load and its one store, L lanes to
// a row (a part of a wave, a wave, or several), so every value crosses the memory bus once.  The backward
// sums dw and db of its rows in registers, each workgroup writes one partial row pair, and a second
// launch adds those in order: no atomics, the same bits every time.
#include "common.h"
#include "launch.h"
#include "rows.h"
#include "timing.h"

namespace yoso {

namespace {

// mean_c around m0 and 1/std of a row from its sums of t = z - m0 and of t^2
__device__ __forceinline__ float row_rstd(float sum2, float m1, float inv, float eps) {
    return rsqrtf(fmaxf(sum2 * inv - m1 * m1, 0.f) + eps);
}

// Workgroups stay for several rows, so that weight and bias are read once each.  16384 x 768 bf16 with residual
// and sum 17 us, 5.9 TB/s; 256 MiB of one input and one output 6.0 to 6.5 TB/s at widths from 32 to 8192, odd ones
// among them (a copy of as much: 7.0, half of it from the memory-side cache), four tensors of 128 MiB 4.9
// to 5.5 TB/s (a copy: 5.4).
template <bool BF16, int LAYOUT, int L, int NV, int T>
__global__ __launch_bounds__(T) void layer_norm_kernel(LayerNorm a) {
    constexpr int N = Vec<BF16>::N, G = T / L;
    using Cols = Columns<BF16, LAYOUT>;
    __shared__ float part[2][2 * (T / 64)];
    const int lane = threadIdx.x % L, group = threadIdx.x / L, d = a.d;
    const float inv = 1.f / d;
    float w[NV][N], b[NV][N];
#pragma unroll
    for (int i = 0; i < NV; i++) {
        load_param(a.weight, Cols(i * L + lane, d), d, 1.f, w[i]);
        load_param(a.bias, Cols(i * L + lane, d), d, 0.f, b[i]);
    }
    for (int64_t r0 = static_cast<int64_t>(blockIdx.x) * G; r0 < a.rows; r0 += static_cast<int64_t>(gridDim.x) * G) {
        const bool active = r0 + group < a.rows;  // the others follow through the barriers
        const int64_t row = (r0 + group) * d;
        float z[NV][N];
        raw4 v[NV], u[NV];
#pragma unroll
        for (int i = 0; i < NV; i++) v[i] = load_vec(a.x, row, Cols(i * L + lane, d), d, active);
        if (a.residual) {
#pragma unroll
            for (int i = 0; i < NV; i++) u[i] = load_vec(a.residual, row, Cols(i * L + lane, d), d, active);
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
        float s[1] = {0.f};
#pragma unroll
        for (int i = 0; i < NV; i++) {
            const Cols col(i * L + lane, d);
#pragma unroll
            for (int j = 0; j < N; j++) s[0] += LAYOUT != kOverlap || i < NV - 1 || j >= col.twice ? z[i][j] : 0.f;
        }
        row_sums<1, L, T>(s, part[0]);
        if (a.sum) {
#pragma unroll
            for (int i = 0; i < NV; i++) store_vec(a.sum, row, Cols(i * L + lane, d), d, active, pack<BF16>(z[i]));
        }
        const float m0 = s[0] / d;
        float q[2] = {0.f, 0.f};
#pragma unroll
        for (int i = 0; i < NV; i++) {
            const Cols col(i * L + lane, d);
            // (only a lane's last vector can be missing, or repeat columns)
            if (i < NV - 1 || col.in)
#pragma unroll
                for (int j = 0; j < N; j++) {
                    z[i][j] -= m0;
                    const float t = LAYOUT == kAligned || i < NV - 1 || col.counts(j, d) ? z[i][j] : 0.f;
                    q[0] += t;
                    q[1] = fmaf(t, t, q[1]);
                }
        }
        row_sums<2, L, T>(q, part[1]);
        const float m1 = q[0] * inv, rstd = row_rstd(q[1], m1, inv, a.eps), shift = -m1 * rstd;
#pragma unroll
        for (int i = 0; i < NV; i++) {
#pragma unroll
            for (int j = 0; j < N; j++) z[i][j] = fmaf(fmaf(z[i][j], rstd, shift), w[i][j], b[i][j]);
            store_vec(a.y, row, Cols(i * L + lane, d), d, active, pack<BF16>(z[i]));
        }
    }
}

// 65536 x 768 bf16 with dsum 77 us, 5.2 TB/s (a copy of as much: 5.4); 65536 x 128 fp32 17 us, and 3 us for the sums of the
// partial rows.  16-bit rows of more than a wave come to 3.9 to 4.8 TB/s, bound by the vector unit (about 16
// operations a value) at two waves a SIMD.
//
// dx of the workgroup's rows; part_w and part_b + blockIdx.x part_stride take the workgroup's sums of
// dy xh and of dy.  Sums of a row in two rounds: of z; then of t = z - m0, t^2, g and g t.
template <bool BF16, int LAYOUT, int L, int NV, int T>
__global__ __launch_bounds__(T, 2) void layer_norm_bwd_kernel(LayerNormBackward a, float *part_w, float *part_b,
                                                           int64_t part_stride) {
    constexpr int N = Vec<BF16>::N, G = T / L;
    constexpr int W = T / 64;  // waves
    using Cols = Columns<BF16, LAYOUT>;
    __shared__ float sums[2][4 * W];
    const int lane = threadIdx.x % L, group = threadIdx.x / L, d = a.d;
    const float inv = 1.f / d;
    float w[NV][N], dw[NV][N], db[NV][N];
#pragma unroll
    for (int i = 0; i < NV; i++) {
        load_param(a.weight, Cols(i * L + lane, d), d, 1.f, w[i]);
#pragma unroll
        for (int j = 0; j < N; j++) dw[i][j] = db[i][j] = 0.f;
    }
    for (int64_t r0 = static_cast<int64_t>(blockIdx.x) * G; r0 < a.rows; r0 += static_cast<int64_t>(gridDim.x) * G) {
        const int64_t row = (r0 + group) * d;
        const bool active = r0 + group < a.rows;
        raw4 zv[NV], gv[NV], sv[NV];
#pragma unroll
        for (int i = 0; i < NV; i++) zv[i] = load_vec(a.z, row, Cols(i * L + lane, d), d, active);
#pragma unroll
        for (int i = 0; i < NV; i++) gv[i] = load_vec(a.dy, row, Cols(i * L + lane, d), d, active);
        if (a.dsum) {
#pragma unroll
            for (int i = 0; i < NV; i++) sv[i] = load_vec(a.dsum, row, Cols(i * L + lane, d), d, active);
        }
        float s[1] = {0.f};
#pragma unroll
        for (int i = 0; i < NV; i++) {
            const Cols col(i * L + lane, d);
#pragma unroll
            for (int j = 0; j < N; j++)
                s[0] += LAYOUT != kOverlap || i < NV - 1 || j >= col.twice ? value<BF16>(zv[i], j) : 0.f;
        }
        row_sums<1, L, T>(s, sums[0]);
        const float m0 = s[0] / d;
        float t[NV][N], q[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < NV; i++) {
            const Cols col(i * L + lane, d);
            if (i < NV - 1 || col.in) {
#pragma unroll
                for (int j = 0; j < N; j++) {
                    t[i][j] = value<BF16>(zv[i], j) - m0;
                    const float g = value<BF16>(gv[i], j) * w[i][j];
                    const bool counts = LAYOUT == kAligned || i < NV - 1 || col.counts(j, d);
                    const float tc = counts ? t[i][j] : 0.f;
                    q[0] += tc;
                    q[1] = fmaf(tc, tc, q[1]);
                    q[2] += counts ? g : 0.f;
                    q[3] = fmaf(g, tc, q[3]);
                }
            } else {
#pragma unroll
                for (int j = 0; j < N; j++) t[i][j] = 0.f;
            }
        }
        row_sums<4, L, T>(q, sums[1]);
        const float m1 = q[0] * inv, rstd = row_rstd(q[1], m1, inv, a.eps), shift = -m1 * rstd;
        const float lift = -(q[2] * inv) * rstd;                       // -mean(g) rstd
        const float tilt = -(q[3] - m1 * q[2]) * inv * rstd * rstd;  // -mean(g xh) rstd
#pragma unroll
        for (int i = 0; i < NV; i++) {
            float o[N];
#pragma unroll
            for (int j = 0; j < N; j++) {
                const float xh = fmaf(t[i][j], rstd, shift), dy = value<BF16>(gv[i], j);
                dw[i][j] = fmaf(dy, xh, dw[i][j]);
                db[i][j] += dy;
                o[j] = fmaf(xh, tilt, fmaf(dy * w[i][j], rstd, lift));
            }
            if (a.dsum) {
#pragma unroll
                for (int j = 0; j < N; j++) o[j] += value<BF16>(sv[i], j);
            }
            store_vec(a.dx, row, Cols(i * L + lane, d), d, active, pack<BF16>(o));
        }
    }
    if (part_w == nullptr) return;
    // one pair of rows per workgroup: the rows of a wave by lane exchanges, then its waves through LDS
    constexpr int R = L < 64 ? W : G;  // rows left after the exchanges
    constexpr int C = L * N;           // columns of a vector index
    __shared__ float join[R > 1 ? 2 * R * C : 1];
    part_w += blockIdx.x * part_stride;
    part_b += blockIdx.x * part_stride;
#pragma unroll
    for (int i = 0; i < NV; i++) {
#pragma unroll
        for (int j = 0; j < N; j++) {
            dw[i][j] = sum_of_groups<L>(dw[i][j]);
            db[i][j] = sum_of_groups<L>(db[i][j]);
        }
        if constexpr (R > 1) {
            const int r = L < 64 ? threadIdx.x >> 6 : group;
            __syncthreads();
            if (L >= 64 || (threadIdx.x & 63) < L)
#pragma unroll
                for (int j = 0; j < N; j += 4) {
                    float *to = join + r * C + lane * N + j;
                    *reinterpret_cast<float4 *>(to) = make_float4(dw[i][j], dw[i][j + 1], dw[i][j + 2], dw[i][j + 3]);
                    *reinterpret_cast<float4 *>(to + R * C) = make_float4(db[i][j], db[i][j + 1], db[i][j + 2], db[i][j + 3]);
                }
            __syncthreads();
            for (int k = threadIdx.x; k < 2 * C; k += T) {
                const int e = k < C ? k : k - C;
                const float *at = join + (k < C ? e : R * C + e);
                float s = 0.f;
#pragma unroll
                for (int q = 0; q < R; q++) s += at[q * C];
                const Cols col(i * L + e / N, d);
                if (col.in && col.c + e % N < d) (k < C ? part_w : part_b)[col.c + e % N] = s;
            }
        } else {
            const Cols col(i * L + lane, d);
#pragma unroll
            for (int j = 0; j < N; j++)
                if (col.in && col.c + j < d) {
                    part_w[col.c + j] = dw[i][j];
                    part_b[col.c + j] = db[i][j];
                }
        }
    }
}

// dw and db from the partial rows [parts][2 d], 2 to 5 us: 16 columns to a workgroup, four to a lane, the parts
// over 64 lanes, so that few columns still spread over the card and a lane has few parts to wait for.
constexpr int kParamThreads = 256;
__global__ __launch_bounds__(kParamThreads) void layer_norm_params_kernel(const float *part, int parts, int d,
                                                                          float *dw, float *db) {
    __shared__ float4 join[kParamThreads / 64][4];
    const int n = 2 * d, c = blockIdx.x * 16 + (threadIdx.x & 3) * 4, first = threadIdx.x >> 2;
    float s[4] = {0.f, 0.f, 0.f, 0.f};
    if (c < n) {
#pragma unroll 8
        for (int p = first; p < parts; p += kParamThreads / 4) {
            const float *at = part + static_cast<int64_t>(p) * n + c;
            if (c + 4 <= n) {
                const float4_any v = *reinterpret_cast<const float4_any *>(at);
#pragma unroll
                for (int j = 0; j < 4; j++) s[j] += v[j];
            } else {
                for (int j = 0; j < n - c; j++) s[j] += at[j];
            }
        }
    }
#pragma unroll
    for (int j = 0; j < 4; j++) s[j] = sum_of_groups<4>(s[j]);
    if ((threadIdx.x & 63) < 4) join[threadIdx.x >> 6][threadIdx.x & 3] = make_float4(s[0], s[1], s[2], s[3]);
    __syncthreads();
    if (threadIdx.x < 16) {
        const int e = blockIdx.x * 16 + threadIdx.x;
        float t = 0.f;
        for (int w = 0; w < kParamThreads / 64; w++) t += reinterpret_cast<const float *>(join[w])[threadIdx.x];
        if (e < n) (e < d ? dw : db)[e < d ? e : e - d] = t;
    }
}

__global__ void layer_norm_no_rows_kernel(int d, float *dw, float *db) {
    for (int c = threadIdx.x; c < d; c += blockDim.x) dw[c] = db[c] = 0.f;
}

// Workgroups of the backward and with them partial rows: one of eight waves to a CU.  With two to a CU the
// registers of a wave halve (spills from d = 1024 on) and the partial rows double: 65536 x 768 bf16 with
// dsum 85 us, with one 77 us.
constexpr int kBwdThreads = 512;
constexpr int64_t kBwdGroups = 256;

// Lanes and vectors a lane for rows of d values: two vectors a lane, which keep loads in flight with few
// registers, up to a wave to a row; then three and four, so that a row's sums stay within its wave as
// long as they can; then more waves.  Backward of 2^26 bf16 values: d = 2048 in four vectors of 64 lanes 82 us, in two
// of 128 lanes (a barrier more) 95 us; d = 4096 92 and 100 us.
struct RowForm {
    int lanes, vectors;
};

RowForm row_form(bool bf16, int d) {
    const int n = bf16 ? 8 : 4, nvec = (d + n - 1) / n;
    int lanes = 4;
    while (nvec > (lanes >= 64 ? 4 : 2) * lanes) lanes *= 2;
    return {lanes, (nvec + lanes - 1) / lanes};
}

int64_t backward_groups(bool bf16, int64_t rows, int d) {
    const int per = kBwdThreads / row_form(bf16, d).lanes;
    const int64_t need = (rows + per - 1) / per;
    // Rows of four rounds are one workgroup's, which writes the sums itself: a launch less, 32 x 768 fp32 14.4 -> 11.7 us a
    // call (eight rounds: the rounds take as long as the launch).
    if (need <= 4) return 1;
    return need < kBwdGroups ? need : kBwdGroups;
}

// Calls f.template operator()<BF16, LAYOUT, L, NV>() for the form that takes rows of d values.
template <bool BF16, int LAYOUT, typename F>
void with_form(int d, F f) {
    const RowForm form = row_form(BF16, d);
#define YOSO_ROW_FORM(L_, NV_) \
    if (form.lanes == L_ && form.vectors == NV_) return f.template operator()<BF16, LAYOUT, L_, NV_>();
    YOSO_ROW_FORM(4, 1)
    if constexpr (LAYOUT != kTiny) {
        YOSO_ROW_FORM(4, 2) YOSO_ROW_FORM(8, 2) YOSO_ROW_FORM(16, 2) YOSO_ROW_FORM(32, 2) YOSO_ROW_FORM(64, 2)
        YOSO_ROW_FORM(64, 3) YOSO_ROW_FORM(128, 3) YOSO_ROW_FORM(256, 3)
        YOSO_ROW_FORM(64, 4) YOSO_ROW_FORM(128, 4) YOSO_ROW_FORM(256, 4)
        if constexpr (!BF16) {
            YOSO_ROW_FORM(512, 3) YOSO_ROW_FORM(512, 4)
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

struct Forward {
    const LayerNorm &a;
    hipStream_t stream;
    template <bool BF16, int LAYOUT, int L, int NV>
    void operator()() const {
        constexpr int T = L > 256 ? L : 256;
        const int64_t need = (a.rows + T / L - 1) / (T / L), most = T > 256 ? 1024 : 2048;
        hipLaunchKernelGGL((layer_norm_kernel<BF16, LAYOUT, L, NV, T>), dim3(static_cast<unsigned>(need < most ? need : most)),
                           dim3(T), 0, stream, a);
    }
};

struct Backward {
    const LayerNormBackward &a;
    int64_t groups;
    hipStream_t stream;
    template <bool BF16, int LAYOUT, int L, int NV>
    void operator()() const {
        float *part = static_cast<float *>(a.workspace);
        float *pw = groups == 1 ? a.dweight : part, *pb = groups == 1 ? a.dbias : part + a.d;
        if (!a.dweight) pw = pb = nullptr;
        hipLaunchKernelGGL((layer_norm_bwd_kernel<BF16, LAYOUT, L, NV, kBwdThreads>), dim3(static_cast<unsigned>(groups)),
                           dim3(kBwdThreads), 0, stream, a, pw, pb, 2 * static_cast<int64_t>(a.d));
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
    bf16 ? with_layout<true>(a.d, Forward{a, stream}) : with_layout<false>(a.d, Forward{a, stream});
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
        const Backward f{a, groups, stream};
        bf16 ? with_layout<true>(a.d, f) : with_layout<false>(a.d, f);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess || groups == 1 || !a.dweight) return e;
    }
    KernelTimer timer("layer_norm_params_kernel", stream);
    hipLaunchKernelGGL(layer_norm_params_kernel, dim3(static_cast<unsigned>((2 * a.d + 15) / 16)), dim3(kParamThreads), 0,
                       stream, static_cast<const float *>(a.workspace), static_cast<int>(groups), a.d, a.dweight, a.dbias);
    return hipGetLastError();
}

}  // namespace yoso
