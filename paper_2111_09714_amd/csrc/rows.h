// Rows of any width in 16-byte vectors (internal header of the row kernels).
//
// A row of d values is taken by L lanes, NV vectors each: vector i of a lane starts at column
// (i L + lane) N, N = 4 fp32 or 8 bf16 values.  Where N does not divide d the rows do not start
// on vector boundaries: full vectors are loaded and stored unaligned all the same (global memory
// takes 16-byte accesses at any address of whole elements), the row's last columns one by one, and
// nothing is touched behind a row's end.
#pragma once

#include "common.h"

namespace yoso {

template <bool BF16>
struct Vec {
    static constexpr int N = BF16 ? 8 : 4;
};

typedef uint32_t raw4 __attribute__((ext_vector_type(4)));
typedef uint32_t raw4_any __attribute__((ext_vector_type(4), aligned(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float floatx2 __attribute__((ext_vector_type(2)));

// value j of a raw vector
template <bool BF16>
__device__ __forceinline__ float value(const raw4 &v, int j) {
    if constexpr (BF16)
        return __uint_as_float((j & 1) ? (v[j >> 1] & 0xFFFF0000u) : (v[j >> 1] << 16));
    else
        return __uint_as_float(v[j]);
}

// rounds to nearest even; NaN stays NaN
template <bool BF16>
__device__ __forceinline__ raw4 pack(const float *f) {
    raw4 v;
#pragma unroll
    for (int i = 0; i < 4; i++) {
        if constexpr (BF16) {
            const floatx2 p = {f[2 * i], f[2 * i + 1]};
            v[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector(p, bf16x2));
        } else {
            v[i] = __float_as_uint(f[i]);
        }
    }
    return v;
}

// The vector at column c of the row that starts at element `row` (0 behind column d).
// ALIGNED: N divides d.
template <bool BF16, bool ALIGNED>
__device__ __forceinline__ raw4 load_vec(const void *base, int64_t row, int c, int d) {
    constexpr int N = Vec<BF16>::N;
    raw4 v = {0, 0, 0, 0};
    const char *p = static_cast<const char *>(base) + (row + c) * (BF16 ? 2 : 4);
    if constexpr (ALIGNED) {
        if (c < d) v = *reinterpret_cast<const raw4 *>(p);
    } else if (c + N <= d) {
        v = *reinterpret_cast<const raw4_any *>(p);
    } else {
#pragma unroll
        for (int j = 0; j < N - 1; j++)
            if (c + j < d) {
                if constexpr (BF16)
                    v[j >> 1] |= static_cast<uint32_t>(reinterpret_cast<const uint16_t *>(p)[j]) << (16 * (j & 1));
                else
                    v[j] = reinterpret_cast<const uint32_t *>(p)[j];
            }
    }
    return v;
}

template <bool BF16, bool ALIGNED>
__device__ __forceinline__ void store_vec(void *base, int64_t row, int c, int d, const raw4 &v) {
    constexpr int N = Vec<BF16>::N;
    char *p = static_cast<char *>(base) + (row + c) * (BF16 ? 2 : 4);
    if constexpr (ALIGNED) {
        if (c < d) *reinterpret_cast<raw4 *>(p) = v;
    } else if (c + N <= d) {
        *reinterpret_cast<raw4_any *>(p) = v;
    } else {
#pragma unroll
        for (int j = 0; j < N - 1; j++)
            if (c + j < d) {
                if constexpr (BF16)
                    reinterpret_cast<uint16_t *>(p)[j] = static_cast<uint16_t>(v[j >> 1] >> (16 * (j & 1)));
                else
                    reinterpret_cast<uint32_t *>(p)[j] = v[j];
            }
    }
}

// NC columns from c of an fp32 parameter vector [d]; `other` behind d or where p is NULL
template <int NC, bool ALIGNED>
__device__ __forceinline__ void load_param(const float *p, int c, int d, float other, float *out) {
#pragma unroll
    for (int j = 0; j < NC; j++) out[j] = other;
    if (p == nullptr) return;
    if (ALIGNED ? c < d : c + NC <= d) {
#pragma unroll
        for (int j = 0; j < NC; j += 4) {
            const float4 f = *reinterpret_cast<const float4 *>(p + c + j);
            out[j] = f.x; out[j + 1] = f.y; out[j + 2] = f.z; out[j + 3] = f.w;
        }
    } else {
#pragma unroll
        for (int j = 0; j < NC; j++)
            if (c + j < d) out[j] = p[c + j];
    }
}

// Sums of K values over the L lanes of each row of a workgroup of T threads (T / L rows).
// L <= 64: within the wave.  Wider rows join their waves through `part`, [T / 64][K] floats, with
// one barrier; callers alternate between two such arrays, so that a fast wave's next sum does not
// overwrite what a slow one still reads.
template <int K, int L, int T>
__device__ __forceinline__ void row_sums(float (&v)[K], float *part) {
#pragma unroll
    for (int k = 0; k < K; k++) v[k] = group_sum(v[k], L < 64 ? L : 64);
    if constexpr (L > 64) {
        constexpr int W = L / 64;  // waves of a row
        const int wave = threadIdx.x >> 6;
        if ((threadIdx.x & 63) == 0)
#pragma unroll
            for (int k = 0; k < K; k++) part[wave * K + k] = v[k];
        __syncthreads();
        const float *row = part + (wave / W) * W * K;
#pragma unroll
        for (int k = 0; k < K; k++) {
            float s = 0.f;
#pragma unroll
            for (int w = 0; w < W; w++) s += row[w * K + k];
            v[k] = s;
        }
    }
}

}  // namespace yoso
