// Rows of any width in 16-byte vectors (internal header of the row kernels).
//
// A row of d values is taken by L lanes, NV vectors of N values (4 fp32, 8 bf16) each; vector i of a
// lane is the row's vector i L + lane.  Three layouts:
//   kAligned  N divides d: every row starts on a vector boundary.
//   kOverlap  d > N, any d: the last vector of a row ends with the row, so that it repeats some columns
//             of the one before it.  Both lanes compute and store the same values there; sums take
//             the repeated columns once.  Rows start anywhere: vectors are loaded and stored unaligned
//             (global memory takes 16-byte accesses at any element).  A store in the place of an input
//             must come after all lanes of the row have loaded it.
//   kTiny     d < N: one lane, value by value.
// Nothing is touched behind a row's end.
#pragma once

#include "common.h"

namespace yoso {

enum RowLayout : int { kAligned = 0, kOverlap = 1, kTiny = 2 };

template <bool BF16>
struct Vec {
    static constexpr int N = BF16 ? 8 : 4;
};

typedef uint32_t raw4 __attribute__((ext_vector_type(4)));
typedef uint32_t raw4_any __attribute__((ext_vector_type(4), aligned(2)));
typedef float float4_any __attribute__((ext_vector_type(4), aligned(4)));
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

// What a lane's vector of a row is: its first column, and which of its columns count.
template <bool BF16, int LAYOUT>
struct Columns {
    static constexpr int N = Vec<BF16>::N;
    int c;      // first column
    int twice;  // kOverlap: columns that the vector before holds too
    bool in;    // there is such a vector

    __device__ __forceinline__ Columns(int index, int d) {
        const int at = index * N;
        in = at < d;
        if constexpr (LAYOUT == kOverlap) {
            c = at + N <= d ? at : d - N;
            twice = at - c;
        } else {
            c = at;
            twice = 0;
        }
    }
    // whether column c + j is this lane's to sum
    __device__ __forceinline__ bool counts(int j, int d) const {
        if constexpr (LAYOUT == kAligned) return in;
        if constexpr (LAYOUT == kOverlap) return in && j >= twice;
        return c + j < d;
    }
};

// The vector of the row that starts at element `row`; 0 where there is none or `active` is false.
template <bool BF16, int LAYOUT>
__device__ __forceinline__ raw4 load_vec(const void *base, int64_t row, const Columns<BF16, LAYOUT> &col, int d,
                                         bool active) {
    raw4 v = {0, 0, 0, 0};
    const char *p = static_cast<const char *>(base) + (row + col.c) * (BF16 ? 2 : 4);
    if (!col.in || !active) return v;
    if constexpr (LAYOUT == kAligned) {
        v = *reinterpret_cast<const raw4 *>(p);
    } else if constexpr (LAYOUT == kOverlap) {
        v = *reinterpret_cast<const raw4_any *>(p);
    } else {
#pragma unroll
        for (int j = 0; j < Vec<BF16>::N - 1; j++)
            if (col.c + j < d) {
                if constexpr (BF16)
                    v[j >> 1] |= static_cast<uint32_t>(reinterpret_cast<const uint16_t *>(p)[j]) << (16 * (j & 1));
                else
                    v[j] = reinterpret_cast<const uint32_t *>(p)[j];
            }
    }
    return v;
}

template <bool BF16, int LAYOUT>
__device__ __forceinline__ void store_vec(void *base, int64_t row, const Columns<BF16, LAYOUT> &col, int d, bool active,
                                          const raw4 &v) {
    char *p = static_cast<char *>(base) + (row + col.c) * (BF16 ? 2 : 4);
    if (!col.in || !active) return;
    if constexpr (LAYOUT == kAligned) {
        *reinterpret_cast<raw4 *>(p) = v;
    } else if constexpr (LAYOUT == kOverlap) {
        *reinterpret_cast<raw4_any *>(p) = v;
    } else {
#pragma unroll
        for (int j = 0; j < Vec<BF16>::N - 1; j++)
            if (col.c + j < d) {
                if constexpr (BF16)
                    reinterpret_cast<uint16_t *>(p)[j] = static_cast<uint16_t>(v[j >> 1] >> (16 * (j & 1)));
                else
                    reinterpret_cast<uint32_t *>(p)[j] = v[j];
            }
    }
}

// the columns' values of an fp32 parameter vector [d]; `other` where p is NULL
template <bool BF16, int LAYOUT>
__device__ __forceinline__ void load_param(const float *p, const Columns<BF16, LAYOUT> &col, int d, float other,
                                           float *out) {
    constexpr int N = Vec<BF16>::N;
#pragma unroll
    for (int j = 0; j < N; j++) out[j] = other;
    if (p == nullptr || !col.in) return;
    if constexpr (LAYOUT != kTiny) {
#pragma unroll
        for (int j = 0; j < N; j += 4) {
            const float4_any f = *reinterpret_cast<const float4_any *>(p + col.c + j);
#pragma unroll
            for (int k = 0; k < 4; k++) out[j + k] = f[k];
        }
    } else {
#pragma unroll
        for (int j = 0; j < N - 1; j++)
            if (col.c + j < d) out[j] = p[col.c + j];
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
        // lane k W + w of every wave takes the sum k of the row's wave w: one read, no more registers
        const int l = threadIdx.x & 63;
        const float x = group_sum(l < K * W ? part[(wave / W) * W * K + (l % W) * K + l / W] : 0.f, W);
#pragma unroll
        for (int k = 0; k < K; k++) v[k] = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), k * W));
    }
}

// Sum over the rows of a wave: lanes of the same place in their groups of L (L = 4 ... 64).
template <int L>
__device__ __forceinline__ float sum_of_groups(float x) {
    if (L <= 4) x += dpp_mov<0x124>(x);  // row_ror:4
    if (L <= 8) x += dpp_mov<0x128>(x);  // row_ror:8
    if (L <= 16) {
        const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
        x = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    }
    if (L <= 32) {
        const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
        x = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    }
    return x;
}

}  // namespace yoso
