// Matrix tiles of the vocabulary's products (internal header): acc[M][N] += sum_k A[k][M] B[k][N] in 16-bit
// operands with fp32 sums.
//
// A workgroup of four waves (2 x 2) takes TM x TN values, a wave (TM / 2) x (TN / 2) in blocks of 32 x 32
// (v_mfma_f32_32x32x16, the shape that reaches the matrix rate here).  Operands come in steps of 32 k from
// global memory straight into LDS, kStages steps deep, so that a step's products run while later steps are
// under way; one barrier a step.  Laid-out operands are planes of blocks of 32 columns, [column / 32][row][32]: what
// a step takes, T rows of one block (k are columns) or 32 rows of T / 32 blocks (k are rows), is whole
// kilobytes either way, where rows side by side give half cache lines to the first.  LDS holds
//   k columns  64 bytes a row, read 16 bytes a lane; a row's 16-byte chunks are permuted by the addresses of the global
//              loads, so that a read's lanes fall on different LDS banks
//   k rows     the blocks, 64 bytes for each k, read by transposing 8-byte reads
// PL = 2: each operand is a pair of planes, v = hi + 2^-12 lo, and a product is hi hi + 2^-12 (hi lo + lo hi), the second sum in
// accumulators of its own.  hi leaves at most 2^-11 of a value (2^-25 of a small one), and with the factor lo takes it up in
// fp16's normal range: 22 bits down to 2^-29 of the largest value of a plane and a smallest step of 2^-51 of it, where a lo without the factor
// lost bits below 2^-17 and ended at 2^-39: gradients of sure tokens and of improbable entries lie there.
#pragma once

#include "common.h"

namespace yoso {

typedef float floatx16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short short4v __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) short4v lds_short4;
typedef __attribute__((address_space(3))) half8 lds_half8;
typedef __attribute__((address_space(3))) char lds_char;

constexpr int kStepK = 32;  // k values of a step
constexpr float kLowUp = 4096.f, kLowDown = 1.f / 4096.f;

// v by (below 2^15) as a pair of planes.  (The empty asm: hi and lo are to come from the one fp32 value; the conversions
// would take up the product that made it otherwise, and round it differently for each.)
__device__ __forceinline__ void pair(float v, float by, _Float16 &hi, _Float16 &lo) {
#pragma clang fp contract(off)
    float s = v * by;
    asm volatile("" : "+v"(s));
    hi = static_cast<_Float16>(s);
    lo = static_cast<_Float16>((s - static_cast<float>(hi)) * kLowUp);
}
template <int N, typename H>
__device__ __forceinline__ void pairs(const float (&v)[N], float by, H &hi, H &lo) {
#pragma unroll
    for (int i = 0; i < N; i++) {
        _Float16 h, l;
        pair(v[i], by, h, l);
        hi[i] = h, lo[i] = l;
    }
}

// LDS address of a __shared__ array
__device__ __forceinline__ uint32_t lds_address(void *p) {
    return static_cast<uint32_t>(reinterpret_cast<uintptr_t>((lds_char *)(p)));
}

// What a wave's lanes wrote to LDS before is what its other lanes read after it.
__device__ __forceinline__ void wave_meet() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// 16 bytes a lane from base + off (base and lds wave-uniform) to LDS bytes lds + 16 lane.  Counted by vmcnt, and
// unknown to the compiler, which waits for every such load before any transposing read otherwise: a wait and
// a barrier stand before the reads.  (No register is written but m0, which cannot be named: it is the compiler's own and not handed out.
// Nothing else in these kernels uses it: no builtin that loads into LDS, no indexed register, no message may be added beside this.)
__device__ __forceinline__ void load_to_lds(uint32_t lds, const void *base, uint32_t off) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds), "v"(off), "s"(base) : "memory");
}

// Waits until at most N of the wave's loads are under way and its LDS reads have come back, then for the other waves.
template <int N>
__device__ __forceinline__ void wait_and_meet() {
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}

// One operand of a tile: T rows (ROWS: T columns, k are rows).
template <int PL, int T, bool ROWS>
struct Operand {
    static constexpr int kLoads = T / 64;          // loads of a wave, a step and plane
    static constexpr int kBytes = T * kStepK * 2;  // of a step and plane in LDS

    const char *base[PL];
    int64_t step;  // bytes from one step to the next
    uint32_t off[kLoads];

    // k columns, rows anywhere: `row_off(r)` is the byte offset of row r of the tile
    template <typename F>
    __device__ __forceinline__ void by_row(F row_off) {
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
        step = kStepK * 2;
#pragma unroll
        for (int i = 0; i < kLoads; i++)
            off[i] = row_off((wave + 4 * i) * 16 + (lane >> 2)) + (((lane & 3) ^ ((lane >> 4) & 3)) << 4);
    }
    // a laid-out plane of `rows` rows, from row `row` and column `column` (a multiple of 32)
    __device__ __forceinline__ void laid(int p, const char *plane, int64_t rows, int64_t row, int64_t column) {
        base[p] = plane + ((column >> 5) * rows + row) * 64;
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
        step = ROWS ? kStepK * 64 : rows * 64;
#pragma unroll
        for (int i = 0; i < kLoads; i++) {
            const int j = wave + 4 * i;
            if constexpr (ROWS)
                off[i] = static_cast<uint32_t>((j >> 1) * (rows * 64)) + (j & 1) * 1024 + lane * 16;
            else
                off[i] = j * 1024 + (lane >> 2) * 64 + (((lane & 3) ^ ((lane >> 4) & 3)) << 4);
        }
    }
    __device__ __forceinline__ void load(uint32_t lds, int64_t k) const {
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
#pragma unroll
        for (int p = 0; p < PL; p++)
#pragma unroll
            for (int i = 0; i < kLoads; i++) load_to_lds(lds + p * kBytes + (wave + 4 * i) * 1024, base[p] + k * step, off[i]);
    }
};

// A wave's blocks of 32 rows of an operand in LDS
template <int PL, int T, bool ROWS, int BLOCKS>
struct Reader {
    uint32_t at[ROWS ? BLOCKS : 2];

    __device__ __forceinline__ Reader(int first) {  // first row of the wave
        const int lane = threadIdx.x & 63;
        if constexpr (ROWS) {
            const int i = (lane & 15) >> 2, a = lane & 3, half = (lane >> 4) & 1;
#pragma unroll
            for (int b = 0; b < BLOCKS; b++)
                at[b] = (first / 32 + b) * (kStepK * 64) + (8 * (lane >> 5) + i) * 64 + 32 * half + 8 * a;
        } else {
            const int r = first + (lane & 31);
#pragma unroll
            for (int ks = 0; ks < 2; ks++) at[ks] = r * 64 + (((2 * ks + (lane >> 5)) ^ ((r >> 2) & 3)) << 4);
        }
    }
    // k = 16 ks + 8 (lane / 32) + 0 ... 7 of row first + 32 b + lane % 32
    __device__ __forceinline__ half8 get(uint32_t lds, int plane, int ks, int b) const {
        const uint32_t p = lds + plane * (T * kStepK * 2);
        if constexpr (ROWS) {
            const uint32_t q = p + at[b] + ks * 16 * 64;
            const short4v x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_short4 *)(static_cast<uintptr_t>(q)));
            const short4v y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_short4 *)(static_cast<uintptr_t>(q + 4 * 64)));
            return __builtin_bit_cast(half8, __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7));
        } else {
            return *(lds_half8 *)(static_cast<uintptr_t>(p + at[ks] + b * 32 * 64));
        }
    }
};

template <bool BF>
__device__ __forceinline__ floatx16 mfma32(const half8 &a, const half8 &b, floatx16 c) {
    if constexpr (BF)
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
}

template <int PL_, int TM_, int TN_, bool AROWS, bool BROWS, bool BF>
struct Product {
    static constexpr int PL = PL_, TM = TM_, TN = TN_;
    static constexpr int IM = TM / 64, IN = TN / 64;  // blocks of a wave
    static constexpr int kStage = PL * (TM + TN) * kStepK * 2;
    static constexpr int kStages = 3 * kStage <= 76 * 1024 ? 3 : 2;  // two workgroups share a CU's LDS
    static constexpr int kLds = kStages * kStage;
    typedef Operand<PL, TM, AROWS> A;
    typedef Operand<PL, TN, BROWS> B;
    static constexpr int kLoads = PL * (A::kLoads + B::kLoads);
    static constexpr uint32_t kB = PL * A::kBytes;

    // Loads the first steps.  All waves have left the LDS of the product before.
    static __device__ __forceinline__ void begin(const A &a, const B &b, int64_t steps, uint32_t lds) {
        const int64_t ahead = steps < kStages - 1 ? steps : kStages - 1;
        for (int64_t k = 0; k < ahead; k++) {
            a.load(lds + static_cast<uint32_t>(k) * kStage, k);
            b.load(lds + static_cast<uint32_t>(k) * kStage + kB, k);
        }
    }
    // acc += the products of steps [0, steps), after begin().
    static __device__ __forceinline__ void run(const A &a, const B &b, int64_t steps, uint32_t lds, floatx16 (&acc)[IM][IN]) {
        const int wave = threadIdx.x >> 6, wm = wave & 1, wn = wave >> 1;
        const Reader<PL, TM, AROWS, IM> ra(wm * (TM / 2));
        const Reader<PL, TN, BROWS, IN> rb(wn * (TN / 2));
        uint32_t now = 0, next = (kStages - 1) * kStage;
        floatx16 low[IM][IN];
        if constexpr (PL == 2)
#pragma unroll
            for (int i = 0; i < IM; i++)
#pragma unroll
                for (int j = 0; j < IN; j++)
#pragma unroll
                    for (int k = 0; k < 16; k++) low[i][j][k] = 0.f;
        for (int64_t k = 0; k < steps; k++) {
            // the loads of this step are here, and every wave has read the step before, whose place is loaded next
            if (k + kStages - 2 < steps)
                wait_and_meet<(kStages - 2) * kLoads>();
            else
                wait_and_meet<0>();
            if (k + kStages - 1 < steps) {
                a.load(lds + next, k + kStages - 1);
                b.load(lds + next + kB, k + kStages - 1);
            }
            const uint32_t at = lds + now;
#pragma unroll
            for (int ks = 0; ks < 2; ks++) {
                half8 fa[PL][IM], fb[PL][IN];
#pragma unroll
                for (int p = 0; p < PL; p++) {
#pragma unroll
                    for (int j = 0; j < IN; j++) fb[p][j] = rb.get(at + kB, p, ks, j);
#pragma unroll
                    for (int i = 0; i < IM; i++) fa[p][i] = ra.get(at, p, ks, i);
                }
#pragma unroll
                for (int i = 0; i < IM; i++)
#pragma unroll
                    for (int j = 0; j < IN; j++) {
                        acc[i][j] = mfma32<BF>(fa[0][i], fb[0][j], acc[i][j]);
                        if constexpr (PL == 2) {
                            low[i][j] = mfma32<BF>(fa[0][i], fb[1][j], low[i][j]);
                            low[i][j] = mfma32<BF>(fa[1][i], fb[0][j], low[i][j]);
                        }
                    }
            }
            now = now + kStage == kLds ? 0 : now + kStage;
            next = next + kStage == kLds ? 0 : next + kStage;
        }
        if constexpr (PL == 2)
#pragma unroll
            for (int i = 0; i < IM; i++)
#pragma unroll
                for (int j = 0; j < IN; j++)
#pragma unroll
                    for (int k = 0; k < 16; k++) acc[i][j][k] = fmaf(low[i][j][k], kLowDown, acc[i][j][k]);
    }
};

}  // namespace yoso
