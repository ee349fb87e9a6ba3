// tiles.h -- the matrix-core main loop that the products of the library share:
// C[m][n] += sum_k P[m][k] * Q[n][k] over one output tile, both operands with k contiguous.
//
// Operands move in bytes: a step of the loop takes 128 bytes of every row (64 fp16 or 128
// fp8 values), from HBM straight into LDS (16 bytes a lane, no registers in between), into
// one of two buffers while the other is multiplied.  Row r keeps its 16-byte chunk c at
// position c ^ (r & 7): the eight rows that one LDS cycle serves then fall on different
// banks, and the load writes LDS in lane order by permuting what each lane fetches.
#ifndef LAZYTRAIN_TILES_H
#define LAZYTRAIN_TILES_H

#include <hip/hip_runtime.h>

#include <cstdint>

namespace tiles {

typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));

constexpr int kStepBytes = 128;  // of every row, per step of the main loop

#define LT_GLOBAL __attribute__((address_space(1)))
#define LT_LDS __attribute__((address_space(3)))

// ROWS rows of 128 bytes from `src` (row pitch in bytes; rows from `limit` on read the last
// row that exists) into LDS.  offset[] holds what does not change between steps.
template <int ROWS, int THREADS>
struct TileLoad {
    static constexpr int N = ROWS * 8 / THREADS;
    static_assert(ROWS * 8 % THREADS == 0, "whole chunks per lane");
    uint32_t offset[N];

    __device__ inline void init(int64_t pitch, int64_t limit)
    {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int q = i * THREADS + int(threadIdx.x);
            int64_t r = q >> 3;
            const int chunk = (q & 7) ^ int(r & 7);
            r = r < limit ? r : limit - 1;
            offset[i] = uint32_t(r * pitch) + uint32_t(chunk * 16);
        }
    }
    __device__ inline void issue(const uint8_t* src, uint8_t* lds) const
    {
        const int wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x) >> 6);
#pragma unroll
        for (int i = 0; i < N; ++i)
            __builtin_amdgcn_global_load_lds(
                (const LT_GLOBAL void*)(src + offset[i]),
                (LT_LDS void*)(lds + (i * THREADS + wave * 64) * 16), 16, 0, 0);
    }
};

__device__ inline void wait_loads() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

// A lane's two 16-byte chunks of row `row16 + lane % 16`: chunks lane / 16 and lane / 16 + 4.
__device__ inline void read_chunks(const uint8_t* tile, int row16, int lane, i32x4 (&c)[2])
{
    const uint8_t* row = tile + (row16 + (lane & 15)) * kStepBytes;
    const int at = ((lane >> 4) ^ (lane & 7)) << 4;
    c[0] = *reinterpret_cast<const i32x4*>(row + at);
    c[1] = *reinterpret_cast<const i32x4*>(row + (at ^ 64));
}

// Products of 16-bit floating point; the lane's chunks hold k = 8 * (lane / 16) + 0..7 of the
// step's first and second 32 values, alike for both operands.
__device__ inline f32x4 mul_half(const i32x4 (&a)[2], const i32x4 (&b)[2], f32x4 c)
{
    c = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8, a[0]),
                                               __builtin_bit_cast(half8, b[0]), c, 0, 0, 0);
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8, a[1]),
                                                  __builtin_bit_cast(half8, b[1]), c, 0, 0, 0);
}

// One BM x BN output tile by waves of WM x WN each; lane l of the wave at (wm, wn) ends with
// acc[i][j][r] = C[wm + 16 i + l % 16][wn + 16 j + 4 (l / 16) + r]
// (the operands are swapped in the instruction, so that a lane holds consecutive columns).
template <int BM, int BN, int WM, int WN>
struct Shape {
    static constexpr int kRows = BM, kCols = BN, I = WM / 16, J = WN / 16;
    static constexpr int kWavesAcross = BN / WN, kWaves = BM / WM * kWavesAcross;
    static constexpr int kThreads = 64 * kWaves;
    static constexpr int kBufferBytes = (BM + BN) * kStepBytes;
    static constexpr int kLdsBytes = 2 * kBufferBytes;
    f32x4 acc[I][J];

    __device__ static inline int wave() { return __builtin_amdgcn_readfirstlane(int(threadIdx.x) >> 6); }
    __device__ static inline int lane() { return int(threadIdx.x) & 63; }
    // this lane's row of block i and first column of block j within the tile
    __device__ static inline int row(int i) { return wave() / kWavesAcross * WM + 16 * i + (lane() & 15); }
    __device__ static inline int col(int j)
    {
        return wave() % kWavesAcross * WN + 16 * j + 4 * (lane() >> 4);
    }
};

typedef Shape<128, 128, 64, 64> Small;
typedef Shape<256, 256, 128, 64> Large;

// The main loop over `steps` >= 1 steps.  P, Q: first rows of the tile's operands, pitches in
// bytes, of which limit_p and limit_q rows exist.
template <typename S>
__device__ inline void product_half(S& c, const void* P, int64_t pitch_p, int64_t limit_p,
                                    const void* Q, int64_t pitch_q, int64_t limit_q, int steps,
                                    uint8_t* lds)
{
    const int lane = S::lane(), wm = S::wave() / S::kWavesAcross * (16 * S::I),
              wn = S::wave() % S::kWavesAcross * (16 * S::J);
    TileLoad<S::kRows, S::kThreads> load_p;
    TileLoad<S::kCols, S::kThreads> load_q;
    load_p.init(pitch_p, limit_p);
    load_q.init(pitch_q, limit_q);
    const auto* p = static_cast<const uint8_t*>(P);
    const auto* q = static_cast<const uint8_t*>(Q);
#pragma unroll
    for (int i = 0; i < S::I; ++i)
#pragma unroll
        for (int j = 0; j < S::J; ++j)
            c.acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    load_p.issue(p, lds);
    load_q.issue(q, lds + S::kRows * kStepBytes);
#pragma unroll 1
    for (int s = 0; s < steps; ++s) {
        uint8_t* now = lds + (s & 1) * S::kBufferBytes;
        uint8_t* next = lds + (~s & 1) * S::kBufferBytes;
        wait_loads();
        __syncthreads();  // the step's tiles are in place, and no wave reads the other buffer
        if (s + 1 < steps) {
            load_p.issue(p + int64_t(s + 1) * kStepBytes, next);
            load_q.issue(q + int64_t(s + 1) * kStepBytes, next + S::kRows * kStepBytes);
        }
        i32x4 b[S::J][2];
#pragma unroll
        for (int j = 0; j < S::J; ++j)
            read_chunks(now + S::kRows * kStepBytes, wn + 16 * j, lane, b[j]);
#pragma unroll
        for (int i = 0; i < S::I; ++i) {
            i32x4 a[2];
            read_chunks(now, wm + 16 * i, lane, a);
#pragma unroll
            for (int j = 0; j < S::J; ++j)
                c.acc[i][j] = mul_half(b[j], a, c.acc[i][j]);
        }
    }
}

}  // namespace tiles

#endif
