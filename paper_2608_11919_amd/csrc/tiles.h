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
struct Half {
    struct Scales {};
    template <int I>
    __device__ static inline f32x4 mul(const i32x4 (&a)[2], const i32x4 (&b)[2], f32x4 c)
    {
        c = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8, a[0]),
                                                   __builtin_bit_cast(half8, b[0]), c, 0, 0, 0);
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8, a[1]),
                                                      __builtin_bit_cast(half8, b[1]), c, 0, 0, 0);
    }
};

}  // namespace tiles

#endif
