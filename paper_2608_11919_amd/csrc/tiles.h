// tiles.h -- the matrix-core main loop that the products of the library share:
// C[m][n] += sum_k P[m][k] * Q[n][k] over one output tile, both operands with k contiguous.
//
// Operands move in bytes: a step of the loop takes 128 bytes of every row (64 fp16 or 128
// fp8 values), whole lines, from HBM straight into LDS (16 bytes a lane, no registers in
// between), into one of two buffers.  Row r keeps its 16-byte chunk c at position c ^ (r / 2 & 7):
// LDS serves 256 bytes a cycle, two rows wide, so the sixteen rows that one cycle reads at 16
// bytes each must differ in position from one pair of rows to the next (by r & 7 every read took
// twice its cycles).  The load writes LDS in lane order, by permuting what each lane fetches.
#ifndef LAZYTRAIN_TILES_H
#define LAZYTRAIN_TILES_H

#include <hip/hip_runtime.h>

#include <cstdint>
#include <type_traits>

namespace tiles {

typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));

// 16 bytes wherever an element may begin: rows of any length are read and written in them (the
// hardware takes global accesses at any address).
typedef int i32x4_any __attribute__((ext_vector_type(4), aligned(2)));

__device__ inline i32x4 load_any(const void* p) { return *static_cast<const i32x4_any*>(p); }

template <typename V>
__device__ inline void store_any(void* p, const V& v)
{
    *static_cast<i32x4_any*>(p) = __builtin_bit_cast(i32x4, v);
}

constexpr int kStepBytes = 128;  // of every row, per step of the main loop

#define LT_GLOBAL __attribute__((address_space(1)))
#define LT_LDS __attribute__((address_space(3)))

// 16 bytes a lane from `from` + offset into LDS, in lane order from `to` on.  With UNSEEN the
// compiler does not know of the copy: it waits for all that it knows of before it reads LDS other
// than by plain loads.  Waits (wait_loads) are written out either way.
template <bool UNSEEN>
__device__ inline void copy_to_lds(const uint8_t* from, uint32_t offset, uint8_t* to)
{
    if constexpr (UNSEEN) {
        const uint32_t at = uint32_t(reinterpret_cast<uintptr_t>((LT_LDS void*)(to)));
        // the compiler sets m0, and knows what is there for copies that it makes itself; one state
        // lies between
        asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %1, %2"
                     :
                     : "{m0}"(at), "v"(offset), "s"(from)
                     : "memory");
    } else {
        __builtin_amdgcn_global_load_lds((const LT_GLOBAL void*)(from + offset), (LT_LDS void*)(to),
                                         16, 0, 0);
    }
}

// ROWS rows of 128 bytes from `src` (row pitch in bytes; rows from `limit` on read the last
// row that exists) into LDS.  offset[] holds what does not change between steps.
template <int ROWS, int THREADS, bool UNSEEN = false>
struct TileLoad {
    static constexpr bool kUnseen = UNSEEN;
    static constexpr int N = ROWS * 8 / THREADS;
    static_assert(N * 32 == ROWS, "a copy is a block of 32 rows");
    uint32_t offset[N];

    __device__ inline void init(int64_t pitch, int64_t limit)
    {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int q = i * THREADS + int(threadIdx.x);
            int64_t r = q >> 3;
            const int chunk = (q & 7) ^ int(r >> 1 & 7);
            r = r < limit ? r : limit - 1;
            offset[i] = uint32_t(r * pitch) + uint32_t(chunk * 16);
        }
    }
    // the i-th of the N copies of this lane
    __device__ inline void issue(int i, const uint8_t* src, uint8_t* lds) const
    {
        const int wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x) >> 6);
        copy_to_lds<UNSEEN>(src, offset[i], lds + (i * THREADS + wave * 64) * 16);
    }
};

// The same from two matrices of one width, whose blocks of 32 rows take turns in the tile, so that
// a wave's blocks of columns 2 j and 2 j + 1 are the same rows of either.
template <int ROWS, int THREADS>
struct PairLoad {
    static constexpr bool kUnseen = false;
    static constexpr int N = ROWS * 8 / THREADS;
    static_assert(N * 32 == ROWS && N % 2 == 0, "a copy is a block of 32 rows");
    uint32_t offset[N];
    int64_t apart;  // from the first matrix to the second

    // `limit` rows of either exist from the tile's first on
    __device__ inline void init(int64_t pitch, int64_t second_pitch, const void* first,
                                const void* second, int64_t limit)
    {
        apart = reinterpret_cast<int64_t>(second) - reinterpret_cast<int64_t>(first);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int in_block = int(threadIdx.x) >> 3;
            int64_t r = i / 2 * 32 + in_block;
            const int chunk = (int(threadIdx.x) & 7) ^ (in_block >> 1 & 7);
            r = r < limit ? r : limit - 1;
            offset[i] = uint32_t(r * (i % 2 == 0 ? pitch : second_pitch)) + uint32_t(chunk * 16);
        }
    }
    __device__ inline void issue(int i, const uint8_t* src, uint8_t* lds) const
    {
        const int wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x) >> 6);
        const int64_t from = reinterpret_cast<int64_t>(src) + (i % 2 == 0 ? 0 : apart);
        __builtin_amdgcn_global_load_lds(
            (const LT_GLOBAL void*)(reinterpret_cast<const uint8_t*>(from) + offset[i]),
            (LT_LDS void*)(lds + (i * THREADS + wave * 64) * 16), 16, 0, 0);
    }
};

// Every LDS read that the wave has under way is complete: lgkmcnt(0), in the form that the
// compiler sees, which then waits for no read of its own again.
__device__ inline void wait_reads()
{
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0xC07F);
    asm volatile("" ::: "memory");
}
// Every copy into LDS but the wave's latest LEFT.
template <int LEFT>
__device__ inline void wait_loads()
{
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(LEFT) : "memory");
}

// The 32 x 32 instructions: of a step's 128 bytes of row `l % 32` of a block of 32 rows a lane
// holds 16-byte chunks l / 32, + 2, + 4 and + 6 (any assignment does that is the same for both
// operands).
typedef float f32x16 __attribute__((ext_vector_type(16)));

struct Chunks {
    i32x4 c[4];
};

__device__ inline i32x4 read_chunk(const uint8_t* tile, int row32, int c, int lane)
{
    const uint8_t* row = tile + (row32 + (lane & 31)) * kStepBytes;
    const int at = ((2 * c + (lane >> 5)) ^ (lane >> 1 & 7)) << 4;
    return *reinterpret_cast<const i32x4*>(row + at);
}

// The 16 x 16 instructions: of row 16 (c % 2) + l % 16 of the block a lane holds 16-byte chunk
// 4 (c / 2) + l / 16.
__device__ inline i32x4 read_chunk_16(const uint8_t* tile, int row32, int c, int lane)
{
    const uint8_t* row = tile + (row32 + 16 * (c & 1) + (lane & 15)) * kStepBytes;
    const int at = ((4 * (c >> 1) + (lane >> 4)) ^ (lane >> 1 & 7)) << 4;
    return *reinterpret_cast<const i32x4*>(row + at);
}

// The accumulators of a block of 32 x 32 in instructions of 16 x 16: quarter 2 i + j is rows
// 16 i .. + 15, columns 16 j .. + 15.
struct Quarters {
    f32x4 q[4];
};

// Products of fp16: 64 values a step, in four instructions; sums over multiples of 128.
struct Half {
    static constexpr int kInstructions = 4;
    static constexpr bool kOddSteps = false;
    __device__ inline void begin() {}
    __device__ inline void copy(int) {}
    __device__ inline void read(int) {}
    __device__ inline void next(int) {}
    __device__ inline f32x16 mul(int t, int, int, const Chunks& a, const Chunks& b, f32x16 c) const
    {
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(half8, a.c[t]),
                                                      __builtin_bit_cast(half8, b.c[t]), c, 0, 0,
                                                      0);
    }
};

// Products of bf16: 64 values a step, in eight instructions of 16 x 16.  PINNED, for tiles whose
// accumulators fill the accumulation registers: written out, with the operand kinds that keep them
// there (left to itself the compiler moves a third of them to and fro, and spills).  Between those
// instructions are no others of these registers; what follows the last waits (settle()).
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

template <bool PINNED>
struct Bf16 : Half {
    static constexpr int kInstructions = 8;
    static constexpr bool kOddSteps = true;
    __device__ inline Quarters mul(int t, int, int, const Chunks& a, const Chunks& b,
                                   Quarters c) const
    {
        const i32x4 p = a.c[t / 4 * 2 + t % 2], q = b.c[t / 4 * 2 + t / 2 % 2];
        if constexpr (PINNED)
            asm volatile("v_mfma_f32_16x16x32_bf16 %0, %1, %2, %0"
                         : "+a"(c.q[t % 4])
                         : "v"(p), "v"(q));
        else
            c.q[t % 4] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, p),
                                                                 __builtin_bit_cast(bf16x8, q),
                                                                 c.q[t % 4], 0, 0, 0);
        return c;
    }
};

// Products of 8-bit integers, likewise: 128 values a step.  The accumulators hold 32-bit integers'
// bits.
template <bool PINNED>
struct Int8 : Half {
    static constexpr int kInstructions = 8;
    static constexpr bool kOddSteps = true;
    __device__ inline Quarters mul(int t, int, int, const Chunks& a, const Chunks& b,
                                   Quarters c) const
    {
        const i32x4 p = a.c[t / 4 * 2 + t % 2], q = b.c[t / 4 * 2 + t / 2 % 2];
        if constexpr (PINNED)
            asm volatile("v_mfma_i32_16x16x64_i8 %0, %1, %2, %0"
                         : "+a"(c.q[t % 4])
                         : "v"(p), "v"(q));
        else
            c.q[t % 4] = __builtin_bit_cast(
                f32x4, __builtin_amdgcn_mfma_i32_16x16x64_i8(
                           p, q, __builtin_bit_cast(i32x4, c.q[t % 4]), 0, 0, 0));
        return c;
    }
};

// One BM x BN output tile by waves of WM x WN each; lane l of the wave at (wm, wn) ends with
// acc[i][j][4 g + r] = C[wm + 32 i + l % 32][wn + 32 j + 8 g + 4 (l / 32) + r]
// (the operands are swapped in the instruction, so that a lane holds consecutive columns), with
// K16, by instructions of 16 x 16, with
// acc[i][j].q[2 g + h][r] = C[wm + 32 i + 16 g + l % 16][wn + 32 j + 16 h + 4 (l / 16) + r].
template <int BM, int BN, int WM, int WN, bool K16 = false>
struct Shape {
    static constexpr bool k16 = K16;
    static constexpr int kRows = BM, kCols = BN, I = WM / 32, J = WN / 32;
    static constexpr int kWavesAcross = BN / WN, kWaves = BM / WM * kWavesAcross;
    static constexpr int kThreads = 64 * kWaves;
    static constexpr int kWavesPerSimd = WM * WN > 64 * 128 ? 1 : 2;  // at this many registers
    static constexpr bool kPinned = K16 && kWavesPerSimd == 1;
    static constexpr int kBufferBytes = (BM + BN) * kStepBytes;
    static constexpr int kLdsBytes = 2 * kBufferBytes;
    static constexpr int kRun = 32 * (kWavesPerSimd == 2 ? 2 : 1);  // tiles an XCD's 32 CUs hold
    typename std::conditional<K16, Quarters, f32x16>::type acc[I][J];

    __device__ static inline int wave() { return __builtin_amdgcn_readfirstlane(int(threadIdx.x) >> 6); }
    __device__ static inline int lane() { return int(threadIdx.x) & 63; }
    __device__ static inline int wave_row() { return wave() / kWavesAcross * WM; }
    __device__ static inline int wave_col() { return wave() % kWavesAcross * WN; }
    __device__ inline f32x4 four(int i, int j, int g) const
    {
        if constexpr (K16)
            return acc[i][j].q[g];
        else
            return f32x4{acc[i][j][4 * g], acc[i][j][4 * g + 1], acc[i][j][4 * g + 2],
                         acc[i][j][4 * g + 3]};
    }
    // before the first and after the last of the pinned instructions: what writes the accumulators
    // is done with them before what reads them begins
    __device__ inline void settle()
    {
        asm volatile("s_nop 15\n\ts_nop 15");
#pragma unroll
        for (int i = 0; i < I; ++i)
#pragma unroll
            for (int j = 0; j < J; ++j)
#pragma unroll
                for (int g = 0; g < 4; ++g)
                    asm volatile("" : "+a"(acc[i][j].q[g]));
    }
    __device__ inline void clear()
    {
#pragma unroll
        for (int i = 0; i < I; ++i)
#pragma unroll
            for (int j = 0; j < J; ++j) {
                if constexpr (K16) {
#pragma unroll
                    for (int g = 0; g < 4; ++g)
                        acc[i][j].q[g] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
                } else {
#pragma unroll
                    for (int r = 0; r < 16; ++r)
                        acc[i][j][r] = 0.0f;
                }
            }
    }
    // this lane's row of block i, and the first of its four columns g of block j, in the tile
    __device__ static inline int row(int i) { return wave_row() + 32 * i + (lane() & 31); }
    __device__ static inline int col(int j, int g) { return wave_col() + 32 * j + 8 * g + 4 * (lane() >> 5); }
};

// The work unit of this workgroup.  Workgroups go to the eight XCDs in turn, each with an L2 of
// its own; units are dealt out so that an XCD works on `run` consecutive units at a time (as
// many as it holds workgroups), which tile_place makes neighbours that share operands.
__device__ inline int64_t unit_of_workgroup(uint32_t b, uint32_t n, int run)
{
    const uint32_t round = 8u * uint32_t(run);
    const uint32_t base = b / round * round, here = min(round, n - base);
    const uint32_t x = b % 8u, i = (b - base) / 8u;
    return int64_t(base + x * (here / 8u) + min(x, here % 8u) + i);
}
__device__ inline int64_t unit_of_workgroup(int run)
{
    return unit_of_workgroup(blockIdx.x, gridDim.x, run);
}

// Row and column of the t-th tile of `down` x `across`: strips of eight rows, column by column.
struct TilePlace {
    int row, col;
};

constexpr int kStrip = 8;

__device__ inline TilePlace tile_place(int t, int down, int across)
{
    const int strip = t / (kStrip * across), first = strip * kStrip;
    const int high = min(kStrip, down - first), left = t - first * across;
    return {first + left % high, left / high};
}

// The same for the tiles on and above the diagonal of side x side.
__device__ inline TilePlace triangle_place(int t, int side)
{
    int first = 0;
    for (;; first += kStrip) {
        const int high = min(kStrip, side - first);
        const int corner = high * (high + 1) / 2, all = corner + (side - first - high) * high;
        if (t >= all) {
            t -= all;
            continue;
        }
        if (t >= corner)
            return {first + (t - corner) % high, first + high + (t - corner) / high};
        int col = 0;
        while (t > col)
            t -= ++col;
        return {first + t, first + col};
    }
}

// Four waves each.  A Large tile has the fewest bytes to copy for a product (two operands' rows
// for 256 results a row) and one workgroup a CU; where there are too few of those, smaller ones.
typedef Shape<64, 64, 32, 32> Tiny;
typedef Shape<128, 128, 64, 64> Small;
typedef Shape<256, 256, 128, 128> Large;
// The same by instructions of 16 x 16.  They take twice the operands' registers for a product and
// half the accumulators': less power.
typedef Shape<64, 64, 32, 32, true> Tiny16;
typedef Shape<128, 128, 64, 64, true> Small16;
typedef Shape<256, 256, 128, 128, true> Large16;
// The smallest tile in which a wave has two blocks of columns.
typedef Shape<64, 128, 32, 64, true> Pair16;

// Products of fp8 (e4m3) with a power-of-two scale for each row and each 128 values: a step's in
// two instructions of 64, which apply the scales themselves.  A scale is a byte, the
// exponent biased by 127; four steps' worth are a word, copied into LDS four steps at a time.
template <typename S>
struct Fp8 {
    static constexpr int kInstructions = 2;
    static constexpr bool kOddSteps = true;
    static constexpr int kRowsAll = S::kRows + S::kCols, kLdsBytes = 2 * kRowsAll * 4;
    const uint8_t *scales_p, *scales_q;  // of the tile's first rows, at the first step
    int64_t pitch, limit_p, limit_q;     // bytes of a row's scales; rows that exist
    int words;                           // of four steps
    uint8_t* lds;                        // kLdsBytes
    uint32_t now_p[S::I], now_q[S::J], then_p[S::I], then_q[S::J];

    // words w of all rows of the tile into their buffer
    __device__ inline void copy_word(int w)
    {
        const int64_t at = int64_t(w < words ? w : words - 1) * 4;
        uint8_t* to = lds + (w & 1) * kRowsAll * 4;
#pragma unroll
        for (int first = 0; first < kRowsAll; first += S::kThreads) {
            const int base = first + S::wave() * 64;
            if (base >= kRowsAll)
                break;
            const bool is_p = base < S::kRows;
            int64_t r = (is_p ? base : base - S::kRows) + S::lane();
            const int64_t limit = is_p ? limit_p : limit_q;
            r = r < limit ? r : limit - 1;
            __builtin_amdgcn_global_load_lds(
                (const LT_GLOBAL void*)((is_p ? scales_p : scales_q) + r * pitch + at),
                (LT_LDS void*)(to + base * 4), 4, 0, 0);
        }
    }
    __device__ inline void begin() { copy_word(0); }
    // before step s: the buffer of the word before last is free
    __device__ inline void copy(int s)
    {
        if ((s & 3) == 0)
            copy_word((s >> 2) + 1);
    }
    // the word that holds the scales of step s
    __device__ inline void read(int s)
    {
        const auto* from = reinterpret_cast<const uint32_t*>(lds + (s >> 2 & 1) * kRowsAll * 4);
#pragma unroll
        for (int i = 0; i < S::I; ++i)
            then_p[i] = from[S::row(i)];
#pragma unroll
        for (int j = 0; j < S::J; ++j)
            then_q[j] = from[S::kRows + S::wave_col() + 32 * j + (S::lane() & 31)];
    }
    // its byte, where the multiplies look for it
    __device__ inline void next(int s)
    {
        const int shift = 8 * (s & 3);
#pragma unroll
        for (int i = 0; i < S::I; ++i)
            now_p[i] = then_p[i] >> shift;
#pragma unroll
        for (int j = 0; j < S::J; ++j)
            now_q[j] = then_q[j] >> shift;
    }
    __device__ inline f32x16 mul(int t, int i, int j, const Chunks& a, const Chunks& b,
                                 f32x16 c) const
    {
        const auto join = [t](const Chunks& x) {
            const i32x4 u = x.c[2 * t], v = x.c[2 * t + 1];
            return i32x8{u[0], u[1], u[2], u[3], v[0], v[1], v[2], v[3]};
        };
        return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(join(a), join(b), c, 0, 0, 0,
                                                               int(now_q[j]), 0, int(now_p[i]));
    }
};

// A wave's blocks of rows in two groups, see below: the blocks [first, first + n) of group g of
// `all`.
struct Groups {
    static constexpr int n(int all, int g) { return g == 0 ? (all + 1) / 2 : all / 2; }
    static constexpr int first(int all, int g) { return g == 0 ? 0 : (all + 1) / 2; }
};

// An address that is the same in all lanes, in scalar registers, for written-out copies: a vector
// instruction's result there may be an address five instructions later.
__device__ inline const uint8_t* uniform(const uint8_t* p)
{
    const auto v = reinterpret_cast<uint64_t>(p);
    const uint64_t low = uint32_t(__builtin_amdgcn_readfirstlane(int(uint32_t(v))));
    const uint64_t high = uint32_t(__builtin_amdgcn_readfirstlane(int(uint32_t(v >> 32))));
    uint64_t same = high << 32 | low;
    asm volatile("s_nop 4" : "+s"(same));
    return reinterpret_cast<const uint8_t*>(same);
}

// What the main loop does with an operand of ROWS rows in the tile, BLOCKS blocks of 32 to a wave:
//   copies(g)             copies of group g's rows, of all waves, in a step;
//   aim(s)                the next copies are step s's;
//   issue(g, k, to)       the k-th of group g's into the operand's place in a buffer;
//   read(from, at, block, c, lane)  a lane's c-th chunk of a block of the wave whose first row is at.
// This one has rows with k contiguous.
template <typename S, int ROWS, int BLOCKS, typename Load>
struct RowOperand {
    const uint8_t* src;
    int steps;
    const uint8_t* now;
    Load load;

    static constexpr int copies(int g) { return ROWS / 32 / BLOCKS * Groups::n(BLOCKS, g); }
    __device__ inline void aim(int s)
    {
        now = src + int64_t(s < steps ? s : steps - 1) * kStepBytes;
        if constexpr (Load::kUnseen)
            now = uniform(now);
    }
    __device__ inline void issue(int g, int k, uint8_t* to) const
    {
        const int n = Groups::n(BLOCKS, g);
        load.issue(k / n * BLOCKS + Groups::first(BLOCKS, g) + k % n, now, to);
    }
    __device__ static inline i32x4 read(const uint8_t* from, int at, int block, int c, int lane)
    {
        return S::k16 ? read_chunk_16(from, at + 32 * block, c, lane)
                      : read_chunk(from, at + 32 * block, c, lane);
    }
};

// Where a step of a turned operand lies: in the first matrix, then in the second, each with `each`
// steps of 64 rows; rows from the full ones on are in copies of their own, zeros behind the last.
struct TurnedSource {
    const uint8_t* base[2];
    const uint8_t* tail[2];
    int64_t pitch;  // bytes, of either
    int each, full;
    __device__ inline const uint8_t* at(int s) const
    {
        const int which = s >= each ? 1 : 0, t = s - which * each;
        return t < full ? (which ? base[1] : base[0]) + int64_t(t) * 64 * pitch
                        : (which ? tail[1] : tail[0]);
    }
};

// This one, of 16-bit values, has the summed index as rows: its tile is 64 rows of the operand's
// columns, read out of LDS four rows of a column at a time (ds_read_b64_tr_b16: of sixteen lanes,
// lanes 4 j .. 4 j + 3 read 16 neighbouring columns of row j, and lane i gets the four rows of
// column i).  A group's columns, of all waves, are an image of their own, so that it is copied and
// free as the group is; rows of 256 bytes (two blocks to a group) or 128.  A cycle serves eight rows
// {0 .. 3, 8 .. 11} of 32 bytes: 16-byte chunk c of row k is at position c ^ f(k), which puts them
// next to each other.  The other operand's copies have to be UNSEEN as this one's are.
template <typename S, int ROWS, int BLOCKS>
struct TurnedOperand {
    static constexpr int kAlong = ROWS / 32 / BLOCKS;  // waves
    TurnedSource src;
    int first, steps;  // of the sum's slice
    const uint8_t* now;
    uint32_t offset[2];

    static constexpr int copies(int g) { return kAlong * Groups::n(BLOCKS, g); }
    static constexpr int pitch(int g) { return 2 * 32 * kAlong * Groups::n(BLOCKS, g); }
    static constexpr int image(int g) { return g == 0 ? 0 : 64 * pitch(0); }
    __device__ static inline int place(int g, int chunk, int row)
    {
        return pitch(g) == 256 ? chunk ^ 2 * ((row & 3) + 4 * (row >> 3 & 1))
                               : chunk ^ 2 * ((row >> 1 & 1) + 2 * (row >> 3 & 1));
    }
    // `limit` columns, a multiple of 8, exist from the tile's first on
    __device__ inline void init(int64_t limit)
    {
#pragma unroll
        for (int g = 0; g < 2; ++g) {
            const int n = Groups::n(BLOCKS, g);
            if (n == 0)
                continue;
            const int byte = int(threadIdx.x) * 16, row = byte / pitch(g);
            const int col = place(g, byte % pitch(g) / 16, row) * 8;  // its own inverse
            int64_t at = col / (32 * n) * (32 * BLOCKS) + 32 * Groups::first(BLOCKS, g) +
                         col % (32 * n);
            at = at < limit ? at : limit - 8;
            offset[g] = uint32_t(row * src.pitch) + uint32_t(at * 2);
        }
    }
    __device__ inline void aim(int s)
    {
        now = uniform(src.at(first + (s < steps ? s : steps - 1)));
    }
    __device__ inline void issue(int g, int k, uint8_t* to) const
    {
        const int wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x) >> 6);
        copy_to_lds<true>(now + int64_t(k) * (4096 / pitch(g)) * src.pitch, offset[g],
                          to + image(g) + k * 4096 + wave * 1024);
    }
    __device__ static inline i32x4 read(const uint8_t* from, int at, int block, int c, int lane)
    {
        typedef short s16x4 __attribute__((ext_vector_type(4)));
        typedef int i32x2 __attribute__((ext_vector_type(2)));
        const int g = block < Groups::n(BLOCKS, 0) ? 0 : 1, n = Groups::n(BLOCKS, g);
        const int col = at / (32 * BLOCKS) * 32 * n + 32 * (block - Groups::first(BLOCKS, g)) +
                        16 * (c & 1);
        const int row = 32 * (c >> 1) + 8 * (lane >> 4) + (lane >> 2 & 3);
        const uint8_t* p = from + image(g) + row * pitch(g) +
                           place(g, col / 8 + (lane >> 1 & 1), row) * 16 + (lane & 1) * 8;
        const auto four = [](const uint8_t* q) {
            return __builtin_bit_cast(
                i32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((LT_LDS s16x4*)(q)));
        };
        const i32x2 u = four(p), v = four(p + 4 * pitch(g));  // four rows on: the same place
        return i32x4{u[0], u[1], v[0], v[1]};
    }
};

// The main loop over `steps` >= 1 steps of the operands p and q.
//
// A wave's block is multiplied in four quarters: the rows' blocks of 32 in two groups a0 and a1,
// the columns' in b0 and b1, in an order in which neighbours share a group:
//   even steps  a0 b0, a0 b1, a1 b1, a1 b0;   odd steps  a0 b1, a0 b0, a1 b0, a1 b1.
// A group's registers are free once its last quarter is multiplied, and take the next step's
// operands out of LDS during the quarters after: b1, a1, then the next step's a0 and b1 (odd
// steps: b0, a1, a0, b0).  A step's first two reads are its late rows, the others early rows of
// the next; each half of a step ends with a barrier, after which all waves have the rows read in
// it in registers, and during the next half the copy of the step after next goes into their
// place.  A copy has three halves' products' time to land, counted by the wave's own copies, and
// copies come evenly, eight to a half: L2 feeds a CU some 26 bytes a cycle (15 TB/s in all),
// and products of fp8 in tiles of 256 take 32.  In stages of 64 bytes of every row, half lines,
// the copies alone took a fifth longer.
// A body of two steps has no branches but one at its top: past the end it copies and reads the
// last step again, unused, and a branch inside made the compiler move all products before it
// behind it, away from the loads that they cover.
template <typename Mul, typename S, typename OpP, typename OpQ>
__device__ inline void product(Mul& mul, S& c, OpP& p, OpQ& q, int steps, uint8_t* lds)
{
    constexpr int I = S::I, J = S::J;
    const int lane = S::lane(), wm = S::wave_row(), wn = S::wave_col();
    constexpr int kLoads = (S::kRows + S::kCols) * 8 / S::kThreads;
    // copies of the early or late rows of an even (0) or odd (1) step
    constexpr auto copies = [](int odd, int late) {
        return OpP::copies(late) + OpQ::copies(odd ^ late);
    };
    Chunks a[I], b[J];
    // the k-th copy of the early or late rows of the step that is aimed at
    const auto load = [&](int odd, int late, int k) {
        uint8_t* to = lds + odd * S::kBufferBytes;
        if (k < OpP::copies(late))
            p.issue(late, k, to);
        else
            q.issue(odd ^ late, k - OpP::copies(late), to + S::kRows * kStepBytes);
    };
    const auto read_a = [&](int odd, int g, int k) {
        const int i = Groups::first(I, g) + k / 4;
        a[i].c[k % 4] = p.read(lds + odd * S::kBufferBytes, wm, i, k % 4, lane);
    };
    const auto read_b = [&](int odd, int g, int k) {
        const int j = Groups::first(J, g) + k / 4;
        b[j].c[k % 4] =
            q.read(lds + odd * S::kBufferBytes + S::kRows * kStepBytes, wn, j, k % 4, lane);
    };
    // the products of groups ga and gb, with reads and copies issued evenly between them: reads
    // within the first three quarters, so that the last covers their latency.  Every border
    // keeps its place: left to itself the compiler issues reads right before the products that
    // wait for them, and products ahead of the barrier.
    const auto multiply = [&](int ga, int gb, int reads, auto read_next, int loads, auto copy) {
        const int ni = Groups::n(I, ga), nj = Groups::n(J, gb);
        const int muls = ni * nj * Mul::kInstructions, paced = muls * 3 / 4;
        const auto share = [](int n, int of, int k) { return k < of ? n * k / of : n; };
        if (muls == 0) {
#pragma unroll
            for (int r = 0; r < loads; ++r)
                copy(r);
#pragma unroll
            for (int r = 0; r < reads; ++r)
                read_next(r);
            return;
        }
#pragma unroll
        for (int k = 0; k < muls; ++k) {
#pragma unroll
            for (int r = share(loads, muls, k); r < share(loads, muls, k + 1); ++r)
                copy(r);
#pragma unroll
            for (int r = share(reads, paced, k); r < share(reads, paced, k + 1); ++r)
                read_next(r);
            const int t = k / (ni * nj), i = Groups::first(I, ga) + k / nj % ni,
                      j = Groups::first(J, gb) + k % nj;
            c.acc[i][j] = mul.mul(t, i, j, b[j], a[i], c.acc[i][j]);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    // step s, odd or even
    const auto step = [&](int s, auto parity) {
        constexpr int odd = decltype(parity)::value;
        constexpr int early = copies(odd, 0), late = copies(odd, 1);
        constexpr int b_first = odd, b_second = 1 - odd;
        mul.next(s);
        p.aim(s + 2);
        q.aim(s + 2);
        multiply(0, b_first, 4 * Groups::n(J, b_second), [&](int k) { read_b(odd, b_second, k); },
                 early / 2, [&](int k) { load(odd, 0, k); });
        multiply(0, b_second, 4 * Groups::n(I, 1), [&](int k) { read_a(odd, 1, k); },
                 early - early / 2, [&](int k) { load(odd, 0, early / 2 + k); });
        wait_reads();
        wait_loads<early + copies(1 - odd, 1)>();  // the next step's early rows are there
        __builtin_amdgcn_s_barrier();
        mul.read(s + 1);
        multiply(1, b_second, 4 * Groups::n(I, 0), [&](int k) { read_a(1 - odd, 0, k); },
                 late / 2, [&](int k) { load(odd, 1, k); });
        multiply(1, b_first, 4 * Groups::n(J, b_second),
                 [&](int k) { read_b(1 - odd, b_second, k); }, late - late / 2,
                 [&](int k) { load(odd, 1, late / 2 + k); });
        wait_reads();
        wait_loads<kLoads>();  // and its late rows
        __builtin_amdgcn_s_barrier();
    };
    c.clear();
    if constexpr (S::kPinned)
        c.settle();
    mul.begin();
#pragma unroll
    for (int s = 0; s < 2; ++s) {
        p.aim(s);
        q.aim(s);
#pragma unroll
        for (int k = 0; k < kLoads; ++k) {
            const int early = copies(s, 0);
            load(s, k >= early, k < early ? k : k - early);
        }
    }
    wait_loads<kLoads>();
    __builtin_amdgcn_s_barrier();
    mul.read(0);
#pragma unroll
    for (int k = 0; k < 4 * Groups::n(I, 0); ++k)
        read_a(0, 0, k);
#pragma unroll
    for (int k = 0; k < 4 * Groups::n(J, 0); ++k)
        read_b(0, 0, k);
    wait_reads();
    __builtin_amdgcn_s_barrier();
    int s = 0;
#pragma unroll 1
    for (; s + 2 <= steps; s += 2) {
        mul.copy(s);
        step(s, std::integral_constant<int, 0>());
        step(s + 1, std::integral_constant<int, 1>());
    }
    if constexpr (Mul::kOddSteps)
        if (s < steps)
            step(s, std::integral_constant<int, 0>());
    if constexpr (S::kPinned)
        c.settle();
    wait_loads<0>();
    __builtin_amdgcn_s_barrier();  // nothing is on its way into LDS any more
}

// The same for operands of pitches in bytes, of which limit_p and limit_q rows exist.
template <typename Mul, typename S>
__device__ inline void product(Mul& mul, S& c, const void* P, int64_t pitch_p, int64_t limit_p,
                               const void* Q, int64_t pitch_q, int64_t limit_q, int steps,
                               uint8_t* lds)
{
    RowOperand<S, S::kRows, S::I, TileLoad<S::kRows, S::kThreads>> p;
    RowOperand<S, S::kCols, S::J, TileLoad<S::kCols, S::kThreads>> q;
    p.src = static_cast<const uint8_t*>(P);
    q.src = static_cast<const uint8_t*>(Q);
    p.steps = q.steps = steps;
    p.load.init(pitch_p, limit_p);
    q.load.init(pitch_q, limit_q);
    product(mul, c, p, q, steps, lds);
}

// For two matrices' rows in turns (PairLoad): columns [0, kCols / 2) of both results.
template <typename Mul, typename S>
__device__ inline void product_pairs(Mul& mul, S& c, const void* P, int64_t pitch_p,
                                     int64_t limit_p, const void* first, int64_t first_pitch,
                                     const void* second, int64_t second_pitch, int64_t limit_q,
                                     int steps, uint8_t* lds)
{
    RowOperand<S, S::kRows, S::I, TileLoad<S::kRows, S::kThreads>> p;
    RowOperand<S, S::kCols, S::J, PairLoad<S::kCols, S::kThreads>> q;
    p.src = static_cast<const uint8_t*>(P);
    q.src = static_cast<const uint8_t*>(first);
    p.steps = q.steps = steps;
    p.load.init(pitch_p, limit_p);
    q.load.init(first_pitch, second_pitch, first, second, limit_q);
    product(mul, c, p, q, steps, lds);
}

// What follows the main loop, for one wave's block, 32 rows at a time through LDS (the loop is
// done with it): a lane then has eight consecutive columns of a row, so that a wave reads and
// writes whole lines, and the code is a few short loops.  From the registers as they come a lane
// has four columns of 32 rows: accesses of 16 bytes a row, unrolled to 36 to 118 KB of code.
// Writer w:
//   w.fetch(row, col, p)     requests what results [row][col .. col + 8) need, into slot p;
//   w.store(row, col, v, p)  takes the sums v, leaves the results there and stores them;
//   w.turn(col, row, v)      with kTurned: stores results [row .. row + 8)[col] of the transpose;
//   w.columns(col)           where it has it: before all, the lane's columns [col .. col + 8).
// Rows and columns count from the tile's origin.
template <typename Writer>
__device__ inline auto tell_columns(Writer& w, int col, int) -> decltype(w.columns(col))
{
    w.columns(col);
}
template <typename Writer>
__device__ inline void tell_columns(Writer&, int, long)
{
}

template <typename S, typename Writer>
__device__ inline void finish(const S& c, uint8_t* lds, Writer& w)
{
    constexpr int W = 32 * S::J, kAcross = W / 8, kDown = 64 / kAcross, kPasses = 32 / kDown;
    constexpr int kPitch = W + 4;
    static_assert(S::kWaves * 32 * kPitch * 4 <= S::kLdsBytes, "every wave's rows fit");
    static_assert(kPasses <= Writer::kSlots, "a slot for every pass");
    float* mine = reinterpret_cast<float*>(lds) + S::wave() * 32 * kPitch;
    const int lane = S::lane(), down = lane / kAcross, across = lane % kAcross * 8;
    const int r0 = S::wave_row(), c0 = S::wave_col();
    tell_columns(w, c0 + across, 0);
#pragma unroll
    for (int i = 0; i < S::I; ++i) {
#pragma unroll
        for (int p = 0; p < kPasses; ++p)
            w.fetch(r0 + 32 * i + p * kDown + down, c0 + across, p);
#pragma unroll
        for (int jg = 0; jg < 4 * S::J; ++jg) {
            const int j = jg / 4, g = jg % 4;
            *reinterpret_cast<f32x4*>(mine + (S::k16 ? 16 * (g >> 1) + (lane & 15) : lane & 31) *
                                             kPitch +
                                      32 * j + (S::k16 ? 16 * (g & 1) + 4 * (lane >> 4)
                                                       : 8 * g + 4 * (lane >> 5))) =
                c.four(i, j, g);
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
        for (int p = 0; p < kPasses; ++p) {
            float* at = mine + (p * kDown + down) * kPitch + across;
            float v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e)
                v[e] = at[e];
            w.store(r0 + 32 * i + p * kDown + down, c0 + across, v, p);
            if constexpr (Writer::kTurned) {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    at[e] = v[e];
            }
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        if constexpr (Writer::kTurned) {
#pragma unroll
            for (int q = 0; q < W / 16; ++q) {
                const int col = q * 16 + lane / 4, row = lane % 4 * 8;
                float v[8];
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    v[e] = mine[(row + e) * kPitch + col];
                w.turn(c0 + col, r0 + 32 * i + row, v);
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        }
    }
}

// The same for results of two matrices' rows in turns:
//   w.fetch(row)               requests what a row's results need;
//   w.store(row, col, u, v, f) takes eight neighbouring columns of either result, which count in
//                              [0, kCols / 2), and what fetch gave.
template <typename S, typename Writer>
__device__ inline void finish_pairs(const S& c, uint8_t* lds, Writer& w)
{
    constexpr int W = 32 * S::J, kAcross = W / 16, kDown = 64 / kAcross, kPasses = 32 / kDown;
    constexpr int kPitch = W + 4;
    static_assert(S::J % 2 == 0 && S::kWaves * 32 * kPitch * 4 <= S::kLdsBytes,
                  "every wave's rows fit");
    float* mine = reinterpret_cast<float*>(lds) + S::wave() * 32 * kPitch;
    const int lane = S::lane(), down = lane / kAcross, across = lane % kAcross * 8;
    const int r0 = S::wave_row(), c0 = S::wave_col() / 2;
    tell_columns(w, c0 + across, 0);
    auto next = w.fetch(r0 + down);
#pragma unroll
    for (int i = 0; i < S::I; ++i) {
#pragma unroll
        for (int jg = 0; jg < 4 * S::J; ++jg) {
            const int j = jg / 4, g = jg % 4;
            *reinterpret_cast<f32x4*>(mine + (S::k16 ? 16 * (g >> 1) + (lane & 15) : lane & 31) *
                                             kPitch +
                                      32 * j + (S::k16 ? 16 * (g & 1) + 4 * (lane >> 4)
                                                       : 8 * g + 4 * (lane >> 5))) =
                c.four(i, j, g);
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
// two passes' chains of instructions overlap (4096 x 2048 x 11008 in integers 222 to 213 us); four
// gain nothing
#pragma unroll 2
        for (int p = 0; p < kPasses; ++p) {
            const float* at = mine + (p * kDown + down) * kPitch + across / 32 * 64 + across % 32;
            float u[8], v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                u[e] = at[e];
                v[e] = at[32 + e];
            }
            const auto now = next;  // rows follow each other, also from block to block
            const int row = r0 + 32 * i + p * kDown + down;
            next = w.fetch(row + kDown);
            w.store(row, c0 + across, u, v, now);
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
}

}  // namespace tiles

#endif
