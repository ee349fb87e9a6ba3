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

// ROWS rows of 128 bytes from `src` (row pitch in bytes; rows from `limit` on read the last
// row that exists) into LDS.  offset[] holds what does not change between steps.
template <int ROWS, int THREADS>
struct TileLoad {
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
        __builtin_amdgcn_global_load_lds((const LT_GLOBAL void*)(src + offset[i]),
                                         (LT_LDS void*)(lds + (i * THREADS + wave * 64) * 16), 16,
                                         0, 0);
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

// One BM x BN output tile by waves of WM x WN each; lane l of the wave at (wm, wn) ends with
// acc[i][j][4 g + r] = C[wm + 32 i + l % 32][wn + 32 j + 8 g + 4 (l / 32) + r]
// (the operands are swapped in the instruction, so that a lane holds consecutive columns).
template <int BM, int BN, int WM, int WN>
struct Shape {
    static constexpr int kRows = BM, kCols = BN, I = WM / 32, J = WN / 32;
    static constexpr int kWavesAcross = BN / WN, kWaves = BM / WM * kWavesAcross;
    static constexpr int kThreads = 64 * kWaves;
    static constexpr int kWavesPerSimd = WM * WN > 64 * 128 ? 1 : 2;  // at this many registers
    static constexpr int kBufferBytes = (BM + BN) * kStepBytes;
    static constexpr int kLdsBytes = 2 * kBufferBytes;
    static constexpr int kRun = 32 * (kWavesPerSimd == 2 ? 2 : 1);  // tiles an XCD's 32 CUs hold
    f32x16 acc[I][J];

    __device__ static inline int wave() { return __builtin_amdgcn_readfirstlane(int(threadIdx.x) >> 6); }
    __device__ static inline int lane() { return int(threadIdx.x) & 63; }
    __device__ static inline int wave_row() { return wave() / kWavesAcross * WM; }
    __device__ static inline int wave_col() { return wave() % kWavesAcross * WN; }
    // this lane's row of block i, and the first of its four columns g of block j, in the tile
    __device__ static inline int row(int i) { return wave_row() + 32 * i + (lane() & 31); }
    __device__ static inline int col(int j, int g) { return wave_col() + 32 * j + 8 * g + 4 * (lane() >> 5); }
};

// The work unit of this workgroup.  Workgroups go to the eight XCDs in turn, each with an L2 of
// its own; units are dealt out so that an XCD works on `run` consecutive units at a time (as
// many as it holds workgroups), which tile_place makes neighbours that share operands.
__device__ inline int64_t unit_of_workgroup(int run)
{
    const uint32_t n = gridDim.x, b = blockIdx.x, round = 8u * uint32_t(run);
    const uint32_t base = b / round * round, here = min(round, n - base);
    const uint32_t x = b % 8u, i = (b - base) / 8u;
    return int64_t(base + x * (here / 8u) + min(x, here % 8u) + i);
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

// The main loop over `steps` >= 1 steps.  P, Q: first rows of the tile's operands, pitches in
// bytes, of which limit_p and limit_q rows exist.
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
template <typename Mul, typename S>
__device__ inline void product(Mul& mul, S& c, const void* P, int64_t pitch_p, int64_t limit_p,
                               const void* Q, int64_t pitch_q, int64_t limit_q, int steps,
                               uint8_t* lds)
{
    constexpr int I = S::I, J = S::J;
    const int lane = S::lane(), wm = S::wave_row(), wn = S::wave_col();
    TileLoad<S::kRows, S::kThreads> load_p;
    TileLoad<S::kCols, S::kThreads> load_q;
    load_p.init(pitch_p, limit_p);
    load_q.init(pitch_q, limit_q);
    const auto* p = static_cast<const uint8_t*>(P);
    const auto* q = static_cast<const uint8_t*>(Q);
    constexpr int kLoads = load_p.N + load_q.N;
    struct Groups {
        // the blocks [first, first + n) of group g of `all`
        static constexpr int n(int all, int g) { return g == 0 ? (all + 1) / 2 : all / 2; }
        static constexpr int first(int all, int g) { return g == 0 ? 0 : (all + 1) / 2; }
        // copies of the early or late rows of an even (0) or odd (1) step
        static constexpr int loads(int odd, int late)
        {
            return S::kRows / 32 / I * n(I, late) + S::kCols / 32 / J * n(J, odd ^ late);
        }
    };
    Chunks a[I], b[J];
    // the k-th copy of step s's early or late rows
    const auto load = [&](int s, int odd, int late, int k) {
        uint8_t* to = lds + odd * S::kBufferBytes;
        const int64_t at = int64_t(s < steps ? s : steps - 1) * kStepBytes;
        const int np = Groups::n(I, late), nq = Groups::n(J, odd ^ late);
        const int all_p = S::kRows / 32 / I * np;
        if (k < all_p) {
            load_p.issue(k / np * I + Groups::first(I, late) + k % np, p + at, to);
        } else {
            const int l = k - all_p;
            load_q.issue(l / nq * J + Groups::first(J, odd ^ late) + l % nq, q + at,
                         to + S::kRows * kStepBytes);
        }
    };
    const auto read_a = [&](int odd, int g, int k) {
        const int i = Groups::first(I, g) + k / 4;
        a[i].c[k % 4] = read_chunk(lds + odd * S::kBufferBytes, wm + 32 * i, k % 4, lane);
    };
    const auto read_b = [&](int odd, int g, int k) {
        const int j = Groups::first(J, g) + k / 4;
        b[j].c[k % 4] = read_chunk(lds + odd * S::kBufferBytes + S::kRows * kStepBytes,
                                   wn + 32 * j, k % 4, lane);
    };
    // the products of groups ga and gb, with reads and copies issued evenly between them: reads
    // within the first three quarters, so that the last covers their latency.  Every border
    // keeps its place: left to itself the compiler issues reads right before the products that
    // wait for them, and products ahead of the barrier.
    const auto multiply = [&](int ga, int gb, int reads, auto read, int loads, auto copy) {
        const int ni = Groups::n(I, ga), nj = Groups::n(J, gb);
        const int muls = ni * nj * Mul::kInstructions, paced = muls * 3 / 4;
        const auto share = [](int n, int of, int k) { return k < of ? n * k / of : n; };
        if (muls == 0) {
#pragma unroll
            for (int r = 0; r < loads; ++r)
                copy(r);
#pragma unroll
            for (int r = 0; r < reads; ++r)
                read(r);
            return;
        }
#pragma unroll
        for (int k = 0; k < muls; ++k) {
#pragma unroll
            for (int r = share(loads, muls, k); r < share(loads, muls, k + 1); ++r)
                copy(r);
#pragma unroll
            for (int r = share(reads, paced, k); r < share(reads, paced, k + 1); ++r)
                read(r);
            const int t = k / (ni * nj), i = Groups::first(I, ga) + k / nj % ni,
                      j = Groups::first(J, gb) + k % nj;
            c.acc[i][j] = mul.mul(t, i, j, b[j], a[i], c.acc[i][j]);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    // step s, odd or even
    const auto step = [&](int s, auto parity) {
        constexpr int odd = decltype(parity)::value;
        constexpr int early = Groups::loads(odd, 0), late = Groups::loads(odd, 1);
        constexpr int b_first = odd, b_second = 1 - odd;
        mul.next(s);
        multiply(0, b_first, 4 * Groups::n(J, b_second), [&](int k) { read_b(odd, b_second, k); },
                 early / 2, [&](int k) { load(s + 2, odd, 0, k); });
        multiply(0, b_second, 4 * Groups::n(I, 1), [&](int k) { read_a(odd, 1, k); },
                 early - early / 2, [&](int k) { load(s + 2, odd, 0, early / 2 + k); });
        wait_reads();
        wait_loads<early + Groups::loads(1 - odd, 1)>();  // the next step's early rows are there
        __builtin_amdgcn_s_barrier();
        mul.read(s + 1);
        multiply(1, b_second, 4 * Groups::n(I, 0), [&](int k) { read_a(1 - odd, 0, k); },
                 late / 2, [&](int k) { load(s + 2, odd, 1, k); });
        multiply(1, b_first, 4 * Groups::n(J, b_second),
                 [&](int k) { read_b(1 - odd, b_second, k); }, late - late / 2,
                 [&](int k) { load(s + 2, odd, 1, late / 2 + k); });
        wait_reads();
        wait_loads<kLoads>();  // and its late rows
        __builtin_amdgcn_s_barrier();
    };
#pragma unroll
    for (int i = 0; i < I; ++i)
#pragma unroll
        for (int j = 0; j < J; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r)
                c.acc[i][j][r] = 0.0f;
    mul.begin();
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int k = 0; k < kLoads; ++k) {
            const int early = Groups::loads(s, 0);
            load(s, s, k >= early, k < early ? k : k - early);
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
    wait_loads<0>();
    __builtin_amdgcn_s_barrier();  // nothing is on its way into LDS any more
}

// What follows the main loop, for one wave's block, 32 rows at a time through LDS (the loop is
// done with it): a lane then has eight consecutive columns of a row, so that a wave reads and
// writes whole lines, and the code is a few short loops.  From the registers as they come a lane
// has four columns of 32 rows: accesses of 16 bytes a row, unrolled to 36 to 118 KB of code.
// Writer w:
//   w.fetch(row, col, p)     requests what results [row][col .. col + 8) need, into slot p;
//   w.store(row, col, v, p)  takes the sums v, leaves the results there and stores them;
//   w.turn(col, row, v)      with kTurned: stores results [row .. row + 8)[col] of the transpose;
// Rows and columns count from the tile's origin.
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
#pragma unroll
    for (int i = 0; i < S::I; ++i) {
#pragma unroll
        for (int p = 0; p < kPasses; ++p)
            w.fetch(r0 + 32 * i + p * kDown + down, c0 + across, p);
#pragma unroll
        for (int jg = 0; jg < 4 * S::J; ++jg) {
            const int j = jg / 4, g = jg % 4;
            *reinterpret_cast<f32x4*>(mine + (lane & 31) * kPitch + 32 * j + 8 * g +
                                      4 * (lane >> 5)) =
                f32x4{c.acc[i][j][4 * g], c.acc[i][j][4 * g + 1], c.acc[i][j][4 * g + 2],
                      c.acc[i][j][4 * g + 3]};
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

}  // namespace tiles

#endif
