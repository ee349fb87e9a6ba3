// orth.hip -- Newton-Schulz orthogonalisation of a list of matrices, and the Muon step.
//
// X_0 = U / ||U||_F; ns_steps times A = X X^T, B = b A + c A A, X = a X + B X, on the side of
// the smaller dimension (A = X^T X and X B where there are more rows than columns).
//
// Long matrices take their steps in pairs.  With n the smaller side and m the larger, A and
// every polynomial of it are n x n and commute, so the second step of a pair needs no new X:
// with P = a I + B, A' = P A P, and X'' = P' P X.  A pair takes 3 n^2 m + 5 n^3 multiply-adds
// where two single steps take 6 n^2 m + 2 n^3 (products of symmetric matrices compute half
// their tiles), and X is written once.  Rounding errors of a pair grow by a^2 in directions of
// small singular values: results are up to five times as far from the exact polynomial as those
// of single steps.  Measured in the 2-norm, single steps at sides of 65 to 500 and pairs at 128 to
// 512: noise 8e-4 and 5e-4, a spectrum over one decade 9e-4 and 1.6e-3, over three 2.8e-3 and
// 4.3e-3, over six 4.4e-3 and 5.7e-3, two directions 100 above the rest 9e-4 and 4.4e-3, half the
// rank 7e-3 and 7e-3, rank 1 1.3e-2 and 2.3e-2, most at the smallest side each, where the fewest
// roundings average (with bf16 operands 1e-2 to 0.12).  What is off lies in directions that U
// hardly has, which the polynomial makes 485 times larger in five steps.  Pairs are taken all the
// same, where they save a quarter of the time: the polynomial itself leaves singular values
// anywhere between 0.7 and 1.2, and an 8-bit momentum is further from its 32-bit form than that.
// Three steps and more are cheaper still but diverge at five.
//
// The singular values of X_0 lie in [0, 1], those of every later X in [0, 1.203]: the
// polynomial's largest value on [0, 1.203] is f(0.5545) = 1.2024.  So the eigenvalues of A lie
// in [0, 1.446], of B in [-2.81, 0], of P in [0.63, 3.45]; powers of two place every operand in
// fp16's range: X times 2^15, n x n matrices times 2^14, P' P times 2^12.
//
// Products take fp16 operands and sum in fp32: fp16 has three bits more than bf16 at the same
// rate.  Two things keep what is rounded small.  X enters the linear term as a sum of two fp16
// numbers: directions whose singular values are far below the largest grow by a factor of a in
// every step, and one fp16 number loses them against the large ones.  And every n x n matrix is
// kept without the part that is a multiple of I: S = A - d I with d the eigenvalue that A would
// have if all were equal (1/n at first, then d' = (a + b d + c d^2)^2 d), and so on for what
// is made of it.  What is left is small wherever singular values are alike, as they mostly are
// after a step or two; it halves the error for Gaussian matrices.
//
// X is kept three times: its leading half row-major (H) and transposed (T), and the rest
// row-major (L).  Every product then has its summed index contiguous in both operands.
// Sizes are padded with zeros to whole tiles, which every product keeps zero, so no load has
// a bound to check.

#include "host.h"
#include "tiles.h"

#include <algorithm>
#include <cmath>
#include <cstring>
#include <mutex>
#include <unordered_map>

namespace {

using host::fail;
using host::Guard;
using host::round_up;
using namespace tiles;

constexpr float kA = 3.4445f, kB = -4.7750f, kC = 2.0315f;
constexpr float kScaleX = 32768.0f;  // X is stored times 2^15
constexpr float kScaleS = 16384.0f;  // n x n matrices times 2^14
constexpr float kScaleR = 4096.0f;   // products of a pair's two P times 2^12
constexpr int kTile = 128;           // what sizes are padded to
constexpr int kThreads = 256;
static_assert(Tiny::kThreads == kThreads && Small::kThreads == kThreads &&
              Large::kThreads == kThreads && Small::kRows == 2 * Tiny::kRows &&
              Large::kRows == 4 * Tiny::kRows, "tiles of one kind by workgroups of one size");
constexpr int kPrep = 64;                         // tile of the transposing pass

struct Matrix {
    const void* src;           // the matrix, or the Muon step's update in fp32
    _Float16 *h[2], *t[2], *l[2];
    _Float16* sym[3];          // n x n matrices
    float* sums;               // G's sums by slices of the summed index
    double* gram;              // sides of 33 to 64: G of every slice of columns
    float* r;                  // and R, behind what X is multiplied by
    double *partial, *square;  // sums of squares of its units; their sum
    void* out;                 // orthogonalise: the result
    float* w;                  // Muon: weights and their bf16 copy (or null)
    uint16_t* wb;
    int32_t rows, cols, rp, cp;  // sizes, and padded sizes
    int32_t units;
    float rate;                // Muon: step size of this matrix
};

// What stops a launch: descriptors that are not its own, a status that skips, a step state
// that lets no step apply.
struct Gate {
    Guard guard;
    const int32_t* status;
    const lt_step_state* state;
};

__device__ inline bool descriptors_ok(const Gate& g) { return *g.guard.at == g.guard.tag; }

__device__ inline bool step_applies(const Gate& g)
{
    if (g.status && *g.status != LT_STATUS_OK)
        return false;
    if (g.state && (g.state->stopped != 0 || g.state->applied < 0 ||
                    g.state->applied >= g.state->table_len))
        return false;
    return true;
}

// The last k in [first, first + n) with prefix[k] <= u, u alike in all lanes of the wave.
__device__ inline int find_matrix(const int64_t* __restrict__ prefix, int first, int n, int64_t u)
{
    const int lane = int(threadIdx.x) & 63;
    int lo = first;
    while (n > 1) {
        const int stride = (n + 63) >> 6;
        const int i = lane * stride;
        const bool below = i < n && prefix[lo + i] <= u;
        const int j = 63 - __builtin_clzll(__builtin_amdgcn_ballot_w64(below) | 1u);
        lo += j * stride;
        n = min(stride, n - j * stride);
    }
    return __builtin_amdgcn_readfirstlane(lo);
}

__device__ inline float load_value(const float* p) { return *p; }
__device__ inline float load_value(const uint16_t* p) { return __uint_as_float(uint32_t(*p) << 16); }

// The values in the 16 bytes at p.
__device__ inline void load_line(const float* p, float (&x)[4])
{
    const f32x4 w = __builtin_bit_cast(f32x4, load_any(p));
#pragma unroll
    for (int i = 0; i < 4; ++i)
        x[i] = w[i];
}
__device__ inline void load_line(const uint16_t* p, float (&x)[8])
{
    const i32x4 w = load_any(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = __uint_as_float(uint32_t(w[i]) << 16);
        x[2 * i + 1] = __uint_as_float(uint32_t(w[i]) & 0xFFFF0000u);
    }
}

__device__ inline uint16_t bf16_bits(float x)
{
    return __builtin_bit_cast(uint16_t, (__bf16)x);  // to nearest even; a NaN becomes quiet
}

// Sum of a workgroup's values in a fixed order; the result is in thread 0.
__device__ inline double sum_workgroup(double x, double* red)
{
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1)
        x += __shfl_xor(x, o, 64);
    if ((threadIdx.x & 63) == 0)
        red[threadIdx.x >> 6] = x;
    __syncthreads();
    return (red[0] + red[1]) + (red[2] + red[3]);
}

// ------------------------------------------------------------- the norm

// The sum of squares in 64 bits, bound by reading: fp32 17408 x 5120 70 to 78 us, 4.6 to 5.1 TB/s.
// A sum for every unit of 16384 elements, added up in a fixed order by k_orth_norm.
constexpr int64_t kSquareUnit = 16384;  // elements of one workgroup

template <typename T>
__global__ __launch_bounds__(kThreads) void k_orth_squares(Gate gate,
                                                           const int64_t* __restrict__ prefix,
                                                           const Matrix* __restrict__ mats,
                                                           int first, int n)
{
    __shared__ double red[kThreads / 64];
    if (!descriptors_ok(gate))
        return;
    const int64_t unit = prefix[first] + blockIdx.x;
    const int k = find_matrix(prefix, first, n, unit);
    const Matrix& m = mats[k];
    const int64_t numel = int64_t(m.rows) * m.cols;
    const int64_t e0 = (unit - prefix[k]) * kSquareUnit;
    const int64_t e1 = e0 + kSquareUnit < numel ? e0 + kSquareUnit : numel;
    const T* src = static_cast<const T*>(m.src);
    double sq = 0.0;
    constexpr int kLine = 16 / sizeof(T);  // values of a 16-byte load; units start aligned
    int64_t e = e0 + int64_t(threadIdx.x) * kLine;
#pragma unroll 8
    for (; e + kLine <= e1; e += kThreads * kLine) {
        float x[kLine];
        load_line(src + e, x);
#pragma unroll
        for (int i = 0; i < kLine; ++i)
            sq += double(x[i]) * double(x[i]);
    }
    for (; e < e1; ++e) {  // the lane that the matrix ends in
        const double x = load_value(src + e);
        sq += x * x;
    }
    sq = sum_workgroup(sq, red);
    if (threadIdx.x == 0)
        m.partial[unit - prefix[k]] = sq;
}

__global__ __launch_bounds__(kThreads) void k_orth_norm(Gate gate, const Matrix* __restrict__ mats,
                                                        int first)
{
    __shared__ double red[kThreads / 64];
    if (!descriptors_ok(gate) || !step_applies(gate))
        return;
    const Matrix& m = mats[first + blockIdx.x];
    if (m.units == 0)
        return;  // an empty matrix: it has no place for its sum
    double sq = 0.0;
    for (int i = threadIdx.x; i < m.units; i += kThreads)
        sq += m.partial[i];
    sq = sum_workgroup(sq, red);
    if (threadIdx.x == 0)
        *m.square = sq;
}

// ------------------------------------------------- X_0 in its three layouts

// One 64 x 64 tile by a workgroup, transposed through LDS, so that all four matrices are read and
// written in whole lines.  Bound by HBM: fp32 17408 x 5120 160 us, 5.6 TB/s read and written.
template <typename T>
__global__ __launch_bounds__(kThreads) void k_orth_prepare(Gate gate,
                                                           const int64_t* __restrict__ prefix,
                                                           const Matrix* __restrict__ mats,
                                                           int first, int n)
{
    __shared__ __align__(16) _Float16 turned[kPrep][kPrep + 8];
    if (!descriptors_ok(gate) || !step_applies(gate))
        return;
    const int64_t unit = prefix[first] + blockIdx.x;
    const int k = find_matrix(prefix, first, n, unit);
    const Matrix& m = mats[k];
    const int across = m.cp / kPrep, tile = int(unit - prefix[k]);
    const int r0 = tile / across * kPrep, c0 = tile % across * kPrep;
    // a zero matrix stays zero; an infinite or NaN sum makes every value NaN
    const double sq = *m.square;
    const double scale = sq == 0.0 ? 0.0 : double(kScaleX) / sqrt(sq);
    const double by = isfinite(sq) ? scale : __builtin_nan("");
    const T* src = static_cast<const T*>(m.src);
    // a lane has eight values of a row, a wave eight rows
    constexpr int kLine = 16 / sizeof(T);
    const int t = int(threadIdx.x), c = t % 8 * 8;
    for (int r = t / 8; r < kPrep; r += kThreads / 8) {
        const int row = r0 + r, col = c0 + c;
        const T* p = src + int64_t(row) * m.cols + col;
        float x[8];
        if (row < m.rows && col + 8 <= m.cols) {
#pragma unroll
            for (int e = 0; e < 8; e += kLine) {
                float w[kLine];
                load_line(p + e, w);
#pragma unroll
                for (int i = 0; i < kLine; ++i)
                    x[e + i] = w[i];
            }
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                x[e] = row < m.rows && col + e < m.cols ? load_value(p + e) : 0.0f;
        }
        half8 hi, lo;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float v = float(double(x[e]) * by);
            hi[e] = _Float16(v);
            lo[e] = _Float16(v - float(hi[e]));
            turned[c + e][r] = hi[e];
        }
        const int64_t at = int64_t(row) * m.cp + col;
        *reinterpret_cast<half8*>(m.h[0] + at) = hi;
        *reinterpret_cast<half8*>(m.l[0] + at) = lo;
    }
    __syncthreads();
    for (int q = t / 8; q < kPrep; q += kThreads / 8)
        *reinterpret_cast<half8*>(m.t[0] + int64_t(c0 + q) * m.rp + r0 + c) =
            *reinterpret_cast<const half8*>(&turned[q][c]);
}

// ------------------------------------------------------------- products


// The multiples of I at step `step`: of A, of P = a I + B and of P A.
struct Shift {
    float d, p;
};

__device__ inline Shift shift_at(const Matrix& m, int step)
{
    Shift s;
    s.d = 1.0f / float(m.rows < m.cols ? m.rows : m.cols);
    for (int i = 0;; ++i) {
        s.p = kA + s.d * (kB + kC * s.d);
        if (i == step)
            return s;
        s.d = s.p * s.p * s.d;
    }
}

// Products of n x n matrices, all symmetric: tiles on and above the diagonal, each stored on
// both sides of it.  With S = A - d I, P^ = P - p I, W^ = P A - p d I, R^ = P' P - p' p I:
// 17408 x 5120: G 400 us (half of 2 n^2 m: 1.14 PFLOP/s on 210 of 256 CUs), each of the others
// 131 to 136 us (1.05).  What bounds them is the matrix cores' power: 1.28 PFLOP/s is what a large
// product of random fp16 numbers reaches at all, zeros 1.8.
enum Sym {
    kGram,    // S = X X^T - d I (or X^T X)
    kStep,    // P^ = c S S + (b + 2 c d) S
    kHalf,    // W^ = P^ S + p S + d P^
    kNext,    // S' = P^ W^ + p W^ + p d P^
    kPair,    // R^ = P'^ P^ + p' P^ + p P'^
};

struct SymArgs {
    int step;      // the number of Newton-Schulz steps before this one
    int from;      // which X
    int m, n, out; // operands and result among sym[]
};

// out = by * sum + at_m * M + at_n * N, in the scales of what is stored.
template <int OP>
struct SymWriter {
    static constexpr bool kTurned = true;
    static constexpr int kSlots = 8;
    float by, at_m, at_n, diagonal;
    int64_t pitch;
    const _Float16 *m, *n;  // at the tile's origin, like the result and its transpose
    _Float16 *to, *turned;
    int below, real;        // of the diagonal: the tile's column minus its row, rows that exist
    bool mirror;
    half8 x[OP == kGram ? 1 : kSlots], y[OP == kGram || OP == kStep ? 1 : kSlots];

    __device__ inline void fetch(int row, int col, int p)
    {
        if constexpr (OP != kGram)
            x[p] = *reinterpret_cast<const half8*>(m + row * pitch + col);
        if constexpr (OP != kGram && OP != kStep)
            y[p] = *reinterpret_cast<const half8*>(n + row * pitch + col);
    }
    __device__ inline void store(int row, int col, float (&v)[8], int p)
    {
        half8 h;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            v[e] *= by;
            if constexpr (OP == kGram)
                v[e] -= row == col + e + below && row < real ? diagonal : 0.0f;
            else
                v[e] += at_m * float(x[p][e]);
            if constexpr (OP != kGram && OP != kStep)
                v[e] += at_n * float(y[p][e]);
            h[e] = _Float16(v[e]);
        }
        *reinterpret_cast<half8*>(to + row * pitch + col) = h;
    }
    __device__ inline void turn(int col, int row, const float (&v)[8]) const
    {
        if (!mirror)
            return;
        half8 h;
#pragma unroll
        for (int e = 0; e < 8; ++e)
            h[e] = _Float16(v[e]);
        *reinterpret_cast<half8*>(turned + col * pitch + row) = h;
    }
};

template <typename Tile, int OP>
__global__ __launch_bounds__(Tile::kThreads, Tile::kWavesPerSimd) void k_orth_sym(Gate gate,
                                                             const int64_t* __restrict__ prefix,
                                                             const Matrix* __restrict__ mats,
                                                             int first, int n, SymArgs args)
{
    __shared__ __align__(1024) uint8_t lds[Tile::kLdsBytes];
    if (!descriptors_ok(gate) || !step_applies(gate))
        return;
    const int64_t unit = prefix[first] + unit_of_workgroup(Tile::kRun);
    const int k = find_matrix(prefix, first, n, unit);
    const Matrix& m = mats[k];
    const bool wide = m.rows <= m.cols;
    const int side = wide ? m.rp : m.cp, real = wide ? m.rows : m.cols;
    const int inner = OP == kGram ? (wide ? m.cp : m.rp) : side;
    const TilePlace at_tile =
        triangle_place(int(unit - prefix[k]), (side + Tile::kRows - 1) / Tile::kRows);
    const int r0 = at_tile.row * Tile::kRows, c0 = at_tile.col * Tile::kCols;
    const _Float16* M = OP == kGram ? (wide ? m.h[args.from] : m.t[args.from]) : m.sym[args.m];
    const _Float16* N = OP == kGram ? M : m.sym[args.n];
    Tile tile;
    Half mul;
    product(mul, tile, M + int64_t(r0) * inner, int64_t(inner) * 2, side - r0,
                 N + int64_t(c0) * inner, int64_t(inner) * 2, side - c0, inner / 64, lds);

    const Shift s = shift_at(m, args.step);
    SymWriter<OP> out = {};
    out.by = 1.0f / kScaleS;
    if constexpr (OP == kGram) {
        out.by = kScaleS / (kScaleX * kScaleX);
    } else if constexpr (OP == kStep) {
        out.by = kC / kScaleS;
        out.at_m = kB + 2.0f * kC * s.d;
    } else if constexpr (OP == kHalf) {
        out.at_m = s.d;
        out.at_n = s.p;
    } else if constexpr (OP == kNext) {
        out.at_m = s.p * s.d;
        out.at_n = s.p;
    } else {
        out.by = kScaleR / (kScaleS * kScaleS);
        const Shift before = shift_at(m, args.step - 1);
        out.at_m = before.p * (kScaleR / kScaleS);
        out.at_n = s.p * (kScaleR / kScaleS);
    }
    if (r0 + Tile::wave_row() >= side || c0 + Tile::wave_col() >= side)
        return;  // sizes are multiples of 128: a wave's block lies inside or outside
    out.pitch = side;
    out.m = M + int64_t(r0) * side + c0;
    out.n = N + int64_t(r0) * side + c0;
    out.to = m.sym[args.out] + int64_t(r0) * side + c0;
    out.turned = m.sym[args.out] + int64_t(c0) * side + r0;
    out.diagonal = s.d * kScaleS;
    out.below = c0 - r0;
    out.real = real - r0;
    out.mirror = r0 != c0;
    finish(tile, lds, out);
}

// G of a few long matrices has few tiles of long sums: the sums are cut into slices of a whole
// number of pairs of steps, and added up in order by the pass that stores G.
__device__ inline int slice_steps(int inner, int slices)
{
    return (inner / 64 + 2 * slices - 1) / (2 * slices) * 2;
}

struct SumWriter {
    static constexpr bool kTurned = false;
    static constexpr int kSlots = 8;
    float* to;  // at the tile's origin
    int64_t pitch;
    __device__ inline void fetch(int, int, int) {}
    __device__ inline void turn(int, int, const float (&)[8]) {}
    __device__ inline void store(int row, int col, float (&v)[8], int)
    {
        float* p = to + row * pitch + col;
        *reinterpret_cast<f32x4*>(p) = f32x4{v[0], v[1], v[2], v[3]};
        *reinterpret_cast<f32x4*>(p + 4) = f32x4{v[4], v[5], v[6], v[7]};
    }
};

template <typename Tile>
__global__ __launch_bounds__(Tile::kThreads, Tile::kWavesPerSimd) void k_orth_gram(Gate gate,
                                                             const int64_t* __restrict__ prefix,
                                                             const Matrix* __restrict__ mats,
                                                             int first, int n, int from)
{
    __shared__ __align__(1024) uint8_t lds[Tile::kLdsBytes];
    if (!descriptors_ok(gate) || !step_applies(gate))
        return;
    const int64_t unit = prefix[first] + unit_of_workgroup(Tile::kRun);
    const int k = find_matrix(prefix, first, n, unit);
    const Matrix& m = mats[k];
    const bool wide = m.rows <= m.cols;
    const int side = wide ? m.rp : m.cp, inner = wide ? m.cp : m.rp;
    const int per = slice_steps(inner, int(gridDim.y)), begin = int(blockIdx.y) * per;
    const int steps = min(per, inner / 64 - begin);
    if (steps <= 0)
        return;
    const TilePlace at_tile =
        triangle_place(int(unit - prefix[k]), (side + Tile::kRows - 1) / Tile::kRows);
    const int r0 = at_tile.row * Tile::kRows, c0 = at_tile.col * Tile::kCols;
    const _Float16* X = (wide ? m.h[from] : m.t[from]) + int64_t(begin) * 64;
    Tile tile;
    Half mul;
    product(mul, tile, X + int64_t(r0) * inner, int64_t(inner) * 2, side - r0,
            X + int64_t(c0) * inner, int64_t(inner) * 2, side - c0, steps, lds);
    if (r0 + Tile::wave_row() >= side || c0 + Tile::wave_col() >= side)
        return;  // sizes are multiples of 128: a wave's block lies inside or outside
    SumWriter out;
    out.pitch = side;
    out.to = m.sums + (int64_t(blockIdx.y) * side + r0) * side + c0;
    finish(tile, lds, out);
}

// G = the slices' sums: a block of 64 x 64 on or above the diagonal and its mirror image by a
// workgroup.
__global__ __launch_bounds__(kThreads) void k_orth_gram_join(Gate gate,
                                                             const int64_t* __restrict__ prefix,
                                                             const Matrix* __restrict__ mats,
                                                             int first, int n, int slices,
                                                             SymArgs args)
{
    __shared__ __align__(16) _Float16 turned[64][64 + 8];
    if (!descriptors_ok(gate) || !step_applies(gate))
        return;
    const int64_t unit = prefix[first] + blockIdx.x;
    const int k = find_matrix(prefix, first, n, unit);
    const Matrix& m = mats[k];
    const bool wide = m.rows <= m.cols;
    const int side = wide ? m.rp : m.cp, inner = wide ? m.cp : m.rp;
    const int real = wide ? m.rows : m.cols;
    const int per = slice_steps(inner, slices), used = (inner / 64 + per - 1) / per;
    const TilePlace at = triangle_place(int(unit - prefix[k]), side / 64);
    const int r0 = at.row * 64, c0 = at.col * 64;
    const int row = int(threadIdx.x) / 4, col = int(threadIdx.x) % 4 * 16;
    const float* from = m.sums + int64_t(r0 + row) * side + c0 + col;
    f32x4 v[4] = {};
    for (int i = 0; i < used; ++i, from += int64_t(side) * side)
#pragma unroll
        for (int c = 0; c < 4; ++c)
            v[c] += *reinterpret_cast<const f32x4*>(from + 4 * c);
    const float by = kScaleS / (kScaleX * kScaleX);
    const float diagonal = shift_at(m, args.step).d * kScaleS;
    half8 h[2];
#pragma unroll
    for (int e = 0; e < 16; ++e) {
        const int r = r0 + row;
        const float x = v[e / 4][e % 4] * by - (r == c0 + col + e && r < real ? diagonal : 0.0f);
        h[e / 8][e % 8] = _Float16(x);
        turned[col + e][row] = _Float16(x);
    }
    _Float16* to = m.sym[args.out];
    half8* p = reinterpret_cast<half8*>(to + int64_t(r0 + row) * side + c0 + col);
    p[0] = h[0];
    p[1] = h[1];
    if (r0 == c0)
        return;
    __syncthreads();
    half8* q = reinterpret_cast<half8*>(to + int64_t(c0 + row) * side + r0 + col);
    const half8* w = reinterpret_cast<const half8*>(&turned[row][col]);
    q[0] = w[0];
    q[1] = w[1];
}

enum Final { kAgain, kOutF32, kOutBf16, kWeights };

struct UpdateArgs {
    int step, steps;  // steps before, and steps applied now: 1 (P) or 2 (P' P)
    int from, sym;    // which X, and where P^ or R^ is
    float decay;
};

typedef uint16_t u16x8 __attribute__((ext_vector_type(8)));

// The rest of k_orth_update: X' = by * sum + linear * X and where it goes.
template <int FINAL>
struct UpdateWriter {
    static constexpr bool kTurned = FINAL == kAgain;
    static constexpr int kSlots = 8;
    float by, linear, rate, decay;
    bool applies;
    const _Float16 *h, *l;    // X at the tile's origin, and X'
    _Float16 *next_h, *next_l, *next_t;
    int64_t pitch, pitch_t;
    int rows, cols, width;    // results that exist from the tile's origin on; the caller's pitch
    float* out;               // the result in fp32 or the weights, at the tile's origin
    uint16_t* out16;          // in bf16, or null
    half8 x[kSlots], y[kSlots];
    float w[FINAL == kWeights ? kSlots : 1][8];

    __device__ inline void fetch(int row, int col, int p)
    {
        if (applies) {
            x[p] = *reinterpret_cast<const half8*>(h + row * pitch + col);
            y[p] = *reinterpret_cast<const half8*>(l + row * pitch + col);
        }
        if constexpr (FINAL == kWeights) {
            if (row < rows && col < cols) {
                const float* from = out + int64_t(row) * width + col;
                if (col + 8 <= cols) {
                    const f32x4 a = __builtin_bit_cast(f32x4, load_any(from));
                    const f32x4 b = __builtin_bit_cast(f32x4, load_any(from + 4));
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        w[p][e] = a[e], w[p][4 + e] = b[e];
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        w[p][e] = col + e < cols ? from[e] : 0.0f;
                }
            }
        }
    }
    __device__ inline void store(int row, int col, float (&v)[8], int p)
    {
        if (applies) {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                v[e] = by * v[e] + linear * (float(x[p][e]) + float(y[p][e]));
        }
        if constexpr (FINAL == kAgain) {
            half8 hi, lo;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                hi[e] = _Float16(v[e]);
                lo[e] = _Float16(v[e] - float(hi[e]));
            }
            *reinterpret_cast<half8*>(next_h + row * pitch + col) = hi;
            *reinterpret_cast<half8*>(next_l + row * pitch + col) = lo;
            return;
        }
        if (row >= rows || col >= cols)
            return;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            v[e] *= 1.0f / kScaleX;
            if constexpr (FINAL == kWeights)
                v[e] = applies ? __builtin_fmaf(-rate, v[e], w[p][e] * decay) : w[p][e];
        }
        const int64_t to = int64_t(row) * width + col;
        const bool whole = col + 8 <= cols;
        if (FINAL == kOutF32 || (FINAL == kWeights && applies)) {
            if (whole) {
                store_any(out + to, f32x4{v[0], v[1], v[2], v[3]});
                store_any(out + to + 4, f32x4{v[4], v[5], v[6], v[7]});
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (col + e < cols)
                        out[to + e] = v[e];
            }
        }
        if (FINAL == kOutBf16 || (FINAL == kWeights && out16)) {
            u16x8 b;
#pragma unroll
            for (int e = 0; e < 8; ++e)
                b[e] = bf16_bits(v[e]);
            if (whole) {
                store_any(out16 + to, b);
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (col + e < cols)
                        out16[to + e] = b[e];
            }
        }
    }
    __device__ inline void turn(int col, int row, const float (&v)[8]) const
    {
        half8 hi;
#pragma unroll
        for (int e = 0; e < 8; ++e)
            hi[e] = _Float16(v[e]);
        *reinterpret_cast<half8*>(next_t + col * pitch_t + row) = hi;
    }
};

// X' = p X + P^ X (or p X + X P^), P standing for P' P after a pair: the next X, or where it
// goes.  17408 x 5120 900 us (1.0 PFLOP/s) where the next X is written, 820 us to bf16: some 720
// are the product, the rest reading X and writing its three layouts.
template <typename Tile, int FINAL>
__global__ __launch_bounds__(Tile::kThreads, Tile::kWavesPerSimd) void k_orth_update(Gate gate,
                                                                const int64_t* __restrict__ prefix,
                                                                const Matrix* __restrict__ mats,
                                                                int first, int n, UpdateArgs args)
{
    __shared__ __align__(1024) uint8_t lds[Tile::kLdsBytes];
    if (!descriptors_ok(gate))
        return;
    const bool applies = step_applies(gate);
    if (!applies && FINAL != kWeights)
        return;
    const int64_t unit = prefix[first] + unit_of_workgroup(Tile::kRun);
    const int k = find_matrix(prefix, first, n, unit);
    const Matrix& m = mats[k];
    const bool wide = m.rows <= m.cols;
    const TilePlace at_tile =
        tile_place(int(unit - prefix[k]), (m.rp + Tile::kRows - 1) / Tile::kRows,
                   (m.cp + Tile::kCols - 1) / Tile::kCols);
    const int r0 = at_tile.row * Tile::kRows, c0 = at_tile.col * Tile::kCols;
    const int from = args.from;
    Tile tile;
    float by = 0.0f, linear = 0.0f;
    if (applies) {
        const int inner = wide ? m.rp : m.cp;
        const _Float16* P = (wide ? m.sym[args.sym] : m.h[from]) + int64_t(r0) * inner;
        const _Float16* Q = (wide ? m.t[from] : m.sym[args.sym]) + int64_t(c0) * inner;
        Half mul;
        product(mul, tile, P, int64_t(inner) * 2, m.rp - r0, Q, int64_t(inner) * 2, m.cp - c0,
                     inner / 64, lds);
        by = 1.0f / (args.steps == 2 ? kScaleR : kScaleS);
        linear = shift_at(m, args.step).p;
        if (args.steps == 2)
            linear *= shift_at(m, args.step + 1).p;
    } else if (!m.wb) {
        return;
    }
    if (r0 + Tile::wave_row() >= m.rp || c0 + Tile::wave_col() >= m.cp)
        return;  // sizes are multiples of 128: a wave's block lies inside or outside
    UpdateWriter<FINAL> out = {};
    out.by = by;
    out.linear = linear;
    out.rate = m.rate;
    out.decay = args.decay;
    out.applies = applies;
    const int64_t at = int64_t(r0) * m.cp + c0, to = int64_t(r0) * m.cols + c0;
    out.h = m.h[from] + at;
    out.l = m.l[from] + at;
    out.next_h = m.h[from ^ 1] + at;
    out.next_l = m.l[from ^ 1] + at;
    out.next_t = m.t[from ^ 1] + int64_t(c0) * m.rp + r0;
    out.pitch = m.cp;
    out.pitch_t = m.rp;
    out.rows = m.rows - r0;
    out.cols = m.cols - c0;
    out.width = m.cols;
    if constexpr (FINAL == kWeights) {
        out.out = m.w + to;
        out.out16 = m.wb ? m.wb + to : nullptr;
    } else if constexpr (FINAL == kOutF32) {
        out.out = static_cast<float*>(m.out) + to;
    } else if constexpr (FINAL == kOutBf16) {
        out.out16 = static_cast<uint16_t*>(m.out) + to;
    }
    finish(tile, lds, out);
}

// ---------------------------------------------------------------- thin matrices
//
// A matrix with n <= 32 rows (or columns), padded to 16 or 32, in one launch: with G = X X^T,
// every step stays n x n (P = a I + b G + c G G, G' = P G P, R' = P R), and the result is R X.
// Adapters, small layers and odd leftovers come in hundreds, and the general path would pad
// each to 128, write X three times a step and take 18 launches: 224 of 32 x 4288 take 141 us
// here, there 2124; one of 32 x 4096 59 and 210, one of 16 x 65536 280 and 1774.  An error of G
// grows by a^2 with every step in directions of small singular values, 2e5 in five: G and the
// steps are in 64 bits (in 32 a 64 x 64 matrix with a few strong directions ends 5e-3 off), R X
// in 32.  The norm is G's trace, so X is read once, into LDS, where it fits, and else twice.
// Where matrices are few, what bounds it is latency (7 us for 16 x 128, 0.5 us more a step; 2.1 at
// 32 x 32) beside G at the 64-bit rate (n^2 m products for every workgroup of a matrix, 3.4 us for
// 16 x 2048); where they are many, that a CU holds one workgroup, which loads, waits and multiplies
// in turn: 224 of 32 x 4288 take 138 us, their bytes 41, their 64-bit products 21.

constexpr int kThinThreads = 512, kThinWaves = kThinThreads / 64;
constexpr int kThinSpan = 16 * kThinWaves;  // columns that a workgroup's waves multiply at a time
constexpr int kThinSide = 32;

typedef double f64x4 __attribute__((ext_vector_type(4)));

template <int NP>
struct Thin {
    static constexpr int kBlocks = NP / 16, kUpper = kBlocks * (kBlocks + 1) / 2;
    static constexpr int kWidth = NP == 16 ? 2048 : 512;  // columns of X at a time
    static constexpr int kPitch = kWidth + 4;
    typedef double Sym[NP][NP + 2];
    float x[NP][kPitch];
    double part[kThinWaves][kUpper][4][64];  // every wave's sums of G, as they lie in its registers
    Sym sym[NP == 16 ? 1 : 4];
    float r[NP][NP + 4];                     // R, and what x is multiplied by
    float power[2];
};

// The 64-bit instruction takes M[lane % 16][k + lane / 16] and N[k + lane / 16][lane % 16] and
// leaves row 4 t + lane / 16, column lane % 16 in a lane's t-th result: what it leaves of a
// symmetric matrix is what it takes of it, so 16 x 16 chains never leave the registers.
__device__ inline f64x4 thin_product16(const f64x4& M, const f64x4& N)
{
    f64x4 acc = {0.0, 0.0, 0.0, 0.0};
#pragma unroll
    for (int t = 0; t < 4; ++t)
        acc = __builtin_amdgcn_mfma_f64_16x16x4f64(M[t], N[t], acc, 0, 0, 0);
    return acc;
}

__device__ inline f64x4 thin_chain16(f64x4 G, int steps)
{
    const int lane = int(threadIdx.x) & 63, r = lane & 15, q = lane >> 4;
    f64x4 R = {};
    for (int step = 0; step < steps; ++step) {
        f64x4 P = thin_product16(G, G);
#pragma unroll
        for (int t = 0; t < 4; ++t)
            P[t] = 2.0315 * P[t] - 4.7750 * G[t] + (4 * t + q == r ? 3.4445 : 0.0);
        R = step == 0 ? P : thin_product16(P, R);
        if (step + 1 < steps)
            G = thin_product16(thin_product16(P, G), P);
    }
    return R;
}

// dst = alpha * M N + beta * N + gamma * I, all symmetric, for 32 x 32: four waves take a block
// of 16 each.
__device__ inline void thin_product32(Thin<32>::Sym& dst, const Thin<32>::Sym& M,
                                      const Thin<32>::Sym& N, double alpha, double beta,
                                      double gamma)
{
    const int lane = int(threadIdx.x) & 63, wave = int(threadIdx.x) >> 6;
    const int r = lane & 15, q = lane >> 4;
    if (wave < 4) {
        const int bi = wave / 2 * 16, bj = wave % 2 * 16;
        f64x4 acc = {0.0, 0.0, 0.0, 0.0};
#pragma unroll
        for (int k = 0; k < 32; k += 4)
            acc = __builtin_amdgcn_mfma_f64_16x16x4f64(M[bi + r][k + q], N[bj + r][k + q], acc, 0,
                                                       0, 0);
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            const int i = bi + 4 * t + q, j = bj + r;
            dst[i][j] = alpha * acc[t] + beta * N[i][j] + (i == j ? gamma : 0.0);
        }
    }
    __syncthreads();
}

// Columns [k0, k0 + kWidth) of X, zeros from column `end` on, into LDS, 32 reads of a lane under way
// at a time.  Rows of X lie along its memory where it is wide, columns where it is tall.
template <int NP, typename T>
__device__ inline void thin_load(Thin<NP>& t, const Matrix& m, bool wide, int k0,
                                 int end)
{
    constexpr int W = Thin<NP>::kWidth, kAhead = 32, kAll = NP * W / kThinThreads;
    constexpr int kPasses = W > kThinThreads ? W / kThinThreads : 1;  // of a row, where wide
    static_assert(W % kThinThreads == 0 && kAll % kAhead == 0, "whole passes");
    const int n = wide ? m.rows : m.cols, len = wide ? m.cols : m.rows;
    const int tid = int(threadIdx.x);
    const T* src = static_cast<const T*>(m.src);
#pragma unroll
    for (int first = 0; first < kAll; first += kAhead) {
        float v[kAhead];
        if (wide) {
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                const int i = (first + u) / kPasses, k = (first + u) % kPasses * kThinThreads + tid;
                v[u] = i < n && k0 + k < end ? load_value(src + i * len + k0 + k) : 0.0f;
            }
#pragma unroll
            for (int u = 0; u < kAhead; ++u)
                t.x[(first + u) / kPasses][(first + u) % kPasses * kThinThreads + tid] = v[u];
        } else {
            const int i = tid % NP;
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                const int k = tid / NP + kThinThreads / NP * (first + u);
                v[u] = i < n && k0 + k < end ? load_value(src + (k0 + k) * n + i) : 0.0f;
            }
#pragma unroll
            for (int u = 0; u < kAhead; ++u)
                t.x[i][tid / NP + kThinThreads / NP * (first + u)] = v[u];
        }
    }
    __syncthreads();
}

// Element `to` of the result, or of the weights.
template <int FINAL>
__device__ inline void thin_store(const Matrix& m, int to, float o, float decay)
{
    if constexpr (FINAL == kOutF32) {
        static_cast<float*>(m.out)[to] = o;
    } else if constexpr (FINAL == kOutBf16) {
        static_cast<uint16_t*>(m.out)[to] = bf16_bits(o);
    } else {
        const float v = __builtin_fmaf(-m.rate, o, m.w[to] * decay);
        m.w[to] = v;
        if (m.wb)
            m.wb[to] = bf16_bits(v);
    }
}

// The same for elements to .. to + 3.
template <int FINAL>
__device__ inline void thin_store4(const Matrix& m, int to, f32x4 o, float decay)
{
    typedef uint16_t u16x4_any __attribute__((ext_vector_type(4), aligned(2)));
    const auto narrow = [](const f32x4& v) {
        return u16x4_any{bf16_bits(v[0]), bf16_bits(v[1]), bf16_bits(v[2]), bf16_bits(v[3])};
    };
    if constexpr (FINAL == kOutF32) {
        store_any(static_cast<float*>(m.out) + to, o);
    } else if constexpr (FINAL == kOutBf16) {
        *reinterpret_cast<u16x4_any*>(static_cast<uint16_t*>(m.out) + to) = narrow(o);
    } else {
        const f32x4 w = __builtin_bit_cast(f32x4, load_any(m.w + to));
#pragma unroll
        for (int e = 0; e < 4; ++e)
            o[e] = __builtin_fmaf(-m.rate, o[e], w[e] * decay);
        store_any(m.w + to, o);
        if (m.wb)
            *reinterpret_cast<u16x4_any*>(m.wb + to) = narrow(o);
    }
}

// Rows i .. i + 3 of column `col` of the n x len result, as far as they exist.
template <int FINAL>
__device__ inline void thin_result(const Matrix& m, bool wide, int n, int len, int i, int col,
                                   const f32x4& o, float decay)
{
    if (!wide && i + 4 <= n) {  // four neighbours in memory
        thin_store4<FINAL>(m, col * n + i, o, decay);
        return;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (i + e < n)
            thin_store<FINAL>(m, wide ? (i + e) * len + col : col * n + i + e, o[e], decay);
}

// 1 / norm as a factor in [1/2, 1) for R and a power of two for X, in two halves; a zero matrix
// stays zero; an infinite or NaN sum makes every value NaN.
__device__ inline double thin_factor(double trace, float* p0, float* p1)
{
    int e = 0;
    const double f = trace == 0.0 ? 0.0
                     : isfinite(trace) ? frexp(1.0 / sqrt(trace), &e)
                                       : __builtin_nan("");
    *p0 = ldexpf(1.0f, e / 2);
    *p1 = ldexpf(1.0f, e - e / 2);
    return f;
}

// Columns [begin, end) of the result, by one workgroup.
template <int NP, typename T, int FINAL>
__device__ inline void thin_matrix(Thin<NP>& t, const Matrix& m, int steps, float decay, int begin,
                                   int end)
{
    constexpr int W = Thin<NP>::kWidth, kBlocks = Thin<NP>::kBlocks;
    const bool wide = m.rows <= m.cols;
    const int n = wide ? m.rows : m.cols, len = wide ? m.cols : m.rows;
    const int lane = int(threadIdx.x) & 63, wave = int(threadIdx.x) >> 6;
    const int r = lane & 15, q = lane >> 4;

    // G of X as it is, each wave over its columns of every piece
    f64x4 g[Thin<NP>::kUpper] = {};
    for (int k0 = 0; k0 < len; k0 += W) {
        if (k0 > 0)
            __syncthreads();
        thin_load<NP, T>(t, m, wide, k0, len);
        for (int k = 16 * wave; k < W && k0 + k < len; k += 16 * kThinWaves) {
            f32x4 x[kBlocks];
#pragma unroll
            for (int b = 0; b < kBlocks; ++b)
                x[b] = *reinterpret_cast<const f32x4*>(&t.x[16 * b + r][k + 4 * q]);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                int u = 0;
#pragma unroll
                for (int a = 0; a < kBlocks; ++a)
#pragma unroll
                    for (int b = a; b < kBlocks; ++b, ++u)
                        g[u] = __builtin_amdgcn_mfma_f64_16x16x4f64(
                            double(x[a][e]), double(x[b][e]), g[u], 0, 0, 0);
            }
        }
    }
#pragma unroll
    for (int u = 0; u < Thin<NP>::kUpper; ++u)
#pragma unroll
        for (int e = 0; e < 4; ++e)
            t.part[wave][u][e][lane] = g[u][e];
    __syncthreads();

    // the waves' sums in their order, the norm, the steps, and R times what X is divided by
    const auto sum = [&](int u, int e, int l) {
        double v = t.part[0][u][e][l];
#pragma unroll
        for (int w = 1; w < kThinWaves; ++w)
            v += t.part[w][u][e][l];
        return v;
    };
    const auto factor = [&](double trace) {
        float p0, p1;
        const double f = thin_factor(trace, &p0, &p1);
        if (threadIdx.x == 0) {
            t.power[0] = p0;
            t.power[1] = p1;
        }
        return f;
    };
    if constexpr (NP == 16) {
        if (wave == 0) {
            f64x4 G;
            double trace = 0.0;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                G[e] = sum(0, e, lane);
                trace += 4 * e + q == r ? G[e] : 0.0;
            }
#pragma unroll
            for (int o = 32; o >= 1; o >>= 1)
                trace += __shfl_xor(trace, o, 64);
            const double f = factor(trace), by = trace == 0.0 ? 0.0 : 1.0 / trace;
            const f64x4 R = thin_chain16(G * by, steps);
#pragma unroll
            for (int e = 0; e < 4; ++e)
                t.r[4 * e + q][r] = float(R[e] * f);
        }
        __syncthreads();
    } else {
        for (int e = threadIdx.x; e < 3 * 256; e += kThinThreads) {
            const int u = e / 256, l = e % 64, a = u / 2 * 16, b = (u + 1) / 2 * 16;
            const int i = a + 4 * (e / 64 % 4) + (l >> 4), j = b + (l & 15);
            const double v = sum(u, e / 64 % 4, l);
            t.sym[0][i][j] = v;
            t.sym[0][j][i] = v;
        }
        __syncthreads();
        double trace = 0.0;
        for (int i = 0; i < NP; ++i)
            trace += t.sym[0][i][i];
        const double f = factor(trace), by = trace == 0.0 ? 0.0 : 1.0 / trace;
        __syncthreads();
        for (int e = threadIdx.x; e < NP * NP; e += kThinThreads)
            t.sym[0][e / NP][e % NP] *= by;
        __syncthreads();
        int G = 0, P = 1, R = 2, S = 3;
        for (int step = 0; step < steps; ++step) {
            thin_product32(t.sym[P], t.sym[G], t.sym[G], 2.0315, -4.7750, 3.4445);
            if (step > 0) {
                thin_product32(t.sym[S], t.sym[P], t.sym[R], 1.0, 0.0, 0.0);
                const int old = R;
                R = S;
                S = old;
            }
            if (step + 1 < steps) {
                thin_product32(t.sym[S], t.sym[P], t.sym[G], 1.0, 0.0, 0.0);
                thin_product32(t.sym[G], t.sym[S], t.sym[P], 1.0, 0.0, 0.0);
            }
            if (step == 0) {
                const int old = R;
                R = P;
                P = old;
            }
        }
        for (int e = threadIdx.x; e < NP * NP; e += kThinThreads)
            t.r[e / NP][e % NP] = float(t.sym[R][e / NP][e % NP] * f);
        __syncthreads();
    }

    // R X over the workgroup's columns, blocks of 16 in turn
    const float p0 = t.power[0], p1 = t.power[1];
    f32x4 a[kBlocks][kBlocks];
#pragma unroll
    for (int bi = 0; bi < kBlocks; ++bi)
#pragma unroll
        for (int bk = 0; bk < kBlocks; ++bk)
            a[bi][bk] = *reinterpret_cast<const f32x4*>(&t.r[16 * bi + r][16 * bk + 4 * q]);
    for (int k0 = begin; k0 < end; k0 += W) {
        const int base = len <= W ? 0 : k0;  // column of X at the head of what LDS holds
        if (len > W) {
            __syncthreads();
            thin_load<NP, T>(t, m, wide, k0, end);
        }
        const int stop = min(end, k0 + W);
        for (int k = k0 + 16 * wave; k < stop; k += 16 * kThinWaves) {
            const int col = k + r;
            f32x4 acc[kBlocks] = {};
#pragma unroll
            for (int bk = 0; bk < kBlocks; ++bk)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float x = t.x[16 * bk + 4 * q + e][k - base + r] * p0 * p1;
#pragma unroll
                    for (int bi = 0; bi < kBlocks; ++bi)
                        acc[bi] = __builtin_amdgcn_mfma_f32_16x16x4f32(a[bi][bk][e], x, acc[bi], 0,
                                                                       0, 0);
                }
            if (col >= len)
                continue;
#pragma unroll
            for (int bi = 0; bi < kBlocks; ++bi)
                thin_result<FINAL>(m, wide, n, len, 16 * bi + 4 * q, col, acc[bi], decay);
        }
    }
}

template <typename T, int FINAL>
__global__ __launch_bounds__(kThinThreads) void k_orth_thin(Gate gate,
                                                            const Matrix* __restrict__ mats,
                                                            int first, int n, int parts, int steps,
                                                            float decay)
{
    __shared__ union {
        Thin<16> t16;
        Thin<32> t32;
    } lds;
    if (!descriptors_ok(gate))
        return;
    const Matrix& m = mats[first + blockIdx.x % uint32_t(n)];
    const int part = int(blockIdx.x / uint32_t(n));
    const int numel = m.rows * m.cols, len = max(m.rows, m.cols);
    if (numel == 0)
        return;
    if (!step_applies(gate)) {
        if (FINAL == kWeights && m.wb && part == 0)
            for (int e = threadIdx.x; e < numel; e += kThinThreads)
                m.wb[e] = bf16_bits(m.w[e]);
        return;
    }
    const int span = ((len + parts - 1) / parts + kThinSpan - 1) / kThinSpan * kThinSpan;
    const int begin = part * span, end = min(len, begin + span);
    if (begin >= len)
        return;
    if (m.rows <= 16 || m.cols <= 16)
        thin_matrix<16, T, FINAL>(lds.t16, m, steps, decay, begin, end);
    else
        thin_matrix<32, T, FINAL>(lds.t32, m, steps, decay, begin, end);
}

// ---------------------------------------------------------------- small matrices
//
// The same for 33 <= n <= 64, where G and its steps no longer leave LDS room for X: G of every
// slice of columns, the steps by one workgroup for each matrix, R X.  X is read twice and written
// once, by as many workgroups as there are slices.  224 of 64 x 4288 in fp32 take 377 us: 166 the
// Gram matrices (246 MB, 42 us at the rate of reading; 64-bit products, 63 us at theirs), 61 the
// steps (35 for a single matrix, one product after the other; a workgroup a CU), 143 R X; of 4288 x
// 64 143, 63 and 168.  What bounds the two passes is waiting: a wave asks for 64 bytes of each of
// 16 rows (single elements where X is tall), then multiplies, with no other read under way.

constexpr int kSmallSide = 64;
constexpr int kSmallSlice = 512;                            // columns
constexpr int kSmallBlocks = kSmallSide / 16;
constexpr int kSmallUpper = kSmallBlocks * (kSmallBlocks + 1) / 2;
constexpr int kSmallGram = kSmallUpper * 256;               // doubles of one slice
constexpr int kSmallR = 64 + kSmallSide * kSmallSide;       // two powers, and R at 64

// X[i][k .. k + 4) of the n x len matrix on its smaller side, zeros outside it.
template <typename T>
__device__ inline f32x4 small_load(const T* src, bool wide, int n, int len, int i, int k)
{
    f32x4 v = {0.0f, 0.0f, 0.0f, 0.0f};
    if (i >= n)
        return v;
    if (wide && k + 4 <= len) {
        const T* p = src + int64_t(i) * len + k;
        if constexpr (sizeof(T) == 4) {
            v = __builtin_bit_cast(f32x4, load_any(p));
        } else {
            typedef uint16_t u16x4_any __attribute__((ext_vector_type(4), aligned(2)));
            const u16x4_any w = *reinterpret_cast<const u16x4_any*>(p);
#pragma unroll
            for (int e = 0; e < 4; ++e)
                v[e] = __uint_as_float(uint32_t(w[e]) << 16);
        }
        return v;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (k + e < len)
            v[e] = load_value(src + (wide ? int64_t(i) * len + k + e : int64_t(k + e) * n + i));
    return v;
}

template <typename T>
__global__ __launch_bounds__(kThreads) void k_orth_small_gram(Gate gate,
                                                              const int64_t* __restrict__ prefix,
                                                              const Matrix* __restrict__ mats,
                                                              int first, int n_mats)
{
    __shared__ double part[kThreads / 64][kSmallGram];
    if (!descriptors_ok(gate) || !step_applies(gate))
        return;
    const int64_t unit = prefix[first] + blockIdx.x;
    const int at = find_matrix(prefix, first, n_mats, unit);
    const Matrix& m = mats[at];
    const int slice = int(unit - prefix[at]);
    const bool wide = m.rows <= m.cols;
    const int n = wide ? m.rows : m.cols, len = wide ? m.cols : m.rows;
    const int lane = int(threadIdx.x) & 63, wave = int(threadIdx.x) >> 6;
    const int r = lane & 15, q = lane >> 4;
    const T* src = static_cast<const T*>(m.src);
    const int k0 = slice * kSmallSlice, k1 = min(len, k0 + kSmallSlice);
    f64x4 g[kSmallUpper] = {};
    for (int k = k0 + 16 * wave; k < k1; k += 16 * (kThreads / 64)) {
        f32x4 x[kSmallBlocks];
#pragma unroll
        for (int b = 0; b < kSmallBlocks; ++b)
            x[b] = small_load(src, wide, n, len, 16 * b + r, k + 4 * q);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            int u = 0;
#pragma unroll
            for (int a = 0; a < kSmallBlocks; ++a)
#pragma unroll
                for (int b = a; b < kSmallBlocks; ++b, ++u)
                    g[u] = __builtin_amdgcn_mfma_f64_16x16x4f64(double(x[a][e]), double(x[b][e]),
                                                                g[u], 0, 0, 0);
        }
    }
#pragma unroll
    for (int u = 0; u < kSmallUpper; ++u)
#pragma unroll
        for (int e = 0; e < 4; ++e)
            part[wave][(u * 4 + e) * 64 + lane] = g[u][e];
    __syncthreads();
    double* to = m.gram + int64_t(slice) * kSmallGram;
    for (int e = threadIdx.x; e < kSmallGram; e += kThreads)
        to[e] = (part[0][e] + part[1][e]) + (part[2][e] + part[3][e]);
}

typedef double SmallSym[kSmallSide][kSmallSide + 2];

// dst = alpha * M N + beta * N + gamma * I, all symmetric: every wave two blocks of 16.
__device__ inline void small_product(SmallSym& dst, const SmallSym& M, const SmallSym& N,
                                     double alpha, double beta, double gamma)
{
    const int lane = int(threadIdx.x) & 63, wave = int(threadIdx.x) >> 6;
    const int r = lane & 15, q = lane >> 4;
    const int bi = wave / 2 * 16, bj = wave % 2 * 32;
    f64x4 acc[2] = {};
#pragma unroll 4
    for (int k = 0; k < kSmallSide; k += 4)
#pragma unroll
        for (int h = 0; h < 2; ++h)
            acc[h] = __builtin_amdgcn_mfma_f64_16x16x4f64(M[bi + r][k + q],
                                                          N[bj + 16 * h + r][k + q], acc[h], 0, 0,
                                                          0);
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            const int i = bi + 4 * t + q, j = bj + 16 * h + r;
            dst[i][j] = alpha * acc[h][t] + beta * N[i][j] + (i == j ? gamma : 0.0);
        }
    __syncthreads();
}

__global__ __launch_bounds__(kThinThreads) void k_orth_small_steps(Gate gate,
                                                                   const Matrix* __restrict__ mats,
                                                                   int first, int steps)
{
    __shared__ SmallSym sym[4];
    if (!descriptors_ok(gate) || !step_applies(gate))
        return;
    const Matrix& m = mats[first + blockIdx.x];
    const int len = max(m.rows, m.cols), slices = (len + kSmallSlice - 1) / kSmallSlice;
    if (len == 0 || m.rows == 0 || m.cols == 0)
        return;
    for (int e = threadIdx.x; e < kSmallGram; e += kThinThreads) {
        double v = m.gram[e];
        for (int i = 1; i < slices; ++i)
            v += m.gram[int64_t(i) * kSmallGram + e];
        // block u of the upper ones, in the order in which they were made
        int a = 0, b = e / 256;
        while (b >= kSmallBlocks - a) {
            b -= kSmallBlocks - a;
            ++a;
        }
        const int l = e % 64, i = 16 * a + 4 * (e / 64 % 4) + (l >> 4), j = 16 * (a + b) + (l & 15);
        sym[0][i][j] = v;
        sym[0][j][i] = v;
    }
    __syncthreads();
    double trace = 0.0;
    for (int i = 0; i < kSmallSide; ++i)
        trace += sym[0][i][i];
    float p0, p1;
    const double f = thin_factor(trace, &p0, &p1), by = trace == 0.0 ? 0.0 : 1.0 / trace;
    __syncthreads();
    for (int e = threadIdx.x; e < kSmallSide * kSmallSide; e += kThinThreads)
        sym[0][e / kSmallSide][e % kSmallSide] *= by;
    __syncthreads();
    int G = 0, P = 1, R = 2, S = 3;
    for (int step = 0; step < steps; ++step) {
        small_product(sym[P], sym[G], sym[G], 2.0315, -4.7750, 3.4445);
        if (step > 0) {
            small_product(sym[S], sym[P], sym[R], 1.0, 0.0, 0.0);
            const int old = R;
            R = S;
            S = old;
        }
        if (step + 1 < steps) {
            small_product(sym[S], sym[P], sym[G], 1.0, 0.0, 0.0);
            small_product(sym[G], sym[S], sym[P], 1.0, 0.0, 0.0);
        }
        if (step == 0) {
            const int old = R;
            R = P;
            P = old;
        }
    }
    if (threadIdx.x == 0) {
        m.r[0] = p0;
        m.r[1] = p1;
    }
    for (int e = threadIdx.x; e < kSmallSide * kSmallSide; e += kThinThreads)
        m.r[64 + e] = float(sym[R][e / kSmallSide][e % kSmallSide] * f);
}

template <typename T, int FINAL>
__global__ __launch_bounds__(kThreads) void k_orth_small_apply(Gate gate,
                                                               const int64_t* __restrict__ prefix,
                                                               const Matrix* __restrict__ mats,
                                                               int first, int n_mats, float decay)
{
    if (!descriptors_ok(gate))
        return;
    const int64_t unit = prefix[first] + blockIdx.x;
    const int at = find_matrix(prefix, first, n_mats, unit);
    const Matrix& m = mats[at];
    const int slice = int(unit - prefix[at]);
    const bool wide = m.rows <= m.cols;
    const int n = wide ? m.rows : m.cols, len = wide ? m.cols : m.rows;
    const int k0 = slice * kSmallSlice, k1 = min(len, k0 + kSmallSlice);
    if (!step_applies(gate)) {
        if (FINAL == kWeights && m.wb)
            for (int e = threadIdx.x; e < n * (k1 - k0); e += kThreads) {
                const int to = wide ? e / (k1 - k0) * len + k0 + e % (k1 - k0) : k0 * n + e;
                m.wb[to] = bf16_bits(m.w[to]);
            }
        return;
    }
    const int lane = int(threadIdx.x) & 63, wave = int(threadIdx.x) >> 6;
    const int r = lane & 15, q = lane >> 4;
    const T* src = static_cast<const T*>(m.src);
    const float p0 = m.r[0], p1 = m.r[1];
    f32x4 a[kSmallBlocks][kSmallBlocks];
#pragma unroll
    for (int bi = 0; bi < kSmallBlocks; ++bi)
#pragma unroll
        for (int bk = 0; bk < kSmallBlocks; ++bk)
            a[bi][bk] = *reinterpret_cast<const f32x4*>(m.r + 64 + (16 * bi + r) * kSmallSide +
                                                        16 * bk + 4 * q);
    for (int k = k0 + 16 * wave; k < k1; k += 16 * (kThreads / 64)) {
        const int col = k + r;
        float x[kSmallBlocks][4];
#pragma unroll
        for (int bk = 0; bk < kSmallBlocks; ++bk)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int i = 16 * bk + 4 * q + e;
                x[bk][e] = i < n && col < len ? load_value(src + (wide ? i * len + col : col * n + i))
                                              : 0.0f;
            }
        f32x4 acc[kSmallBlocks] = {};
#pragma unroll
        for (int bk = 0; bk < kSmallBlocks; ++bk)
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int bi = 0; bi < kSmallBlocks; ++bi)
                    acc[bi] = __builtin_amdgcn_mfma_f32_16x16x4f32(a[bi][bk][e],
                                                                   x[bk][e] * p0 * p1, acc[bi], 0,
                                                                   0, 0);
        if (col < len)
#pragma unroll
            for (int bi = 0; bi < kSmallBlocks; ++bi)
                thin_result<FINAL>(m, wide, n, len, 16 * bi + 4 * q, col, acc[bi], decay);
    }
}

// ---------------------------------------------------------------- host side

// The workspace: [tag][prefixes][momentum descriptors][matrices][square sums][partials] and
// the region that the batches share.
//
// A batch is what one sequence of launches works on.  Large ones fill the last rounds of their
// launches: the three feed-forward matrices of a 27B-class layer (2.7e8 elements) one by one
// leave a fifth of the CUs idle in every product (its Muon step 27.5 ms, one by one 28.0).  16 bytes
// of workspace go with an element.
constexpr int64_t kBatchElems = int64_t(1) << 27;  // padded elements of a batch of several,
constexpr int64_t kBatchLargest = 4;               // or this many of the list's largest matrix

enum { kPreUnits, kPreSlices, kPrePrep, kPreSym, kPreTile = kPreSym + 3, kPrefixes = kPreTile + 3 };

// Tile size and slices of the sums of a batch's G.
struct GramWay {
    int size, slices;
};

struct Plan {
    size_t prefix[kPrefixes], momentum, mats, header, squares, partials, region[2], total;
    std::vector<int> order;    // the list's matrices in the order in which they are worked on
    std::vector<int> batch;    // first place of each batch, and the list's length
    std::vector<int> way;      // of each batch: how its matrices are worked on
    std::vector<size_t> sums;  // where in its region its sums of G's slices lie
    std::vector<GramWay> gram;
};

// How a matrix is worked on.  Thin and small ones in 64 bits on their smaller side.  Long ones take
// their steps in pairs, which saves a sixth of the multiply-adds or more (17408 x 5120: 5.5 ms, in
// single steps 7.3; the projections of a 3B-class layer 2.6 and 3.5); 128 rows or columns are what
// sizes are padded to anyway.
enum { kThin, kSmall, kSingle, kPairs, kWays };

int way_of(int64_t rows, int64_t cols)
{
    const int64_t n = std::min(rows, cols), m = std::max(rows, cols);
    if (n <= kThinSide)
        return kThin;
    if (n <= kSmallSide)
        return kSmall;
    return n >= kTile && m >= 2 * n ? kPairs : kSingle;
}

int64_t padded(int64_t x) { return int64_t(round_up(size_t(x), kTile)); }

int64_t slices_of(int64_t rows, int64_t cols)
{
    return host::ceil_div(std::max(rows, cols), kSmallSlice);
}

int64_t units_of(int64_t numel, int64_t span) { return (numel + span - 1) / span; }

bool tiled(int way) { return way == kSingle || way == kPairs; }

// Tiles of `tile` on and above the diagonal of side x side.
int64_t triangle(int64_t side, int64_t tile)
{
    const int64_t n = host::ceil_div(side, tile);
    return n * (n + 1) / 2;
}

// The cheapest tiles and slices, for sums of up to `steps` steps and `bytes` of one slice's sums.  A
// round's step takes 0.48 us by two tiles of 64 a CU (0.39 by one), 1.12 by two of 128 (0.6) and 1.5
// by one of 256, the rest of a round 3, 5 and 9; joining slices takes 12 us beside their bytes'
// way to memory and back.  In slices only where that saves a fifth by this account: 128 x 17408 takes
// 151 us and in one piece 336, 1024 x 17408 502 and 641, eight of 256 x 8192 328 and 387; without the
// sums' bytes in the account 4096 x 4096 was cut as well and took 2253 instead of 1671.
GramWay gram_way(const int64_t (&tiles)[3], int64_t steps, size_t bytes)
{
    constexpr int64_t kCus = 256;
    constexpr double kAlone[3] = {0.39, 0.6, 1.5}, kFull[3] = {0.48, 1.12, 1.5}, kRest[3] = {3, 5, 9};
    GramWay best{-1, 1};  // tiles as for the other products
    double whole = 0.0, least = 0.0;
    for (const int slices : {1, 2, 4, 8, 16}) {
        const int64_t per = host::ceil_div(steps, 2 * slices) * 2;
        if (slices > 1 && per < 8)
            break;
        for (int size = 0; size < 3; ++size) {
            const int64_t all = tiles[size] * slices, places = size == 2 ? kCus : 2 * kCus;
            const double step = all <= kCus ? kAlone[size] : kFull[size];
            double cost = double(host::ceil_div(all, places)) * (double(per) * step + kRest[size]);
            if (slices == 1) {
                whole = size == 0 ? cost : std::min(whole, cost);
                least = 0.8 * whole;
                continue;
            }
            cost += 12.0 + double(bytes) * slices / 4.0e6;
            if (cost < least) {
                least = cost;
                best = GramWay{size, slices};
            }
        }
    }
    return best;
}

// Bytes of a matrix in the region: X in three layouts twice, three n x n matrices, the Muon
// step's update.
struct Place {
    size_t h[2], t[2], l[2], sym[3], gram, r, u, bytes;
};

Place place(int64_t rows, int64_t cols, bool muon)
{
    Place p;
    const int way = way_of(rows, cols);
    const size_t x = tiled(way) ? size_t(padded(rows)) * size_t(padded(cols)) * 2 : 0;
    const size_t side = tiled(way) ? size_t(std::min(padded(rows), padded(cols))) : 0;
    const size_t slices = way == kSmall ? size_t(slices_of(rows, cols)) : 0;
    size_t at = 0;
    const auto take = [&](size_t bytes) {
        const size_t here = at;
        at += round_up(bytes, 256);
        return here;
    };
    for (int i = 0; i < 2; ++i) {
        p.h[i] = take(x);
        p.t[i] = take(x);
        p.l[i] = take(x);
    }
    for (int i = 0; i < 3; ++i)
        p.sym[i] = take(side * side * 2);
    p.gram = take(slices * kSmallGram * sizeof(double));
    p.r = take(way == kSmall ? kSmallR * sizeof(float) : 0);
    p.u = take(muon ? size_t(rows) * size_t(cols) * 4 : 0);
    p.bytes = at;
    return p;
}

// span: elements of a unit of the sums of squares.
Plan make_plan(const int64_t* rows, const int64_t* cols, int K, bool muon, int64_t span)
{
    Plan p;
    size_t at = host::kTagBytes;
    for (int i = 0; i < kPrefixes; ++i) {
        p.prefix[i] = at;
        at += round_up(sizeof(int64_t) * (size_t(K) + 1), 64);
    }
    p.momentum = at;
    at += muon ? round_up(sizeof(host::MomentumTensor) * size_t(K), 64) : 0;
    p.mats = at;
    at += round_up(sizeof(Matrix) * size_t(K), 64);
    p.header = at;
    p.squares = round_up(at, 256);
    p.partials = p.squares + round_up(sizeof(double) * size_t(K), 256);
    for (int way = 0; way < kWays; ++way)
        for (int k = 0; k < K; ++k)
            if (way_of(rows[k], cols[k]) == way)
                p.order.push_back(k);
    int64_t most = kBatchElems;
    for (int k = 0; k < K; ++k)
        most = std::max(most, kBatchLargest * padded(rows[k]) * padded(cols[k]));
    int64_t units = 0, elems = 0;
    for (int i = 0; i < K; ++i) {
        const int k = p.order[i];
        const int way = way_of(rows[k], cols[k]);
        const int64_t n = tiled(way) ? padded(rows[k]) * padded(cols[k]) : rows[k] * cols[k];
        if (p.batch.empty() || way != p.way.back() || (elems > 0 && elems + n > most)) {
            p.batch.push_back(i);
            p.way.push_back(way);
            elems = 0;
        }
        units += units_of(rows[k] * cols[k], span);
        elems += n;
    }
    size_t region[2] = {0, 0};  // of single steps, and of everything else
    for (size_t b = 0; b < p.way.size(); ++b) {
        const int end = b + 1 < p.way.size() ? p.batch[b + 1] : K;
        int64_t tiles[3] = {}, steps = 0;
        size_t bytes = 0, squares = 0;
        for (int i = p.batch[b]; i < end; ++i) {
            const int k = p.order[i];
            if (rows[k] == 0 || cols[k] == 0)
                continue;
            bytes += place(rows[k], cols[k], muon).bytes;
            if (!tiled(p.way[b]))
                continue;
            const int64_t side = std::min(padded(rows[k]), padded(cols[k]));
            for (int size = 0; size < 3; ++size)
                tiles[size] += triangle(side, Tiny::kRows << size);
            steps = std::max(steps, std::max(padded(rows[k]), padded(cols[k])) / 64);
            squares += size_t(side) * size_t(side) * sizeof(float);
        }
        p.gram.push_back(gram_way(tiles, steps, squares));
        p.sums.push_back(bytes);
        if (p.gram[b].slices > 1)
            bytes += squares * size_t(p.gram[b].slices);
        size_t& most_bytes = region[p.way[b] == kSingle ? 0 : 1];
        most_bytes = std::max(most_bytes, bytes);
    }
    p.batch.push_back(K);
    p.region[0] = p.partials + round_up(sizeof(double) * size_t(units), 256);
    p.region[1] = p.region[0] + round_up(region[0], 256);
    p.total = p.region[1] + round_up(region[1], 256);
    return p;
}

// Sizes a call can take: rows and columns in [0, 2^23), so that 256 rows of the widest matrix, the
// largest tile's, stay within the 32-bit offsets of a tile's loads: the last is 255 * 2^24 on.
bool valid_sizes(const int64_t* rows, const int64_t* cols, int K)
{
    if (K < 0 || (K > 0 && (!rows || !cols)))
        return false;
    for (int k = 0; k < K; ++k)
        if (rows[k] < 0 || cols[k] < 0 || rows[k] >= (1 << 23) || cols[k] >= (1 << 23))
            return false;
    return true;
}

struct Call {
    const int64_t *rows, *cols;
    int K;
    bool muon;
    int64_t span;
    int in_dtype, out_dtype;  // of the sources (gradients) and of the results
    int ns_steps;
    void* workspace;
    size_t workspace_bytes;
    const int32_t* status;
    const void* state;
    hipStream_t st;
};

// The product launches of one batch.
struct Launch {
    const Gate& gate;
    const Matrix* mats;
    int first, n, cus;
    hipStream_t st;
    const int64_t* const* dev;  // prefixes on the device and on the host
    int64_t* const* pre;

    int64_t blocks(int i) const { return pre[i][first + n] - pre[i][first]; }

    template <int OP>
    void sym(const SymArgs& a) const
    {
        const int size = tile_size(kPreSym), i = kPreSym + size;
        auto* kernel = size == 0 ? k_orth_sym<Tiny, OP>
                       : size == 1 ? k_orth_sym<Small, OP> : k_orth_sym<Large, OP>;
        kernel<<<dim3(uint32_t(blocks(i))), kThreads, 0, st>>>(gate, dev[i], mats, first, n, a);
    }
    void gram(const SymArgs& a, const GramWay& way) const
    {
        if (way.slices == 1) {
            sym<kGram>(a);
            return;
        }
        const int i = kPreSym + way.size;
        auto* kernel = way.size == 0 ? k_orth_gram<Tiny>
                       : way.size == 1 ? k_orth_gram<Small> : k_orth_gram<Large>;
        kernel<<<dim3(uint32_t(blocks(i)), uint32_t(way.slices)), kThreads, 0, st>>>(
            gate, dev[i], mats, first, n, a.from);
        k_orth_gram_join<<<dim3(uint32_t(blocks(kPreSym))), kThreads, 0, st>>>(
            gate, dev[kPreSym], mats, first, n, way.slices, a);
    }
    template <int FINAL>
    void update(const UpdateArgs& a) const
    {
        const int size = tile_size(kPreTile), i = kPreTile + size;
        auto* kernel = size == 0 ? k_orth_update<Tiny, FINAL>
                       : size == 1 ? k_orth_update<Small, FINAL> : k_orth_update<Large, FINAL>;
        kernel<<<dim3(uint32_t(blocks(i))), kThreads, 0, st>>>(gate, dev[i], mats, first, n, a);
    }
    // Tiles of 64, 128 or 256 on a side, whose rounds are cheapest.  A step of 64 summed values takes
    // 1.85 us a round of one tile of 256 a CU, 1.12 us a round of two of 128 (0.6 where a CU has
    // one), 0.48 us of two of 64 (four: 1.15).  1024 x 1024 by tiles of 64 161 us, of 128 212, of
    // 256 524; 2048 x 2048 423, 365 and 776; 17408 x 5120 by tiles of 256 5.5 ms, of 128 6.5.
    int tile_size(int i) const
    {
        if (blocks(i) <= 2 * cus)
            return 0;
        const int64_t large = host::ceil_div(blocks(i + 2), cus) * 185;
        return large < host::ceil_div(blocks(i + 1), 2 * cus) * 112 ? 2 : 1;
    }
};

// A few thin matrices leave CUs idle: several workgroups take one, all of them its Gram matrix and
// steps, each its columns of the result.  Eight of 16 x 2048 take 14 us so, 19 by one workgroup
// each (of 2048 x 16 15 and 27, of 32 x 2048 36 and 50); 256 of them 26 either way.
constexpr int kThinParts = 16;

void launch_thin(const Gate& gate, const Matrix* mats, int first, int n, const Call& c, int cus,
                 float decay)
{
    const int parts = std::min(std::max(cus / n, 1), kThinParts);
    const bool wide_src = c.muon || c.in_dtype == LT_DTYPE_F32;
    auto* kernel = c.muon ? k_orth_thin<float, kWeights>
                   : c.out_dtype == LT_DTYPE_F32
                       ? (wide_src ? k_orth_thin<float, kOutF32> : k_orth_thin<uint16_t, kOutF32>)
                       : (wide_src ? k_orth_thin<float, kOutBf16> : k_orth_thin<uint16_t, kOutBf16>);
    kernel<<<dim3(uint32_t(n * parts)), kThinThreads, 0, c.st>>>(gate, mats, first, n, parts,
                                                                 c.ns_steps, decay);
}

void launch_small(const Gate& gate, const int64_t* prefix, const Matrix* mats, int first, int n,
                  int64_t slices, const Call& c, float decay)
{
    const bool wide_src = c.muon || c.in_dtype == LT_DTYPE_F32;
    auto* gram = wide_src ? k_orth_small_gram<float> : k_orth_small_gram<uint16_t>;
    gram<<<dim3(uint32_t(slices)), kThreads, 0, c.st>>>(gate, prefix, mats, first, n);
    k_orth_small_steps<<<dim3(uint32_t(n)), kThinThreads, 0, c.st>>>(gate, mats, first, c.ns_steps);
    auto* apply = c.muon ? k_orth_small_apply<float, kWeights>
                  : c.out_dtype == LT_DTYPE_F32
                      ? (wide_src ? k_orth_small_apply<float, kOutF32>
                                  : k_orth_small_apply<uint16_t, kOutF32>)
                      : (wide_src ? k_orth_small_apply<float, kOutBf16>
                                  : k_orth_small_apply<uint16_t, kOutBf16>);
    apply<<<dim3(uint32_t(slices)), kThreads, 0, c.st>>>(gate, prefix, mats, first, n, decay);
}

// A second stream of the library's own, for the batches of single steps beside those of pairs:
// the launches of a few square matrices fill half the CUs (two of 2048 x 2048: 272 tiles of
// 128 x 128; the projections of a 3B-class layer take 2.64 ms, on one stream 2.86).  It starts
// after what the caller's stream holds and the caller's stream goes on after it.  Calls enqueue on
// it one at a time; under capture there is none, and everything goes into the caller's stream.
class Fork {
public:
    Fork() = default;
    Fork(const Fork&) = delete;
    lt_err begin(hipStream_t st)
    {
        hipStreamCaptureStatus capture = hipStreamCaptureStatusNone;
        LT_TRY_HIP(hipStreamIsCapturing(st, &capture));
        if (capture != hipStreamCaptureStatusNone)
            return LT_OK;
        int dev;
        LT_TRY_HIP(hipGetDevice(&dev));
        static std::mutex mu;
        static std::unordered_map<int, Lane> lanes;
        lock_ = std::unique_lock<std::mutex>(mu);
        Lane& l = lanes[dev];
        if (!l.stream) {
            Lane made;
            LT_TRY_HIP(hipEventCreateWithFlags(&made.forked, hipEventDisableTiming));
            LT_TRY_HIP(hipEventCreateWithFlags(&made.joined, hipEventDisableTiming));
            LT_TRY_HIP(hipStreamCreateWithFlags(&made.stream, hipStreamNonBlocking));
            l = made;
        }
        LT_TRY_HIP(hipEventRecord(l.forked, st));
        LT_TRY_HIP(hipStreamWaitEvent(l.stream, l.forked, 0));
        lane_ = &l;
        st_ = st;
        return LT_OK;
    }
    ~Fork() { (void)end(); }  // a call that fails half way is joined too
    hipStream_t side(hipStream_t st) const { return lane_ ? lane_->stream : st; }
    lt_err end()
    {
        if (!lane_)
            return LT_OK;
        Lane& l = *lane_;
        lane_ = nullptr;
        LT_TRY_HIP(hipEventRecord(l.joined, l.stream));
        LT_TRY_HIP(hipStreamWaitEvent(st_, l.joined, 0));
        return LT_OK;
    }

private:
    struct Lane {
        hipStream_t stream = nullptr;
        hipEvent_t forked = nullptr, joined = nullptr;
    };
    Lane* lane_ = nullptr;
    hipStream_t st_ = nullptr;
    std::unique_lock<std::mutex> lock_;
};

// Descriptors in place, then every batch in turn: `begin` enqueues what leaves the sources
// and their sums of squares, `fill` completes a matrix's descriptor.
template <typename Fill, typename Begin>
lt_err run_batches(const Call& c, float decay, Fill fill, Begin begin)
{
    const int K = c.K;
    const Plan p = make_plan(c.rows, c.cols, K, c.muon, c.span);
    if (!c.workspace || !host::aligned(c.workspace, 256) || c.workspace_bytes < p.total)
        return fail(LT_ERR_WORKSPACE, "workspace must be 256-byte aligned and hold " +
                                          std::to_string(p.total) + " bytes");
    std::vector<uint8_t> image(p.header, 0);
    auto* ws = static_cast<uint8_t*>(c.workspace);
    int64_t* pre[kPrefixes];
    for (int i = 0; i < kPrefixes; ++i)
        pre[i] = reinterpret_cast<int64_t*>(image.data() + p.prefix[i]);
    auto* momentum = reinterpret_cast<host::MomentumTensor*>(image.data() + p.momentum);
    auto* mats = reinterpret_cast<Matrix*>(image.data() + p.mats);
    auto* partial = reinterpret_cast<double*>(ws + p.partials);
    for (size_t b = 0; b + 1 < p.batch.size(); ++b) {
        uint8_t* at = ws + p.region[p.way[b] == kSingle ? 0 : 1];
        auto* sums = reinterpret_cast<float*>(at + p.sums[b]);
        for (int i = p.batch[b]; i < p.batch[b + 1]; ++i) {
            const int k = p.order[i];  // the i-th matrix of the descriptors
            const int64_t numel = c.rows[k] * c.cols[k];
            Matrix& m = mats[i];
            int64_t grid[kPrefixes] = {};
            if (numel > 0) {
                const Place x = place(c.rows[k], c.cols[k], c.muon);
                for (int j = 0; j < 2; ++j) {
                    m.h[j] = reinterpret_cast<_Float16*>(at + x.h[j]);
                    m.t[j] = reinterpret_cast<_Float16*>(at + x.t[j]);
                    m.l[j] = reinterpret_cast<_Float16*>(at + x.l[j]);
                }
                for (int j = 0; j < 3; ++j)
                    m.sym[j] = reinterpret_cast<_Float16*>(at + x.sym[j]);
                m.gram = reinterpret_cast<double*>(at + x.gram);
                m.r = reinterpret_cast<float*>(at + x.r);
                m.partial = partial;
                m.square = reinterpret_cast<double*>(ws + p.squares) + i;
                m.rows = int32_t(c.rows[k]);
                m.cols = int32_t(c.cols[k]);
                m.rp = int32_t(padded(c.rows[k]));
                m.cp = int32_t(padded(c.cols[k]));
                m.units = int32_t(units_of(numel, c.span));
                fill(k, m, momentum[c.muon ? i : 0], reinterpret_cast<float*>(at + x.u));
                partial += m.units;
                at += x.bytes;
                const int64_t side = std::min(m.rp, m.cp);
                if (tiled(p.way[b]) && p.gram[b].slices > 1) {
                    m.sums = sums;
                    sums += side * side * p.gram[b].slices;
                }
                const auto rectangle = [&](int64_t t) {
                    return host::ceil_div(m.rp, t) * host::ceil_div(m.cp, t);
                };
                grid[kPreUnits] = m.units;
                grid[kPreSlices] = slices_of(c.rows[k], c.cols[k]);
                grid[kPrePrep] = rectangle(kPrep);
                for (int size = 0; size < 3; ++size) {
                    grid[kPreSym + size] = triangle(side, Tiny::kRows << size);
                    grid[kPreTile + size] = rectangle(Tiny::kRows << size);
                }
            }
            for (int j = 0; j < kPrefixes; ++j)
                pre[j][i + 1] = pre[j][i] + grid[j];
        }
    }
    if (K == 0 || pre[kPreTile][K] == 0)
        return LT_OK;  // every matrix is empty
    Gate gate;
    if (lt_err e = host::put_descriptors(image, ws, c.st, &gate.guard))
        return e;
    gate.status = c.status;
    gate.state = static_cast<const lt_step_state*>(c.state);
    const int64_t* dev[kPrefixes];
    for (int i = 0; i < kPrefixes; ++i)
        dev[i] = reinterpret_cast<const int64_t*>(ws + p.prefix[i]);
    const auto* d_mats = reinterpret_cast<const Matrix*>(ws + p.mats);
    const auto* d_momentum = reinterpret_cast<const host::MomentumTensor*>(ws + p.momentum);
    int cus;
    if (lt_err e = host::compute_units(&cus))
        return e;
    Fork fork;
    const auto has = [&](int way) {
        return std::find(p.way.begin(), p.way.end(), way) != p.way.end();
    };
    if (has(kSingle) && has(kPairs))
        if (lt_err e = fork.begin(c.st))
            return e;
    for (size_t b = 0; b + 1 < p.batch.size(); ++b) {
        const hipStream_t st = p.way[b] == kSingle ? fork.side(c.st) : c.st;
        const int first = p.batch[b], n = p.batch[b + 1] - first;
        const auto blocks = [&](int i) { return pre[i][first + n] - pre[i][first]; };
        if (n == 0 || blocks(kPreTile) == 0)
            continue;
        if (c.muon || tiled(p.way[b]))
            if (lt_err e = begin(gate, dev[kPreUnits], d_momentum, d_mats, first, n,
                                 pre[kPreUnits][first], blocks(kPreUnits), st))
                return e;
        if (!tiled(p.way[b])) {
            if (p.way[b] == kThin)
                launch_thin(gate, d_mats, first, n, c, cus, decay);
            else
                launch_small(gate, dev[kPreSlices], d_mats, first, n, blocks(kPreSlices), c, decay);
            LT_TRY_HIP(hipGetLastError());
            continue;
        }
        k_orth_norm<<<dim3(uint32_t(n)), kThreads, 0, st>>>(gate, d_mats, first);
        const bool wide_src = c.muon || c.in_dtype == LT_DTYPE_F32;
        auto* prep = wide_src ? k_orth_prepare<float> : k_orth_prepare<uint16_t>;
        prep<<<dim3(uint32_t(blocks(kPrePrep))), kThreads, 0, st>>>(gate, dev[kPrePrep], d_mats,
                                                                    first, n);
        const Launch launch{gate, d_mats, first, n, cus, st, dev, pre};
        int from = 0;
        for (int step = 0; step < c.ns_steps; from ^= 1) {
            launch.gram({step, from, 0, 0, 0}, p.gram[b]);
            launch.sym<kStep>({step, from, 0, 0, 1});
            const int now = p.way[b] == kPairs && step + 1 < c.ns_steps ? 2 : 1;
            if (now == 2) {
                launch.sym<kHalf>({step, from, 1, 0, 2});
                launch.sym<kNext>({step, from, 1, 2, 0});
                launch.sym<kStep>({step + 1, from, 0, 0, 2});
                launch.sym<kPair>({step + 1, from, 2, 1, 0});
            }
            const UpdateArgs args{step, now, from, now == 2 ? 0 : 1, decay};
            step += now;
            if (step < c.ns_steps)
                launch.update<kAgain>(args);
            else if (c.muon)
                launch.update<kWeights>(args);
            else if (c.out_dtype == LT_DTYPE_F32)
                launch.update<kOutF32>(args);
            else
                launch.update<kOutBf16>(args);
        }
        LT_TRY_HIP(hipGetLastError());
    }
    return fork.end();
}

void add_range(std::vector<host::Range>& r, const void* p, size_t bytes, bool written)
{
    const auto lo = reinterpret_cast<uintptr_t>(p);
    if (lo && bytes)
        r.push_back({lo, lo + bytes, written});
}

constexpr int kMaxNsSteps = 64;

}  // namespace

extern "C" {

size_t lt_orthogonalize_workspace_bytes(const int64_t* rows, const int64_t* cols, int n_matrices)
try {
    return valid_sizes(rows, cols, n_matrices)
               ? make_plan(rows, cols, n_matrices, false, kSquareUnit).total
               : 0;
} catch (...) {
    return 0;
}

lt_err lt_orthogonalize(const void* const* matrices, int in_dtype, void* const* out, int out_dtype,
                        const int64_t* rows, const int64_t* cols, int n_matrices, int ns_steps,
                        void* workspace, size_t workspace_bytes, void* stream)
try {
    host::clear_error();
    const int K = n_matrices;
    if (!valid_sizes(rows, cols, K) || (K > 0 && (!matrices || !out)))
        return fail(LT_ERR_INVALID_ARG, "matrix lists must hold n_matrices >= 0 entries with rows "
                                        "and cols in [0, 2^23)");
    if ((in_dtype != LT_DTYPE_F32 && in_dtype != LT_DTYPE_BF16) ||
        (out_dtype != LT_DTYPE_F32 && out_dtype != LT_DTYPE_BF16))
        return fail(LT_ERR_INVALID_ARG, "in_dtype and out_dtype must be LT_DTYPE_F32 or "
                                        "LT_DTYPE_BF16");
    if (ns_steps < 1 || ns_steps > kMaxNsSteps)
        return fail(LT_ERR_INVALID_ARG, "ns_steps must lie in [1, 64]");
    const size_t in = in_dtype == LT_DTYPE_BF16 ? 2 : 4, size = out_dtype == LT_DTYPE_BF16 ? 2 : 4;
    std::vector<host::Range> ranges;
    for (int k = 0; k < K; ++k) {
        const size_t numel = size_t(rows[k]) * size_t(cols[k]);
        if (numel == 0)
            continue;
        if (!matrices[k] || !out[k])
            return fail(LT_ERR_INVALID_ARG, "NULL matrix pointer at index " + std::to_string(k));
        if (!host::aligned(matrices[k], 16) || !host::aligned(out[k], 16))
            return fail(LT_ERR_ALIGNMENT, "matrix " + std::to_string(k) + " is not 16-byte aligned");
        add_range(ranges, matrices[k], numel * in, false);
        add_range(ranges, out[k], numel * size, true);
    }
    const std::string e = host::overlap(ranges);
    if (!e.empty())
        return fail(LT_ERR_INVALID_ARG, e);
    Call c{rows, cols, K, false, kSquareUnit, in_dtype, out_dtype, ns_steps, workspace,
           workspace_bytes, nullptr, nullptr, static_cast<hipStream_t>(stream)};
    return run_batches(
        c, 1.0f,
        [&](int k, Matrix& m, host::MomentumTensor&, float*) {
            m.src = matrices[k];
            m.out = out[k];
        },
        [&](const Gate& gate, const int64_t* prefix, const host::MomentumTensor*,
            const Matrix* mats, int first, int n, int64_t, int64_t units, hipStream_t st) {
            auto* squares = in_dtype == LT_DTYPE_F32 ? k_orth_squares<float>
                                                     : k_orth_squares<uint16_t>;
            squares<<<dim3(uint32_t(units)), kThreads, 0, st>>>(gate, prefix, mats, first, n);
            LT_TRY_HIP(hipGetLastError());
            return LT_OK;
        });
} catch (...) {
    return host::caught();
}

size_t lt_muon_workspace_bytes(const int64_t* rows, const int64_t* cols, int n_matrices,
                               int block_size)
try {
    return valid_sizes(rows, cols, n_matrices) && host::valid_block_size(block_size)
               ? make_plan(rows, cols, n_matrices, true, host::momentum_unit(block_size)).total
               : 0;
} catch (...) {
    return 0;
}

lt_err lt_muon_step(float* const* params, const void* const* grads, int grad_dtype,
                    int8_t* const* m_codes, float* const* m_absmax, uint16_t* const* params_bf16,
                    const int64_t* rows, const int64_t* cols, int n_matrices, int block_size,
                    int code_map, double lr, double momentum, int nesterov, double weight_decay,
                    double update_rms, int ns_steps, const float* coef, const int32_t* status,
                    const void* step_state, void* workspace, size_t workspace_bytes, void* stream)
try {
    host::clear_error();
    const int K = n_matrices;
    if (!valid_sizes(rows, cols, K) ||
        (K > 0 && (!params || !grads || !m_codes || !m_absmax)))
        return fail(LT_ERR_INVALID_ARG, "matrix lists must hold n_matrices >= 0 entries with rows "
                                        "and cols in [0, 2^23)");
    if (grad_dtype != LT_DTYPE_F32 && grad_dtype != LT_DTYPE_BF16)
        return fail(LT_ERR_INVALID_ARG, "grad_dtype must be LT_DTYPE_F32 or LT_DTYPE_BF16");
    if (!host::valid_block_size(block_size))
        return fail(LT_ERR_INVALID_ARG, "block_size must be a multiple of 64 in [64, 65536]");
    if (code_map != LT_MAP_LINEAR && code_map != LT_MAP_DYNAMIC)
        return fail(LT_ERR_INVALID_ARG, "code_map must be LT_MAP_LINEAR or LT_MAP_DYNAMIC");
    if (!(std::isfinite(lr) && lr >= 0.0 && std::isfinite(weight_decay) && weight_decay >= 0.0 &&
          momentum >= 0.0 && momentum < 1.0 && std::isfinite(update_rms) && update_rms > 0.0))
        return fail(LT_ERR_INVALID_ARG, "need finite lr >= 0, weight_decay >= 0 and "
                                        "update_rms > 0, and 0 <= momentum < 1");
    if (ns_steps < 1 || ns_steps > kMaxNsSteps)
        return fail(LT_ERR_INVALID_ARG, "ns_steps must lie in [1, 64]");
    if ((coef && !host::aligned(coef, 4)) || (status && !host::aligned(status, 4)) ||
        (step_state && !host::aligned(step_state, 16)))
        return fail(LT_ERR_ALIGNMENT, "coef and status must be 4-byte aligned, step_state 16-byte");
    const size_t gbytes = grad_dtype == LT_DTYPE_BF16 ? 2 : 4;
    std::vector<host::Range> ranges;
    for (int k = 0; k < K; ++k) {
        const size_t numel = size_t(rows[k]) * size_t(cols[k]);
        if (numel == 0)
            continue;
        if (!params[k] || !grads[k] || !m_codes[k] || !m_absmax[k])
            return fail(LT_ERR_INVALID_ARG, "NULL matrix pointer at index " + std::to_string(k));
        uint16_t* wb = params_bf16 ? params_bf16[k] : nullptr;
        if (!host::aligned(params[k], 16) || !host::aligned(grads[k], 16) ||
            !host::aligned(m_codes[k], 16) || !host::aligned(m_absmax[k], 4) ||
            !host::aligned(wb, 16))
            return fail(LT_ERR_ALIGNMENT, "matrix " + std::to_string(k) +
                                              ": arrays must be 16-byte aligned, absmax 4-byte");
        add_range(ranges, params[k], numel * 4, true);
        add_range(ranges, grads[k], numel * gbytes, false);
        add_range(ranges, m_codes[k], numel, true);
        add_range(ranges, m_absmax[k],
                  (numel + size_t(block_size) - 1) / size_t(block_size) * 4, true);
        add_range(ranges, wb, numel * 2, true);
    }
    const std::string e = host::overlap(ranges);
    if (!e.empty())
        return fail(LT_ERR_INVALID_ARG, e);
    host::MomentumScalars s;
    s.beta = float(momentum);
    s.rest = float(1.0 - momentum);
    s.nesterov = nesterov != 0;
    const int64_t span = host::momentum_unit(block_size);
    Call c{rows, cols, K, true, span, grad_dtype, LT_DTYPE_F32, ns_steps, workspace,
           workspace_bytes, status, step_state, static_cast<hipStream_t>(stream)};
    return run_batches(
        c, float(1.0 - lr * weight_decay),
        [&](int k, Matrix& m, host::MomentumTensor& d, float* u) {
            m.src = u;
            m.w = params[k];
            m.wb = params_bf16 ? params_bf16[k] : nullptr;
            m.rate = float(lr * update_rms * std::sqrt(double(std::max(rows[k], cols[k]))));
            d = host::MomentumTensor{grads[k], m_codes[k], m_absmax[k], u, m.partial,
                                     rows[k] * cols[k]};
        },
        [&](const Gate& gate, const int64_t* prefix, const host::MomentumTensor* momenta,
            const Matrix*, int first, int n, int64_t first_unit, int64_t units, hipStream_t st) {
            return host::launch_momentum(gate.guard, prefix, momenta, first, n, first_unit, units,
                                         grad_dtype, block_size, code_map, s, coef, status,
                                         step_state, st);
        });
} catch (...) {
    return host::caught();
}

}  // extern "C"
