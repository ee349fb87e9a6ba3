// int8.hip -- matrix products in 8-bit integers with a scale for each row of either operand (a
// token's, an output channel's), the gated projections made of them, and the quantizer.
//
// value = code * scale with scale = most / 127, `most` the row's largest magnitude.  Products of
// codes are summed in 32-bit integers, exactly and in any order: 127^2 * 2^17 fits them.  The
// scales leave the sum, so a result is one integer times two scales, three roundings of fp32.

#include "gated.h"
#include "host.h"

#include <algorithm>
#include <string>
#include <vector>

namespace {

using host::fail;
using namespace tiles;
using gated::store_row;

constexpr int kPitch = 128;  // a row of codes is padded with zeros to a multiple of this

int64_t code_pitch(int64_t cols) { return host::ceil_div(cols, kPitch) * kPitch; }

// ------------------------------------------------------------- quantizer

struct QuantizeArgs {
    const void* x;
    int64_t rows, cols, stride, pitch;
    int8_t* codes;
    float* scales;
};

// A row's factor for its codes and its scale, from its largest magnitude.  Below 2^-100 the
// factor would leave fp32's range: such a row is quantized as if it reached that.  A NaN or an
// infinity makes the scale NaN and the codes 0.
struct RowScale {
    float factor, scale;
};

__device__ inline RowScale scale_of(uint32_t top)
{
    if (top >= 0x7F800000u)
        return {0.0f, __builtin_nanf("")};
    const float most = fmaxf(__uint_as_float(top), 0x1p-100f);
    return {127.0f / most, most / 127.0f};
}

// The integer nearest to x * factor, ties to even, as a byte: the sum with 1.5 * 2^23 rounds the
// exact product once, at its last bit.
__device__ inline uint32_t code_of(float x, RowScale s)
{
    const float v = __builtin_fmaf(x, s.factor, 12582912.0f);
    return s.factor == 0.0f ? 0u : __float_as_uint(v) & 0xFFu;
}

// Eight values of a row, as they are stored.
template <typename T>
struct Eight {
    i32x4 w[sizeof(T) / 2];
    __device__ inline float at(int e) const
    {
        if constexpr (sizeof(T) == 2) {
            const auto v = uint32_t(w[0][e / 2]);
            return __uint_as_float(e % 2 == 0 ? v << 16 : v & 0xFFFF0000u);
        } else {
            return __int_as_float(w[e / 4][e % 4]);
        }
    }
    __device__ inline uint32_t largest(uint32_t top) const
    {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            top = max(top, __float_as_uint(at(e)) & 0x7FFFFFFFu);
        return top;
    }
    __device__ inline uint2 codes(RowScale s) const
    {
        uint32_t c[2] = {0, 0};
#pragma unroll
        for (int e = 0; e < 8; ++e)
            c[e / 4] |= code_of(at(e), s) << (8 * (e % 4));
        return make_uint2(c[0], c[1]);
    }
};

// From column `at` on; zeros behind the row's end.
template <typename T>
__device__ inline Eight<T> load_eight(const T* row, int64_t at, int64_t cols)
{
    constexpr int kLines = sizeof(T) / 2, kEach = 8 / kLines;
    Eight<T> v = {};
    if (at + 8 <= cols) {
#pragma unroll
        for (int c = 0; c < kLines; ++c)
            v.w[c] = load_any(row + at + c * kEach);
        return v;
    }
    if (at >= cols)
        return v;
#pragma unroll
    for (int c = 0; c < kLines; ++c)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if constexpr (sizeof(T) == 2) {
                const int64_t i = at + 2 * e;
                const uint32_t lo = i < cols ? row[i] : 0u, hi = i + 1 < cols ? row[i + 1] : 0u;
                v.w[c][e] = int(lo | hi << 16);
            } else {
                const int64_t i = at + 4 * c + e;
                v.w[c][e] = i < cols ? __float_as_int(row[i]) : 0;
            }
        }
    return v;
}

// A row by WAVES waves, eight values a lane and HELD pieces of the row in registers; what is
// longer is read a second time (out of L2).  More registers mean fewer waves and cost more than
// that: rows of 17408 by sixteen waves with one piece 88 us (8192 rows of bf16, 4.8 TB/s), with
// three 101, by four with four 105; rows of 5120 by four waves with two pieces 46 (17408 rows,
// 5.8 TB/s), with four 59; rows of 1024 by one wave with one 34 (65536 rows), by four 60.
template <typename T, int WAVES, int HELD>
__global__ __launch_bounds__(WAVES < 4 ? 256 : 64 * WAVES) void k_int8_quantize(QuantizeArgs a)
{
    constexpr int kThreads = 64 * WAVES, kRows = WAVES < 4 ? 4 / WAVES : 1;
    __shared__ uint32_t tops[WAVES];
    const int t = int(threadIdx.x) % kThreads, wave = int(threadIdx.x) >> 6;
    for (int64_t r0 = int64_t(blockIdx.x) * kRows; r0 < a.rows; r0 += int64_t(gridDim.x) * kRows) {
        const int64_t row = r0 + int(threadIdx.x) / kThreads;
        const bool there = row < a.rows;
        const T* x = static_cast<const T*>(a.x) + (there ? row : 0) * a.stride;
        const int64_t cols = there ? a.cols : 0;
        Eight<T> v[HELD];
        uint32_t top = 0;
#pragma unroll
        for (int h = 0; h < HELD; ++h)
            v[h] = load_eight(x, (h * kThreads + t) * 8, cols);
#pragma unroll
        for (int h = 0; h < HELD; ++h)
            top = v[h].largest(top);
        for (int64_t at = (HELD * kThreads + t) * 8; at < cols; at += kThreads * 8)
            top = load_eight(x, at, cols).largest(top);
#pragma unroll
        for (int o = 32; o >= 1; o >>= 1)
            top = max(top, uint32_t(__shfl_xor(int(top), o, 64)));
        if constexpr (WAVES > 1) {
            if (t % 64 == 0)
                tops[wave] = top;
            __syncthreads();
#pragma unroll
            for (int i = 0; i < WAVES; ++i)
                top = max(top, tops[i]);
            __syncthreads();
        }
        if (!there)
            continue;
        const RowScale s = scale_of(top);
        int8_t* to = a.codes + row * a.pitch;
        if (t == 0)
            a.scales[row] = s.scale;
#pragma unroll
        for (int h = 0; h < HELD; ++h) {
            const int64_t at = (h * kThreads + t) * 8;
            if (at < a.pitch)
                *reinterpret_cast<uint2*>(to + at) = v[h].codes(s);
        }
        for (int64_t at = (HELD * kThreads + t) * 8; at < a.pitch; at += kThreads * 8)
            *reinterpret_cast<uint2*>(to + at) = load_eight(x, at, cols).codes(s);
    }
}

// ------------------------------------------------------------- products

struct ProductArgs {
    const uint8_t *a, *b, *c;  // c: the second weight of a pair
    const float *a_scales, *b_scales, *c_scales;
    int64_t m, n, pitch;
    int steps, slice;
    int activation;
    void* out;
    int64_t stride;
    int32_t* partial;  // several slices: [slice][weight][m][n]
};

__device__ inline float scaled(float bits, float row, float col)
{
    return float(__float_as_int(bits)) * row * col;
}

template <bool F32>
struct ProductWriter {
    static constexpr bool kTurned = false;
    static constexpr int kSlots = 8;
    const ProductArgs& g;
    int64_t r0, c0;
    float s[8], t[8];  // the lane's columns' scales, of either weight
    float x[kSlots];   // rows'
    __device__ inline void columns(int col_)
    {
        const int64_t col = c0 + col_;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int64_t at = col + e < g.n ? col + e : g.n - 1;
            s[e] = g.b_scales[at];
            t[e] = g.c_scales ? g.c_scales[at] : 0.0f;
        }
    }
    __device__ inline float fetch(int row_) const
    {
        const int64_t row = r0 + row_;
        return g.a_scales[row < g.m ? row : g.m - 1];
    }
    __device__ inline void fetch(int row, int, int p) { x[p] = fetch(row); }
    __device__ inline void turn(int, int, const float (&)[8]) {}
    __device__ inline void store(int row_, int col_, float (&v)[8], int p)
    {
        const int64_t row = r0 + row_, col = c0 + col_;
        if (row >= g.m || col >= g.n)
            return;
        if (g.partial) {  // the integers' bits
            store_row<true>(g.partial, (int64_t(blockIdx.y) * g.m + row) * g.n + col, v,
                            g.n - col);
            return;
        }
#pragma unroll
        for (int e = 0; e < 8; ++e)
            v[e] = scaled(v[e], x[p], s[e]);
        store_row<F32>(g.out, row * g.stride + col, v, g.n - col);
    }
    // of a pair
    __device__ inline void store(int row_, int col_, float (&u)[8], float (&v)[8], float scale)
    {
        const int64_t row = r0 + row_, col = c0 + col_;
        if (row >= g.m || col >= g.n)
            return;
        if (g.partial) {
            const int64_t at = (int64_t(blockIdx.y) * 2 * g.m + row) * g.n + col;
            store_row<true>(g.partial, at, u, g.n - col);
            store_row<true>(g.partial, at + g.m * g.n, v, g.n - col);
            return;
        }
        float a[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            u[e] = scaled(u[e], scale, s[e]);
            v[e] = scaled(v[e], scale, t[e]);
        }
        gated::activate(g.activation, u, a);
#pragma unroll
        for (int e = 0; e < 8; ++e)
            u[e] = a[e] * v[e];
        store_row<F32>(g.out, row * g.stride + col, u, g.n - col);
    }
};

// Bound by the matrix cores' power: 8192 x 17408 x 5120 565 to 620 us by the card (2.4 to 2.6
// POP/s; the cores work 64% of the cycles at 1.97 GHz).  1237 x 2011 x 5003 22 us: 400 tiles of 128
// x 128 with 16 steps each, where 512 would fill the CUs.
template <typename Tile, bool F32>
__global__ __launch_bounds__(Tile::kThreads, Tile::kWavesPerSimd) void k_int8_product(ProductArgs g)
{
    __shared__ __align__(1024) uint8_t lds[Tile::kLdsBytes];
    const TilePlace at = tile_place(int(unit_of_workgroup(Tile::kRun)),
                                    int((g.m + Tile::kRows - 1) / Tile::kRows),
                                    int((g.n + Tile::kCols - 1) / Tile::kCols));
    const int64_t r0 = int64_t(at.row) * Tile::kRows, c0 = int64_t(at.col) * Tile::kCols;
    const int first = int(blockIdx.y) * g.slice, steps = min(g.slice, g.steps - first);
    Tile tile;
    Int8<Tile::kPinned> mul;
    const int64_t k0 = int64_t(first) * kStepBytes;
    product(mul, tile, g.a + r0 * g.pitch + k0, g.pitch, g.m - r0, g.b + c0 * g.pitch + k0, g.pitch,
            g.n - c0, steps, lds);
    ProductWriter<F32> w{g, r0, c0};
    finish(tile, lds, w);
}

// A tile's columns are half either weight's.  Short sums are bound by the tiles' ends (scales,
// activation, stores: 14 us of a largest tile's 35 with 16 steps): 4096 x 2048 x 11008 200 us.
template <typename Tile, bool F32>
__global__ __launch_bounds__(Tile::kThreads, Tile::kWavesPerSimd) void k_int8_gated(ProductArgs g)
{
    __shared__ __align__(1024) uint8_t lds[Tile::kLdsBytes];
    constexpr int kCols = Tile::kCols / 2;
    const TilePlace at = tile_place(int(unit_of_workgroup(Tile::kRun)),
                                    int((g.m + Tile::kRows - 1) / Tile::kRows),
                                    int((g.n + kCols - 1) / kCols));
    const int64_t r0 = int64_t(at.row) * Tile::kRows, c0 = int64_t(at.col) * kCols;
    const int first = int(blockIdx.y) * g.slice, steps = min(g.slice, g.steps - first);
    Tile tile;
    Int8<Tile::kPinned> mul;
    const int64_t k0 = int64_t(first) * kStepBytes;
    product_pairs(mul, tile, g.a + r0 * g.pitch + k0, g.pitch, g.m - r0, g.b + c0 * g.pitch + k0,
                  g.pitch, g.c + c0 * g.pitch + k0, g.pitch, g.n - c0, steps, lds);
    ProductWriter<F32> w{g, r0, c0};
    finish_pairs(tile, lds, w);
}

// Results of the slices' sums.  Bound by latency: 64 x 2048 from eight slices 4.0 us.
template <int B, bool F32>
__global__ __launch_bounds__(256) void k_int8_join(ProductArgs g, int slices)
{
    const int64_t all = g.m * g.n;
    for (int64_t e = int64_t(blockIdx.x) * 256 + threadIdx.x; e < all;
         e += int64_t(gridDim.x) * 256) {
        int s[B];
#pragma unroll
        for (int b = 0; b < B; ++b)
            s[b] = g.partial[b * all + e];
#pragma unroll 4
        for (int i = 1; i < slices; ++i)
#pragma unroll
            for (int b = 0; b < B; ++b)
                s[b] += g.partial[(i * B + b) * all + e];
        const int64_t row = e / g.n, col = e % g.n;
        float v = float(s[0]) * g.a_scales[row] * g.b_scales[col];
        if constexpr (B == 2) {
            const float u[1] = {v};
            float a[1];
            gated::activate(g.activation, u, a);
            v = a[0] * (float(s[1]) * g.a_scales[row] * g.c_scales[col]);
        }
        if constexpr (F32)
            static_cast<float*>(g.out)[row * g.stride + col] = v;
        else
            static_cast<uint16_t*>(g.out)[row * g.stride + col] = gated::bf16_bits(v);
    }
}

// ------------------------------------------------------------- few tokens

// Results for up to 16 tokens where a wave can hold its share of them: eight waves cut the sum,
// each with up to STEPS steps of 128 values of every token as codes in its registers, and go
// through blocks of 16 weight rows together, the next block's codes under way while one is
// multiplied.  x is read once for a workgroup, and where it comes as values (X) it is quantized
// there, with the tokens' largest magnitudes from all eight waves: an answer is one launch.  Bound
// by reading the weights, short ones by latency: 16 tokens' codes through two of 5120 x 17408 36 us
// (4.9 TB/s), a token's values through one of 2048 x 11008 8.8.
enum { kCodes, kF32, kBf16 };

struct HeldArgs {
    const uint8_t* w[2];         // one or two weights
    const float* w_scales[2];
    const void* x;
    int64_t x_stride;            // of values
    const float* x_scales;       // of codes
    int64_t m, n, k, pitch;
    int steps;
    int activation, f32;
    void* out;
    int64_t stride;
};

constexpr int kHeldWaves = 8;

struct Codes32 {
    i32x4 w[2];
};

template <int STEPS, int B, int X>
__global__ __launch_bounds__(64 * kHeldWaves) void k_int8_held(HeldArgs g)
{
    typedef typename std::conditional<X == kF32, float, uint16_t>::type Value;
    extern __shared__ i32x4 held_lds[];  // x's codes, m rows of pitch + 16 bytes, before the sums
    typedef int Sums[B][kHeldWaves][256];
    auto* sums = reinterpret_cast<Sums*>(held_lds);  // [2]
    __shared__ uint32_t tops[kHeldWaves];
    __shared__ float x_scale[16];
    const int lane = int(threadIdx.x) & 63, r = lane & 15, q = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x) >> 6);
    const int first = g.steps * wave / kHeldWaves;
    const int count = g.steps * (wave + 1) / kHeldWaves - first;
    const int64_t blocks = (g.n + 15) / 16;

    struct Rows {
        Codes32 codes[STEPS];
    } even, odd;
    const auto load = [&](int b, int64_t block, Rows& w) {
        int64_t row = block * 16 + r;
        row = row < g.n ? row : g.n - 1;
        const uint8_t* p = g.w[b] + row * g.pitch + int64_t(first) * 128 + 32 * q;
#pragma unroll
        for (int i = 0; i < STEPS; ++i)
            if (i < count) {
                w.codes[i].w[0] = load_any(p + i * 128);
                w.codes[i].w[1] = load_any(p + i * 128 + 16);
            }
    };

    // of a pair's rows both are under way as soon as there is room (16 tokens' codes through
    // 5120 x 17408 41.8 to 40.7 us; blocks of one weight gained nothing, and the longest shares
    // of values have no registers left)
    constexpr bool kBoth = B == 2 && (X == kCodes || STEPS < 8);
    const auto load_first = [&] {
        load(0, blockIdx.x, even);
        if constexpr (kBoth)
            load(1, blockIdx.x, odd);
    };

    Codes32 x[STEPS];
    const int64_t token = r < g.m ? r : g.m - 1;
    if constexpr (X == kCodes) {
        load_first();
        const uint8_t* p = static_cast<const uint8_t*>(g.x) + token * g.pitch +
                           int64_t(first) * 128 + 32 * q;
#pragma unroll
        for (int i = 0; i < STEPS; ++i)
            if (i < count) {
                x[i].w[0] = load_any(p + i * 128);
                x[i].w[1] = load_any(p + i * 128 + 16);
            }
        if (threadIdx.x < 16)
            x_scale[threadIdx.x] = g.x_scales[token];
    } else {
        // each value once: a token by one wave, or few tokens by several each; the first part is
        // under way before the weights are
        const int share = g.m == 1 ? 8 : g.m == 2 ? 4 : g.m <= 4 ? 2 : 1;
        const int part = wave % share, at_once = kHeldWaves / share;
        constexpr int kKept = 4;
        const int64_t step = int64_t(share) * 64 * 8, from = (part * 64 + lane) * 8;
        const int64_t code_row = g.pitch + 16;
        auto* codes = reinterpret_cast<uint8_t*>(held_lds);
        for (int t0 = 0; t0 < g.m; t0 += at_once) {
            const int t = t0 + wave / share;
            const bool there = t < g.m;
            const Value* row = static_cast<const Value*>(g.x) + (there ? t : 0) * g.x_stride;
            const int64_t cols = there ? g.k : 0;
            Eight<Value> v[kKept];
#pragma unroll
            for (int h = 0; h < kKept; ++h)
                v[h] = load_eight(row, from + h * step, cols);
            if (t0 == 0)
                load_first();
            uint32_t top = 0;
#pragma unroll
            for (int h = 0; h < kKept; ++h)
                top = v[h].largest(top);
            for (int64_t at = from + kKept * step; at < cols; at += step)
                top = load_eight(row, at, cols).largest(top);
#pragma unroll
            for (int o = 32; o >= 1; o >>= 1)
                top = max(top, uint32_t(__shfl_xor(int(top), o, 64)));
            if (share > 1) {  // all tokens at once
                if (lane == 0)
                    tops[wave] = top;
                __syncthreads();
                for (int i = 0; i < share; ++i)
                    top = max(top, tops[wave / share * share + i]);
            }
            if (!there)
                continue;
            const RowScale scale = scale_of(top);
            if (lane == 0)
                x_scale[t] = scale.scale;
#pragma unroll
            for (int h = 0; h < kKept; ++h)
                if (from + h * step < g.pitch)
                    *reinterpret_cast<uint2*>(codes + t * code_row + from + h * step) =
                        v[h].codes(scale);
            for (int64_t at = from + kKept * step; at < g.pitch; at += step)
                *reinterpret_cast<uint2*>(codes + t * code_row + at) =
                    load_eight(row, at, cols).codes(scale);
        }
        __syncthreads();
        const uint8_t* p = codes + token * code_row + int64_t(first) * 128 + 32 * q;
#pragma unroll
        for (int i = 0; i < STEPS; ++i)
            if (i < count) {
                x[i].w[0] = *reinterpret_cast<const i32x4*>(p + i * 128);
                x[i].w[1] = *reinterpret_cast<const i32x4*>(p + i * 128 + 16);
            }
        __syncthreads();
    }

    const auto multiply = [&](const Rows& w, int (&to)[kHeldWaves][256]) {
        i32x4 acc = {0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < STEPS; ++i)
            if (i < count)
#pragma unroll
                for (int c = 0; c < 2; ++c)
                    acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(w.codes[i].w[c], x[i].w[c], acc, 0,
                                                                0, 0);
        *reinterpret_cast<i32x4*>(&to[wave][lane * 4]) = acc;  // rows 4 q + e of token r
    };
    const auto finish = [&](int64_t block, int turn) {
        __syncthreads();  // and the other buffer's sums have been read
        const int e = int(threadIdx.x);
        const int64_t row = block * 16 + 4 * (e >> 6) + e % 4, tok = e / 4 % 16;
        if (e >= 256 || row >= g.n || tok >= g.m)
            return;
        float v[B];
#pragma unroll
        for (int b = 0; b < B; ++b) {
            int s = 0;
#pragma unroll
            for (int i = 0; i < kHeldWaves; ++i)
                s += sums[turn][b][i][e];
            v[b] = float(s) * x_scale[tok] * g.w_scales[b][row];
        }
        float y = v[0];
        if constexpr (B == 2) {
            const float u[1] = {v[0]};
            float a[1];
            gated::activate(g.activation, u, a);
            y = a[0] * v[1];
        }
        if (g.f32)
            static_cast<float*>(g.out)[tok * g.stride + row] = y;
        else
            static_cast<uint16_t*>(g.out)[tok * g.stride + row] = gated::bf16_bits(y);
    };
    int turn = 0;
    for (int64_t b = blockIdx.x; b < blocks; b += gridDim.x, turn ^= 1) {
        const int64_t next = b + gridDim.x;
        if constexpr (B == 2) {
            if constexpr (!kBoth)
                load(1, b, odd);
            multiply(even, sums[turn][0]);
            if (next < blocks)
                load(0, next, even);
            multiply(odd, sums[turn][1]);
            if constexpr (kBoth)
                if (next < blocks)
                    load(1, next, odd);
            finish(b, turn);
        } else {
            if (next < blocks)
                load(0, next, odd);
            multiply(even, sums[turn][0]);
            finish(b, turn);
            even = odd;
        }
    }
}

// ---------------------------------------------------------------- host side

constexpr int64_t kMostSummed = int64_t(1) << 17;  // 127^2 * 2^17 < 2^31
constexpr int64_t kMostGroups = int64_t(1) << 24;  // a grid counts threads in 32 bits

using gated::Way;

Way way_of(int64_t m, int64_t n, int64_t k, bool pair)
{
    return gated::way_of(m, n, int(host::ceil_div(k, kPitch)), pair);
}

bool valid_sizes(int64_t m, int64_t n, int64_t k)
{
    const int64_t most = int64_t(1) << 26;
    return m >= 0 && n >= 0 && k >= 0 && m < most && n < most && k <= kMostSummed &&
           host::ceil_div(m, 64) * host::ceil_div(n, 64) < kMostGroups;
}

bool valid_stride(int64_t rows, int64_t cols, int64_t stride)
{
    return stride >= cols && stride <= (int64_t(1) << 46) / std::max<int64_t>(rows, 1);
}

bool valid_dtype(int dtype) { return dtype == LT_DTYPE_F32 || dtype == LT_DTYPE_BF16; }

size_t span_bytes(int64_t rows, int64_t cols, int64_t stride, int dtype)
{
    if (rows == 0 || cols == 0)
        return 0;
    return size_t((rows - 1) * stride + cols) * (dtype == LT_DTYPE_BF16 ? 2 : 4);
}

lt_err launch_quantize(const void* x, int dtype, int64_t rows, int64_t cols, int64_t stride,
                       int8_t* codes, float* scales, hipStream_t st)
{
    const QuantizeArgs a{x, rows, cols, stride, code_pitch(cols), codes, scales};
    // by what measured fastest, see the kernel
    const auto go = [&](auto* kernel, int64_t rows_each, int threads) {
        const int64_t groups = std::min<int64_t>(host::ceil_div(rows, rows_each), 1 << 20);
        kernel<<<dim3(uint32_t(groups)), threads, 0, st>>>(a);
    };
    const auto pick = [&](auto zero) {
        typedef decltype(zero) T;
        if (a.pitch <= 1024)
            go(k_int8_quantize<T, 1, 1>, 4, 256);
        else if (a.pitch <= 2048)
            go(k_int8_quantize<T, 4, 1>, 1, 256);
        else if (a.pitch <= 6144)
            go(k_int8_quantize<T, 4, 2>, 1, 256);
        else if (a.pitch <= 8192)
            go(k_int8_quantize<T, 4, 4>, 1, 256);
        else
            go(k_int8_quantize<T, 16, 1>, 1, 1024);
    };
    if (dtype == LT_DTYPE_BF16)
        pick(uint16_t());
    else
        pick(float());
    LT_TRY_HIP(hipGetLastError());
    return LT_OK;
}

void launch_product(const ProductArgs& g, const Way& w, bool f32, hipStream_t st)
{
    const auto go = [&](auto* kernel, auto tile) {
        typedef decltype(tile) Tile;
        const dim3 grid(uint32_t(host::ceil_div(g.m, Tile::kRows) * host::ceil_div(g.n, Tile::kCols)),
                        uint32_t(w.slices));
        kernel<<<grid, Tile::kThreads, 0, st>>>(g);
    };
    if (w.tile == 256)
        go(f32 ? k_int8_product<Large16, true> : k_int8_product<Large16, false>, Large16());
    else if (w.tile == 128)
        go(f32 ? k_int8_product<Small16, true> : k_int8_product<Small16, false>, Small16());
    else
        go(f32 ? k_int8_product<Tiny16, true> : k_int8_product<Tiny16, false>, Tiny16());
}

void launch_gated(const ProductArgs& g, const Way& w, bool f32, hipStream_t st)
{
    const auto go = [&](auto* kernel, auto tile) {
        typedef decltype(tile) Tile;
        const dim3 grid(uint32_t(host::ceil_div(g.m, Tile::kRows) *
                                 host::ceil_div(g.n, Tile::kCols / 2)),
                        uint32_t(w.slices));
        kernel<<<grid, Tile::kThreads, 0, st>>>(g);
    };
    if (w.tile == 256)
        go(f32 ? k_int8_gated<Large16, true> : k_int8_gated<Large16, false>, Large16());
    else if (w.tile == 128)
        go(f32 ? k_int8_gated<Small16, true> : k_int8_gated<Small16, false>, Small16());
    else
        go(f32 ? k_int8_gated<Pair16, true> : k_int8_gated<Pair16, false>, Pair16());
}

lt_err zero_rows(void* out, int dtype, int64_t m, int64_t n, int64_t stride, hipStream_t st)
{
    return host::launch_zero(out, dtype == LT_DTYPE_F32 ? 4 : 2, m, n, stride, st);
}

// Whether few tokens' codes fit the registers of a workgroup.
bool held(int64_t m, int64_t k)
{
    return m <= gated::kFewTokens && k <= kHeldWaves * 8 * 128;
}

// Whether every workgroup quantizes x itself: 4 tokens through 5120 x 17408 23.1 us, with a launch
// of the quantizer before 23.6; 8 tokens 25.5 and 24.1; 8 through 2048 x 11008 9.0 and 9.6.
bool one_launch(int64_t m, int64_t k) { return held(m, k) && m * k <= 32768; }

// Of a product whose sums are cut.
size_t partial_bytes(int64_t m, int64_t n, int64_t k, bool pair)
{
    if (held(m, k))
        return 0;
    const Way w = way_of(m, n, k, pair);
    return w.slices == 1 ? 0 : size_t(w.slices) * size_t(m) * size_t(n) * (pair ? 8 : 4);
}

// Workspace of the calls that quantize x themselves: [codes][scales][the product's].
struct LinearLayout {
    size_t scales, matmul, total;
};

LinearLayout linear_layout(int64_t m, int64_t n, int64_t k, bool pair)
{
    LinearLayout l{0, 0, host::kNoWorkspace};
    if (one_launch(m, k))
        return l;
    l.scales = host::round_up(size_t(m) * size_t(code_pitch(k)), 256);
    l.matmul = l.scales + host::round_up(size_t(m) * 4, 256);
    l.total = l.matmul + partial_bytes(m, n, k, pair);
    return l;
}

// For sums that held() allows.
template <int B, int X>
void launch_held(const HeldArgs& g, int cus, hipStream_t st)
{
    const int each = int(host::ceil_div(g.steps, kHeldWaves));
    const auto go = [&](auto* kernel, int a_cu) {
        const int64_t groups = std::min<int64_t>(host::ceil_div(g.n, 16), int64_t(a_cu) * cus);
        const size_t codes = X == kCodes ? 0 : size_t(g.m) * size_t(g.pitch + 16);
        kernel<<<dim3(uint32_t(groups)), 64 * kHeldWaves,
                 std::max(codes, size_t(2 * B * kHeldWaves * 1024)), st>>>(g);
    };
    // one workgroup to a CU (a token through 5120 x 17408 21 us, with two 23, with one for every
    // block 26), two where they are small and find their codes made (16 tokens through
    // 2048 x 11008, codes given, 7.7 us, with one 8.2)
    if (each <= 2)
        go(k_int8_held<2, B, X>, X == kCodes ? 2 : 1);
    else if (each <= 5)
        go(k_int8_held<5, B, X>, 1);
    else
        go(k_int8_held<8, B, X>, 1);
}

template <int X>
lt_err run_held(const ProductArgs& g, const void* x, int64_t x_stride, int64_t k, int out_dtype,
                hipStream_t st)
{
    HeldArgs h{};
    h.w[0] = g.b;
    h.w[1] = g.c;
    h.w_scales[0] = g.b_scales;
    h.w_scales[1] = g.c_scales;
    h.x = x;
    h.x_stride = x_stride;
    h.x_scales = g.a_scales;
    h.m = g.m;
    h.n = g.n;
    h.k = k;
    h.pitch = code_pitch(k);
    h.steps = int(host::ceil_div(k, kPitch));
    h.activation = g.activation;
    h.f32 = out_dtype == LT_DTYPE_F32;
    h.out = g.out;
    h.stride = g.stride;
    int cus;
    if (lt_err e = host::compute_units(&cus))
        return e;
    if (g.c)
        launch_held<2, X>(h, cus, st);
    else
        launch_held<1, X>(h, cus, st);
    LT_TRY_HIP(hipGetLastError());
    return LT_OK;
}

// The product of codes, its arguments checked.  c: the second weight of a pair, or null.
lt_err run_product(const ProductArgs& args, int64_t k, int out_dtype, void* workspace,
                   hipStream_t st)
{
    ProductArgs g = args;
    const bool f32 = out_dtype == LT_DTYPE_F32, pair = g.c != nullptr;
    g.pitch = code_pitch(k);
    g.steps = int(host::ceil_div(k, kPitch));
    if (held(g.m, k))
        return run_held<kCodes>(g, g.a, 0, k, out_dtype, st);
    const Way w = way_of(g.m, g.n, k, pair);
    g.slice = w.slice;
    if (w.slices > 1)
        g.partial = static_cast<int32_t*>(workspace);
    if (pair)
        launch_gated(g, w, f32, st);
    else
        launch_product(g, w, f32, st);
    if (g.partial) {
        auto* join = pair ? f32 ? k_int8_join<2, true> : k_int8_join<2, false>
                     : f32 ? k_int8_join<1, true> : k_int8_join<1, false>;
        join<<<dim3(uint32_t(std::min<int64_t>(4096, host::ceil_div(g.m * g.n, 256)))), 256, 0,
               st>>>(g, w.slices);
    }
    LT_TRY_HIP(hipGetLastError());
    return LT_OK;
}

// f11's and f12's answers to values: w2 is the second weight of a pair, or not given.
lt_err answer(const void* x, int dtype, int64_t x_stride, const int8_t* w, const float* w_scales,
              bool pair, const int8_t* w2, const float* w2_scales, int activation, int64_t m,
              int64_t n, int64_t k, void* out, int out_dtype, int64_t out_stride, void* workspace,
              size_t workspace_bytes, void* stream)
{
    if (!valid_sizes(m, n, k) || !valid_stride(m, n, out_stride) || !valid_stride(m, k, x_stride))
        return fail(LT_ERR_INVALID_ARG, "need 0 <= m, n < 2^26, tiles of 64 x 64 < 2^24, 0 <= k <= "
                                        "2^17, x_stride >= k and out_stride >= n");
    if (!valid_dtype(dtype) || !valid_dtype(out_dtype))
        return fail(LT_ERR_INVALID_ARG, "dtypes must be LT_DTYPE_F32 or LT_DTYPE_BF16");
    if (pair && (activation < LT_ACT_SILU || activation > LT_ACT_RELU))
        return fail(LT_ERR_INVALID_ARG, "unknown activation");
    if (m == 0 || n == 0)
        return LT_OK;
    if (!out || (k > 0 && (!x || !w || !w_scales || (pair && (!w2 || !w2_scales)))))
        return fail(LT_ERR_INVALID_ARG, "x, the weight and out must not be NULL");
    if (!host::aligned(x, dtype == LT_DTYPE_BF16 ? 2 : 4) || !host::aligned(w, 16) ||
        !host::aligned(w2, 16) || !host::aligned(out, 16) || !host::aligned(w_scales, 4) ||
        !host::aligned(w2_scales, 4))
        return fail(LT_ERR_ALIGNMENT, "x and scales must be aligned to their elements, codes and "
                                      "out to 16 bytes");
    const hipStream_t st = static_cast<hipStream_t>(stream);
    if (k == 0)
        return zero_rows(out, out_dtype, m, n, out_stride, st);
    const bool one = one_launch(m, k);  // without a workspace
    const LinearLayout l = linear_layout(m, n, k, pair);
    if (!one && (!workspace || !host::aligned(workspace, 256) || workspace_bytes < l.total))
        return fail(LT_ERR_WORKSPACE, "workspace must be 256-byte aligned and hold " +
                                          std::to_string(l.total) + " bytes");
    const size_t ws_bytes = one ? 0 : l.total;
    const size_t out_bytes = span_bytes(m, n, out_stride, out_dtype);
    const size_t w_bytes = size_t(n) * size_t(code_pitch(k));
    const struct {
        const void* p;
        size_t bytes;
    } read[] = {{x, span_bytes(m, k, x_stride, dtype)}, {w, w_bytes}, {w_scales, size_t(n) * 4},
                {w2, w_bytes}, {w2_scales, size_t(n) * 4}};
    for (const auto& r : read)
        if (host::overlaps(out, out_bytes, r.p, r.bytes) ||
            host::overlaps(workspace, ws_bytes, r.p, r.bytes))
            return fail(LT_ERR_INVALID_ARG, "out or the workspace overlaps x or a weight");
    if (host::overlaps(out, out_bytes, workspace, ws_bytes))
        return fail(LT_ERR_INVALID_ARG, "out overlaps the workspace");
    ProductArgs g{};
    g.b = reinterpret_cast<const uint8_t*>(w);
    g.c = pair ? reinterpret_cast<const uint8_t*>(w2) : nullptr;
    g.b_scales = w_scales;
    g.c_scales = w2_scales;
    g.m = m;
    g.n = n;
    g.activation = activation;
    g.out = out;
    g.stride = out_stride;
    if (one)
        return dtype == LT_DTYPE_F32 ? run_held<kF32>(g, x, x_stride, k, out_dtype, st)
                                     : run_held<kBf16>(g, x, x_stride, k, out_dtype, st);
    auto* ws = static_cast<uint8_t*>(workspace);
    if (lt_err e = host::workspace_written(ws, l.total, st))
        return e;
    auto* codes = reinterpret_cast<int8_t*>(ws);
    auto* scales = reinterpret_cast<float*>(ws + l.scales);
    if (lt_err e = launch_quantize(x, dtype, m, k, x_stride, codes, scales, st))
        return e;
    g.a = ws;
    g.a_scales = scales;
    return run_product(g, k, out_dtype, ws + l.matmul, st);
}

}  // namespace

extern "C" {

int64_t lt_int8_code_pitch(int64_t cols) { return cols < 0 ? 0 : code_pitch(cols); }

lt_err lt_int8_quantize(const void* x, int dtype, int64_t rows, int64_t cols, int64_t row_stride,
                        int8_t* codes, float* scales, void* stream)
try {
    host::clear_error();
    if (!valid_dtype(dtype))
        return fail(LT_ERR_INVALID_ARG, "dtype must be LT_DTYPE_F32 or LT_DTYPE_BF16");
    const int64_t most = int64_t(1) << 31;
    if (rows < 0 || cols < 0 || rows >= most || cols >= most ||
        !valid_stride(rows, cols, row_stride))
        return fail(LT_ERR_INVALID_ARG, "need 0 <= rows, cols < 2^31 and row_stride >= cols");
    if (rows == 0 || cols == 0)
        return LT_OK;
    if (!x || !codes || !scales)
        return fail(LT_ERR_INVALID_ARG, "x, codes and scales must not be NULL");
    if (!host::aligned(x, dtype == LT_DTYPE_BF16 ? 2 : 4) || !host::aligned(codes, 16) ||
        !host::aligned(scales, 4))
        return fail(LT_ERR_ALIGNMENT, "x and scales must be aligned to their elements, codes to 16 "
                                      "bytes");
    const size_t x_bytes = span_bytes(rows, cols, row_stride, dtype);
    const size_t code_bytes = size_t(rows) * size_t(code_pitch(cols));
    if (host::overlaps(codes, code_bytes, x, x_bytes) ||
        host::overlaps(scales, size_t(rows) * 4, x, x_bytes) ||
        host::overlaps(codes, code_bytes, scales, size_t(rows) * 4))
        return fail(LT_ERR_INVALID_ARG, "x, codes and scales overlap");
    return launch_quantize(x, dtype, rows, cols, row_stride, codes, scales,
                           static_cast<hipStream_t>(stream));
} catch (...) {
    return host::caught();
}

size_t lt_int8_matmul_workspace_bytes(int64_t m, int64_t n, int64_t k)
{
    if (!valid_sizes(m, n, k))
        return 0;
    return size_t(host::workspace_for(int64_t(partial_bytes(m, n, k, false))));
}

lt_err lt_int8_matmul(const int8_t* a_codes, const float* a_scales, const int8_t* b_codes,
                      const float* b_scales, int64_t m, int64_t n, int64_t k, void* out,
                      int out_dtype, int64_t out_stride, void* workspace, size_t workspace_bytes,
                      void* stream)
try {
    host::clear_error();
    if (!valid_sizes(m, n, k) || !valid_stride(m, n, out_stride))
        return fail(LT_ERR_INVALID_ARG, "need 0 <= m, n < 2^26, tiles of 64 x 64 < 2^24, 0 <= k <= "
                                        "2^17 and out_stride >= n");
    if (!valid_dtype(out_dtype))
        return fail(LT_ERR_INVALID_ARG, "out_dtype must be LT_DTYPE_F32 or LT_DTYPE_BF16");
    if (m == 0 || n == 0)
        return LT_OK;
    if (!out || (k > 0 && (!a_codes || !a_scales || !b_codes || !b_scales)))
        return fail(LT_ERR_INVALID_ARG, "operands and out must not be NULL");
    if (!host::aligned(a_codes, 16) || !host::aligned(b_codes, 16) || !host::aligned(out, 16) ||
        !host::aligned(a_scales, 4) || !host::aligned(b_scales, 4))
        return fail(LT_ERR_ALIGNMENT, "codes and out must be 16-byte aligned, scales 4-byte");
    const hipStream_t st = static_cast<hipStream_t>(stream);
    if (k == 0)
        return zero_rows(out, out_dtype, m, n, out_stride, st);
    const size_t need = lt_int8_matmul_workspace_bytes(m, n, k);
    const bool sliced = partial_bytes(m, n, k, false) > 0;
    if (sliced && (!workspace || !host::aligned(workspace, 256) || workspace_bytes < need))
        return fail(LT_ERR_WORKSPACE, "workspace must be 256-byte aligned and hold " +
                                          std::to_string(need) + " bytes");
    const size_t out_bytes = span_bytes(m, n, out_stride, out_dtype);
    const size_t pitch = size_t(code_pitch(k));
    const struct {
        const void* p;
        size_t bytes;
    } read[] = {{a_codes, size_t(m) * pitch}, {b_codes, size_t(n) * pitch},
                {a_scales, size_t(m) * 4}, {b_scales, size_t(n) * 4}};
    for (const auto& r : read)
        if (host::overlaps(out, out_bytes, r.p, r.bytes) ||
            (sliced && host::overlaps(workspace, need, r.p, r.bytes)))
            return fail(LT_ERR_INVALID_ARG, "out or the workspace overlaps an operand");
    if (sliced) {
        if (host::overlaps(out, out_bytes, workspace, need))
            return fail(LT_ERR_INVALID_ARG, "out overlaps the workspace");
        if (lt_err e = host::workspace_written(workspace, need, st))
            return e;
    }
    ProductArgs g{};
    g.a = reinterpret_cast<const uint8_t*>(a_codes);
    g.b = reinterpret_cast<const uint8_t*>(b_codes);
    g.a_scales = a_scales;
    g.b_scales = b_scales;
    g.m = m;
    g.n = n;
    g.out = out;
    g.stride = out_stride;
    return run_product(g, k, out_dtype, workspace, st);
} catch (...) {
    return host::caught();
}

size_t lt_int8_linear_workspace_bytes(int64_t m, int64_t n, int64_t k)
{
    return valid_sizes(m, n, k) ? linear_layout(m, n, k, false).total : 0;
}

lt_err lt_int8_linear(const void* x, int dtype, int64_t x_stride, const int8_t* w_codes,
                      const float* w_scales, int64_t m, int64_t n, int64_t k, void* out,
                      int out_dtype, int64_t out_stride, void* workspace, size_t workspace_bytes,
                      void* stream)
try {
    host::clear_error();
    return answer(x, dtype, x_stride, w_codes, w_scales, false, nullptr, nullptr, 0, m, n, k, out,
                  out_dtype, out_stride, workspace, workspace_bytes, stream);
} catch (...) {
    return host::caught();
}

size_t lt_int8_gated_workspace_bytes(int64_t m, int64_t n, int64_t k)
{
    return valid_sizes(m, n, k) ? linear_layout(m, n, k, true).total : 0;
}

lt_err lt_int8_gated(const void* x, int dtype, int64_t x_stride, const int8_t* gate_codes,
                     const float* gate_scales, const int8_t* up_codes, const float* up_scales,
                     int activation, int64_t m, int64_t n, int64_t k, void* out, int out_dtype,
                     int64_t out_stride, void* workspace, size_t workspace_bytes, void* stream)
try {
    host::clear_error();
    return answer(x, dtype, x_stride, gate_codes, gate_scales, true, up_codes, up_scales,
                  activation, m, n, k, out, out_dtype, out_stride, workspace, workspace_bytes,
                  stream);
} catch (...) {
    return host::caught();
}

}  // extern "C"
