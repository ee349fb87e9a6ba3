// gated.hip -- the gated projections of a feed-forward block in bf16, forward and backward:
//
//   g = x Wg^T,  u = x Wu^T,  h = act(g) * u
//   a = u act'(g),  b = act(g)                       (kept by the forward pass, 24 bits each)
//   dg = dh * a,  du = dh * b                        (rounded to bf16 for the products)
//   dx = dg Wg + du Wu,  dWg = dg^T x,  dWu = du^T x
//
// Sums are fp32's.  The forward pass takes both products in one tile, the weights' rows in turns
// of 32, so that a lane ends with g and u of the same places and no product is stored.

#include "gated.h"
#include "host.h"

#include <algorithm>
#include <string>
#include <vector>

namespace {

using host::fail;
using namespace tiles;
using gated::store_row;
using gated::u16x8;

constexpr int kStep = 64;  // values of every row, per step of the main loop

int64_t padded(int64_t values) { return host::ceil_div(values, kStep) * kStep; }

// ------------------------------------------------------------- layouts

// Up to three matrices of bf16 as the products read them, in one launch: rows of whole steps, or
// whole steps of rows, with zeros behind, where a matrix as it is has other sizes or places.
struct Layout {
    const uint16_t* x;
    int64_t rows, cols, stride;
    uint16_t* out;
    int64_t out_rows, pitch;
    uint32_t first;  // workgroup of the launch
};

struct Layouts {
    Layout of[3];
    int count;
};

constexpr int64_t kPackLines = 256 * 4;  // of 16 bytes, to a workgroup

__device__ inline void pack(const Layouts& g, uint32_t group)
{
    const Layout& a = g.of[g.count > 2 && group >= g.of[2].first
                               ? 2
                               : g.count > 1 && group >= g.of[1].first ? 1 : 0];
    const int64_t lines = a.pitch / 8, all = a.out_rows * lines;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int64_t i = (int64_t(group) - a.first) * kPackLines + j * 256 + threadIdx.x;
        if (i >= all)
            return;
        const int64_t row = i / lines, col = i % lines * 8;
        const uint16_t* p = a.x + row * a.stride + col;
        u16x8 v = {};
        if (row < a.rows && col + 8 <= a.cols) {
            v = __builtin_bit_cast(u16x8, load_any(p));
        } else if (row < a.rows) {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                v[e] = col + e < a.cols ? p[e] : uint16_t(0);
        }
        *reinterpret_cast<i32x4*>(a.out + row * a.pitch + col) = __builtin_bit_cast(i32x4, v);
    }
}

// 16 bytes a lane, bound by memory: two weights of 5003 x 2011 and 1237 such tokens 15.9 us, 5.7
// TB/s read and written.
__global__ __launch_bounds__(256) void k_gated_pack(Layouts g) { pack(g, blockIdx.x); }

struct ZeroArgs {
    void* out;
    int64_t m, n, stride;
};

template <typename T>
__global__ __launch_bounds__(256) void k_zero_rows(ZeroArgs a)
{
    const int64_t all = a.m * a.n;
    for (int64_t e = int64_t(blockIdx.x) * 256 + threadIdx.x; e < all;
         e += int64_t(gridDim.x) * 256)
        static_cast<T*>(a.out)[e / a.n * a.stride + e % a.n] = 0;
}

// ------------------------------------------------------------- the forward pass

// What the backward pass needs of every result, a and b, in 24 bits each: their upper halves as
// bf16 and a byte more.  In bf16 alone either rounding would add as much to the gradients as
// theirs; in fp32 they take a third more memory.
struct Saved {
    uint16_t *a_high, *b_high;
    uint8_t *a_low, *b_low;
    int64_t pitch;  // values of a row, a multiple of 8
};

Saved saved_layout(void* saved, int64_t m, int64_t n)
{
    Saved s;
    s.pitch = host::ceil_div(n, 8) * 8;
    s.a_high = static_cast<uint16_t*>(saved);
    s.b_high = s.a_high + m * s.pitch;
    s.a_low = reinterpret_cast<uint8_t*>(s.b_high + m * s.pitch);
    s.b_low = s.a_low + m * s.pitch;
    return s;
}

// Eight values in 24 bits, rounded to nearest (halves away from zero) by a sum: an infinity stays
// one, and so does a NaN, whose payload comes from bf16 operands or the hardware and leaves the
// last byte clear.
__device__ inline void save_eight(uint16_t* high, uint8_t* low, int64_t at, const float (&v)[8])
{
    uint32_t r[8], h[4], l[4];
#pragma unroll
    for (int e = 0; e < 8; ++e)
        r[e] = __float_as_uint(v[e]) + 0x80u;
#pragma unroll
    for (int e = 0; e < 4; ++e) {  // bytes 3 and 2 of either, and byte 1
        h[e] = __builtin_amdgcn_perm(r[2 * e + 1], r[2 * e], 0x07060302u);
        l[e] = __builtin_amdgcn_perm(r[2 * e + 1], r[2 * e], 0x0C0C0501u);
    }
    *reinterpret_cast<uint4*>(high + at) = make_uint4(h[0], h[1], h[2], h[3]);
    *reinterpret_cast<uint2*>(low + at) =
        make_uint2(l[0] | l[1] << 16, l[2] | l[3] << 16);
}

// One of them.
__device__ inline void save_one(uint16_t* high, uint8_t* low, int64_t at, float v)
{
    const uint32_t r = __float_as_uint(v) + 0x80u;
    high[at] = uint16_t(r >> 16);
    low[at] = uint8_t(r >> 8);
}

// A result from its sums; with SAVE what the backward pass needs of it is kept.
template <bool SAVE>
__device__ inline float answer_one(const Saved& saved, int activation, int64_t row, int64_t col,
                                   float u, float v)
{
    const float g[1] = {u};
    float b[1], a[1];
    if constexpr (SAVE) {
        gated::activate(activation, g, b, a);
        const int64_t at = row * saved.pitch + col;
        save_one(saved.a_high, saved.a_low, at, a[0] * v);
        save_one(saved.b_high, saved.b_low, at, b[0]);
    } else {
        gated::activate(activation, g, b);
    }
    return b[0] * v;
}

__device__ inline void load_eight(const uint16_t* high, const uint8_t* low, int64_t at,
                                  float (&v)[8])
{
    const uint4 h = *reinterpret_cast<const uint4*>(high + at);
    const uint2 l = *reinterpret_cast<const uint2*>(low + at);
    const uint32_t hs[4] = {h.x, h.y, h.z, h.w}, ls[2] = {l.x, l.y};
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const uint32_t top = e % 2 == 0 ? hs[e / 2] << 16 : hs[e / 2] & 0xFFFF0000u;
        v[e] = __uint_as_float(top | (ls[e / 4] >> (8 * (e % 4)) & 0xFFu) << 8);
    }
}

struct ForwardArgs {
    const uint8_t *x, *gate, *up;
    int64_t x_pitch, gate_pitch, up_pitch;  // bytes
    int64_t m, n;
    int steps;
    int activation;
    void* out;
    int64_t stride;
    Saved saved;
    int slice;       // steps of each slice of the sum
    float* partial;  // several slices: [slice][weight][m][n]
};

template <bool F32, bool SAVE>
struct ForwardWriter {
    const ForwardArgs& g;
    int64_t r0, c0;
    __device__ inline int fetch(int) const { return 0; }
    __device__ inline void store(int row_, int col_, float (&u)[8], float (&v)[8], int)
    {
        const int64_t row = r0 + row_, col = c0 + col_;
        if (row >= g.m || col >= g.n)
            return;
        float h[8];
        if constexpr (SAVE) {
            float a[8], b[8];
            gated::activate(g.activation, u, b, a);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                a[e] *= v[e];
                h[e] = b[e] * v[e];
            }
            const int64_t at = row * g.saved.pitch + col;
            save_eight(g.saved.a_high, g.saved.a_low, at, a);
            save_eight(g.saved.b_high, g.saved.b_low, at, b);
        } else {
            if (g.partial) {
                const int64_t at = (int64_t(blockIdx.y) * 2 * g.m + row) * g.n + col;
                store_row<true>(g.partial, at, u, g.n - col);
                store_row<true>(g.partial, at + g.m * g.n, v, g.n - col);
                return;
            }
            gated::activate(g.activation, u, h);
#pragma unroll
            for (int e = 0; e < 8; ++e)
                h[e] *= v[e];
        }
        store_row<F32>(g.out, row * g.stride + col, h, g.n - col);
    }
};

// A tile's columns are half the gate's and half the up weight's.  Bound by the matrix cores' power:
// the largest tile, four waves of 128 x 128 each, reads the least from L2 and LDS for a product,
// which leaves the clock highest.  8192 x 2048 x 11008 575 us (1.29 PFLOP/s), with SAVE 663: the
// 256 KB that a tile then writes leave at its end and overlap nothing, as a tile fills its CU.
// 16384 x 5120 x 17408 4240 us (1.38 PFLOP/s), with SAVE 4560.
template <typename Tile, bool F32, bool SAVE>
__global__ __launch_bounds__(Tile::kThreads, Tile::kWavesPerSimd) void k_gated_forward(ForwardArgs g)
{
    __shared__ __align__(1024) uint8_t lds[Tile::kLdsBytes];
    constexpr int kCols = Tile::kCols / 2;
    const TilePlace at = tile_place(int(unit_of_workgroup(Tile::kRun)),
                                    int((g.m + Tile::kRows - 1) / Tile::kRows),
                                    int((g.n + kCols - 1) / kCols));
    const int64_t r0 = int64_t(at.row) * Tile::kRows, c0 = int64_t(at.col) * kCols;
    const int first = int(blockIdx.y) * g.slice, steps = min(g.slice, g.steps - first);
    Tile tile;
    Bf16<Tile::kPinned> mul;
    const int64_t k0 = int64_t(first) * kStepBytes;
    product_pairs(mul, tile, g.x + r0 * g.x_pitch + k0, g.x_pitch, g.m - r0,
                  g.gate + c0 * g.gate_pitch + k0, g.gate_pitch, g.up + c0 * g.up_pitch + k0,
                  g.up_pitch, g.n - c0, steps, lds);
    ForwardWriter<F32, SAVE> w{g, r0, c0};
    finish_pairs(tile, lds, w);
}

// Results of the slices' sums, added in their order, four loads under way at once; with SAVE what the
// backward pass needs of them is kept here (the tiles of a cut sum keep nothing).  Bound by
// latency: 64 x 2048 from eight slices 4.0 us, a token's 5120 from sixteen 5.1 (one after the other
// 7.4).
template <bool F32, bool SAVE>
__global__ __launch_bounds__(256) void k_gated_answer(ForwardArgs g, int slices)
{
    const int64_t all = g.m * g.n;
    for (int64_t e = int64_t(blockIdx.x) * 256 + threadIdx.x; e < all;
         e += int64_t(gridDim.x) * 256) {
        float u = g.partial[e], v = g.partial[all + e];
#pragma unroll 4
        for (int i = 1; i < slices; ++i) {
            u += g.partial[2 * i * all + e];
            v += g.partial[(2 * i + 1) * all + e];
        }
        const int64_t row = e / g.n, col = e % g.n, to = row * g.stride + col;
        const float h = answer_one<SAVE>(g.saved, g.activation, row, col, u, v);
        if constexpr (F32)
            static_cast<float*>(g.out)[to] = h;
        else
            static_cast<uint16_t*>(g.out)[to] = gated::bf16_bits(h);
    }
}

// ------------------------------------------------------------- few tokens

struct FewArgs {
    const uint8_t* w[2];    // rows of k values
    int64_t w_pitch[2];     // bytes
    const uint8_t* x;
    int64_t x_pitch;
    int64_t m, n;
    int64_t bytes;          // of a row's values
    int activation;
    void* out;
    int64_t stride;
    Saved saved;
};

// 32 bytes of a row from byte `at` on; what lies behind its end is 0.
__device__ inline void few_load(const uint8_t* row, int64_t at, int64_t bytes, i32x4 (&v)[2])
{
    if (at + 32 <= bytes) {
        v[0] = load_any(row + at);
        v[1] = load_any(row + at + 16);
        return;
    }
#pragma unroll
    for (int c = 0; c < 2; ++c)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int64_t i = at + 16 * c + 4 * e;
            const auto* p = reinterpret_cast<const uint16_t*>(row + i);
            const uint32_t lo = i < bytes ? p[0] : 0u, hi = i + 2 < bytes ? p[1] : 0u;
            v[c][e] = int(lo | hi << 16);
        }
}

// Results for up to 16 tokens, 16 rows of both weights to a workgroup, bound by reading the weights
// once: no LDS tiles, every lane loads its bytes of the instruction's rows straight from HBM, and
// the waves cut the sum into runs of neighbouring steps.  An instruction is 16 rows x 16 tokens: a
// lane holds 16 bytes of row and token l % 16, and ends with rows 4 (l / 16) + e of token l % 16.
// One token through 2048 x 11008 16.9 us, 5.4 TB/s; 16 tokens 23.
template <bool F32, bool SAVE>
__global__ __launch_bounds__(512) void k_few(FewArgs g)
{
    extern __shared__ f32x4 few_sums[];  // [wave][B][lane], of 16 bytes
    constexpr int B = 2;
    const int lane = int(threadIdx.x) & 63, r = lane & 15, q = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x) >> 6);
    const int waves = int(blockDim.x) >> 6;
    const int64_t n0 = int64_t(blockIdx.x) * 16;
    const uint8_t* w[B];
#pragma unroll
    for (int b = 0; b < B; ++b) {
        const int64_t row = n0 + r < g.n ? n0 + r : g.n - 1;
        w[b] = g.w[b] + row * g.w_pitch[b];
    }
    const uint8_t* x = g.x + (r < g.m ? r : g.m - 1) * g.x_pitch;
    f32x4 acc[B] = {};
    struct Loaded {
        i32x4 w[B][2], x[2];
    };
    const auto load = [&](int s, Loaded& in) {
        const int64_t at = int64_t(s) * kStepBytes + 32 * q;
#pragma unroll
        for (int b = 0; b < B; ++b)
            few_load(w[b], at, g.bytes, in.w[b]);
        few_load(x, at, g.bytes, in.x);
    };
    const auto multiply = [&](const Loaded& in) {
#pragma unroll
        for (int c = 0; c < 2; ++c)
#pragma unroll
            for (int b = 0; b < B; ++b)
                acc[b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                    __builtin_bit_cast(bf16x8, in.w[b][c]),
                    __builtin_bit_cast(bf16x8, in.x[c]), acc[b], 0, 0, 0);
    };
    const int steps = int((g.bytes + kStepBytes - 1) / kStepBytes);
    const int first = steps * wave / waves, last = steps * (wave + 1) / waves;
    if (first < last) {
        Loaded even, odd;
        load(first, even);
        int s = first;
        for (; s + 1 < last; s += 2) {
            load(s + 1, odd);
            multiply(even);
            if (s + 2 < last)
                load(s + 2, even);
            multiply(odd);
        }
        if (s < last)
            multiply(even);
    }
#pragma unroll
    for (int b = 0; b < B; ++b)
        few_sums[(wave * B + b) * 64 + lane] = acc[b];
    __syncthreads();
    // the waves' sums, added in their order
    const float* sums = reinterpret_cast<const float*>(few_sums);
    const int e = int(threadIdx.x), l = e / 4;
    const int64_t row = n0 + 4 * (l >> 4) + e % 4, tok = l & 15;
    if (e >= 256 || row >= g.n || tok >= g.m)
        return;
    float v[B];
#pragma unroll
    for (int b = 0; b < B; ++b) {
        const float* from = sums + b * 256 + e;
        v[b] = from[0];
        for (int i = 1; i < waves; ++i)
            v[b] += from[i * B * 256];
    }
    const float y = answer_one<SAVE>(g.saved, g.activation, tok, row, v[0], v[1]);
    if constexpr (F32)
        static_cast<float*>(g.out)[tok * g.stride + row] = y;
    else
        static_cast<uint16_t*>(g.out)[tok * g.stride + row] = gated::bf16_bits(y);
}

void launch_few(const FewArgs& g, bool f32, bool save, hipStream_t st)
{
    const int64_t steps = (g.bytes + kStepBytes - 1) / kStepBytes;
    const int waves = steps >= 8 ? 8 : 4;
    auto* kernel = save ? (f32 ? k_few<true, true> : k_few<false, true>)
                        : (f32 ? k_few<true, false> : k_few<false, false>);
    kernel<<<dim3(uint32_t((g.n + 15) / 16)), 64 * waves, size_t(waves) * 2 * 1024, st>>>(g);
}

// ------------------------------------------------------------- the backward pass

// dg and du as the products read them, next to each other in rows of 2 * half values: zeros in
// columns from n up to half, and in rows from m up to whole steps.  In bf16, the matrix cores'
// operands: this rounding, half a step of each, is as large as that of a gradient in bf16.  The
// gradients of 8192 x 2048 x 11008 lie 0.0023 from 64 bits (2-norm, relative), without it 0.0017.  A
// second operand with what it leaves would double the products, four fifths of the backward pass's
// time and more.
struct SlopeArgs {
    const void* dh;
    int64_t stride;
    Saved saved;
    int64_t m, n;
    uint16_t* out;
    int64_t half, rows;
    Layouts copies;      // what the products read besides, by the workgroups behind
    uint32_t own;        // workgroups before those
};

// Eight channels of a token to a lane.  Bound by HBM: 8 bytes read and 4 written a value, 205 to
// 212 us for 8192 x 11008 values (5.2 TB/s), 620 for 16384 x 17408 (5.5 TB/s).
template <bool F32>
__global__ __launch_bounds__(256) void k_gated_slopes(SlopeArgs g)
{
    if (blockIdx.x >= g.own) {
        pack(g.copies, blockIdx.x - g.own);
        return;
    }
    const int64_t lines = g.half / 8, all = g.rows * lines;
    const int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x;
    if (i >= all)
        return;
    const int64_t row = i / lines, col = i % lines * 8;
    u16x8 dg = {}, du = {};
    if (row < g.m && col < g.n) {
        float a[8], b[8], d[8];
        load_eight(g.saved.a_high, g.saved.a_low, row * g.saved.pitch + col, a);
        load_eight(g.saved.b_high, g.saved.b_low, row * g.saved.pitch + col, b);
        const int64_t from = row * g.stride + col;
        if (col + 8 <= g.n) {
            if constexpr (F32) {
                const auto* p = static_cast<const float*>(g.dh) + from;
                const f32x4 lo = __builtin_bit_cast(f32x4, load_any(p));
                const f32x4 hi = __builtin_bit_cast(f32x4, load_any(p + 4));
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    d[e] = lo[e];
                    d[4 + e] = hi[e];
                }
            } else {
                const i32x4 w = load_any(static_cast<const uint16_t*>(g.dh) + from);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    d[2 * e] = __uint_as_float(uint32_t(w[e]) << 16);
                    d[2 * e + 1] = __uint_as_float(uint32_t(w[e]) & 0xFFFF0000u);
                }
            }
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                d[e] = 0.0f;
                if (col + e < g.n) {
                    if constexpr (F32)
                        d[e] = static_cast<const float*>(g.dh)[from + e];
                    else
                        d[e] = __uint_as_float(
                            uint32_t(static_cast<const uint16_t*>(g.dh)[from + e]) << 16);
                }
            }
        }
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (col + e < g.n) {  // what is kept behind a row's end is anything
                dg[e] = gated::bf16_bits(d[e] * a[e]);
                du[e] = gated::bf16_bits(d[e] * b[e]);
            }
    }
    uint16_t* to = g.out + row * 2 * g.half + col;
    *reinterpret_cast<i32x4*>(to) = __builtin_bit_cast(i32x4, dg);
    *reinterpret_cast<i32x4*>(to + g.half) = __builtin_bit_cast(i32x4, du);
}

// dx = [dg | du] [gate; up], or dgate = dg^T x and dup = du^T x.  No operand is turned in memory:
// what has the summed index as rows is turned on its way out of LDS.  Bound by the matrix cores'
// power (they work 73% of the cycles for dx at 1.83 GHz, 71% at 1.82 for the weights) and by what
// L2 feeds a CU, 23.5 of some 26 bytes a cycle.  16384 x 5120 x 17408: dx 4.03 to 4.22 ms, the
// weights' 4.15 to 4.41 (1.32 to 1.45 PFLOP/s, by the card); 8192 x 2048 x 11008, all in one
// launch, 1.07 to 1.27.
struct ProductArgs {
    const uint8_t* a;    // dg and du by rows
    int64_t a_pitch;     // bytes
    TurnedSource b;      // the weights, or x
    int64_t b_cols;      // a multiple of 8
    int64_t m, n;        // of one result
    int count;           // results
    int steps, slice, slices;
    void* out[2];
    int64_t stride[2];
    int f32;
    float* partial;      // several slices: [slice][count][m][n]
    uint32_t tiles;      // of a slice
};

// Both in one launch: neither needs the other, and the workgroups of one fill the CUs that the
// other leaves.
struct ProductsArgs {
    ProductArgs dx, dw;
    uint32_t dx_first, dw_first, dx_end, dw_end;  // workgroups
};

struct ProductWriter {
    static constexpr bool kTurned = false;
    static constexpr int kSlots = 8;
    void* out;
    int64_t stride, rows, cols;  // from the tile's origin on
    bool f32;
    __device__ inline void fetch(int, int, int) {}
    __device__ inline void turn(int, int, const float (&)[8]) {}
    __device__ inline void store(int row, int col, float (&v)[8], int)
    {
        if (row >= rows || col >= cols)
            return;
        if (f32)
            store_row<true>(out, row * stride + col, v, cols - col);
        else
            store_row<false>(out, row * stride + col, v, cols - col);
    }
};

template <typename Tile, bool DW>
__device__ inline void gated_product(const ProductArgs& g, uint32_t group, uint8_t* lds)
{
    const int down = int((g.m + Tile::kRows - 1) / Tile::kRows);
    const int across = int((g.n + Tile::kCols - 1) / Tile::kCols);
    const int part = int(group / g.tiles);
    const int64_t unit = unit_of_workgroup(group % g.tiles, g.tiles, Tile::kRun);
    const int which = unit >= int64_t(down) * across ? 1 : 0;
    const TilePlace at = tile_place(int(unit - int64_t(which) * down * across), down, across);
    const int64_t r0 = int64_t(at.row) * Tile::kRows, c0 = int64_t(at.col) * Tile::kCols;
    const int first = part * g.slice, steps = min(g.slice, g.steps - first);
    Tile tile;
    Bf16<Tile::kPinned> mul;
    TurnedOperand<Tile, Tile::kCols, Tile::J> q;
    q.src = g.b;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        q.src.base[i] += c0 * 2;
        q.src.tail[i] += c0 * 2;
    }
    q.first = first;
    q.steps = steps;
    q.init(g.b_cols - c0);
    if constexpr (DW) {
        const int64_t half = g.a_pitch / 4;  // columns of either
        TurnedOperand<Tile, Tile::kRows, Tile::I> p;
        p.src.base[0] = p.src.base[1] = g.a + (which * half + r0) * 2;
        p.src.tail[0] = p.src.tail[1] = p.src.base[0];
        p.src.pitch = g.a_pitch;
        p.src.each = p.src.full = g.steps;
        p.first = first;
        p.steps = steps;
        p.init(half - r0);
        product(mul, tile, p, q, steps, lds);
    } else {
        RowOperand<Tile, Tile::kRows, Tile::I, TileLoad<Tile::kRows, Tile::kThreads, true>> p;
        p.src = g.a + r0 * g.a_pitch + int64_t(first) * kStepBytes;
        p.steps = steps;
        p.load.init(g.a_pitch, g.m - r0);
        product(mul, tile, p, q, steps, lds);
    }
    ProductWriter w;
    w.rows = g.m - r0;
    w.cols = g.n - c0;
    w.stride = g.partial ? g.n : which ? g.stride[1] : g.stride[0];
    w.f32 = g.partial || g.f32;
    const int64_t to = r0 * w.stride + c0;
    if (g.partial)
        w.out = g.partial + (int64_t(part) * g.count + which) * g.m * g.n + to;
    else
        w.out = static_cast<uint8_t*>(which ? g.out[1] : g.out[0]) + to * (g.f32 ? 4 : 2);
    finish(tile, lds, w);
}

template <typename Tile>
__global__ __launch_bounds__(Tile::kThreads, Tile::kWavesPerSimd) void k_gated_products(
    ProductsArgs g)
{
    __shared__ __align__(1024) uint8_t lds[Tile::kLdsBytes];
    if (blockIdx.x >= g.dx_first && blockIdx.x < g.dx_end)
        gated_product<Tile, false>(g.dx, blockIdx.x - g.dx_first, lds);
    else
        gated_product<Tile, true>(g.dw, blockIdx.x - g.dw_first, lds);
}

// out = the slices' sums, added in their order.
__global__ __launch_bounds__(256) void k_gated_join(ProductArgs g)
{
    const int64_t one = g.m * g.n, all = one * g.count;
    for (int64_t e = int64_t(blockIdx.x) * 256 + threadIdx.x; e < all;
         e += int64_t(gridDim.x) * 256) {
        float s = g.partial[e];
        for (int i = 1; i < g.slices; ++i)
            s += g.partial[i * all + e];
        const int which = e >= one ? 1 : 0;
        const int64_t i = e - which * one;
        const int64_t to = i / g.n * (which ? g.stride[1] : g.stride[0]) + i % g.n;
        void* out = which ? g.out[1] : g.out[0];
        if (g.f32)
            static_cast<float*>(out)[to] = s;
        else
            static_cast<uint16_t*>(out)[to] = gated::bf16_bits(s);
    }
}

// ---------------------------------------------------------------- host side

// Dimensions and strides stay within the 32-bit offsets of a tile's loads: 256 rows of 2^23 bytes.
constexpr int64_t kMost = int64_t(1) << 21;
constexpr int64_t kMostGroups = int64_t(1) << 24;  // a grid counts threads in 32 bits

using gated::Way;
using gated::way_of;

bool valid_sizes(int64_t m, int64_t n, int64_t k)
{
    const auto tiles = [](int64_t a, int64_t b) {
        return host::ceil_div(a, 64) * host::ceil_div(b, 64) < kMostGroups / 4;
    };
    return m >= 0 && n >= 0 && k >= 0 && m < kMost && n < kMost && k < kMost && tiles(m, n) &&
           tiles(m, k) && tiles(n, k);
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

// Whether the tiles can read rows of k values, `stride` apart, as they are.
bool readable(int64_t k, int64_t stride) { return k % kStep == 0 && stride % 8 == 0 && stride < 2 * kMost; }

int64_t take(int64_t& at, int64_t bytes)
{
    const int64_t from = at;
    at += int64_t(host::round_up(size_t(bytes), 256));
    return from;
}

struct ForwardLayout {
    int64_t x = -1, gate = -1, up = -1;  // of packed copies
    int64_t partial = -1;                // of the slices' sums
    Way way;
    bool few = false;  // no tiles, and no workspace
    int64_t total = 0;
};

ForwardLayout forward_layout(int64_t m, int64_t n, int64_t k, int64_t x_stride,
                             int64_t gate_stride, int64_t up_stride)
{
    ForwardLayout l;
    const int64_t pitch = padded(k) * 2;
    const bool copy_x = !readable(k, x_stride), copy_gate = !readable(k, gate_stride),
               copy_up = !readable(k, up_stride);
    // tiles read a long sum faster, in slices (a token through 5120 x 2048 32 us and 26, through
    // 11008 x 2048 29 and 23; through 2048 x 11008 21 and 27), but not what has to be copied first.
    // Whether results are kept makes no difference here: h has the same bits either way
    l.few = m <= gated::kFewTokens && (k <= 4096 || copy_x || copy_gate || copy_up);
    if (l.few) {
        l.total = host::kNoWorkspace;
        return l;
    }
    if (copy_x)
        l.x = take(l.total, m * pitch);
    if (copy_gate)
        l.gate = take(l.total, n * pitch);
    if (copy_up)
        l.up = take(l.total, n * pitch);
    l.way = way_of(m, n, int(padded(k) / kStep), true);
    if (l.way.slices > 1)
        l.partial = take(l.total, l.way.slices * m * n * 8);
    l.total = host::workspace_for(l.total);
    return l;
}

// Whether the tiles can turn a matrix with rows of k values as it is: whole lines of 16 bytes, and
// rows near enough that a copy of the last ones at that distance is small.
bool turnable(int64_t k, int64_t stride)
{
    return k % 8 == 0 && stride % 8 == 0 && stride <= 4 * k + 64 && stride < 2 * kMost;
}

// A matrix that the backward products turn: as it is, with the rows behind the last whole step
// copied at the same distance, or copied as a whole.
struct TurnedPlace {
    int64_t at = -1;  // of the copy, none if negative
    int64_t rows = 0, from = 0;  // that are copied, and the first of them
    int64_t out_rows = 0, pitch = 0;
    bool whole = false;
};

TurnedPlace turned_place(int64_t& total, int64_t rows, int64_t k, int64_t stride, bool as_it_is)
{
    TurnedPlace p;
    if (as_it_is && rows % kStep == 0)
        return p;
    p.whole = !as_it_is;
    p.from = as_it_is ? rows / kStep * kStep : 0;
    p.rows = rows - p.from;
    p.out_rows = padded(p.rows);
    p.pitch = as_it_is ? stride : padded(k);
    p.at = take(total, p.out_rows * p.pitch * 2);
    return p;
}

// What a tile of these products costs, in microseconds: a step where every CU is busy and where
// it has the CU to itself (the smaller tiles wait for their operands then), and beside its steps.
struct TurnedCost {
    int tile;
    double step, alone, rest;
};

constexpr TurnedCost kTurnedCosts[] = {
    {256, 1.83, 1.83, 7.8}, {128, 0.67, 0.95, 2.0}, {64, 0.25, 0.53, 0.83}};

// A matrix product of the backward pass, as its launch is planned: `count` results of m x n.
struct Plan {
    int64_t m = 0, n = 0, count = 0;
    int steps = 0, slice = 0, slices = 1;
    double alone(const TurnedCost& c) const { return c.alone * slice + c.rest; }
    double busy(const TurnedCost& c) const { return c.step * slice + c.rest; }
    int64_t tiles(const TurnedCost& c) const
    {
        return host::ceil_div(m, c.tile) * host::ceil_div(n, c.tile) * count;
    }
    // what the tiles read
    double bytes(const TurnedCost& c) const
    {
        return double(count) * steps * kStepBytes *
               (double(m) * double(host::ceil_div(n, c.tile)) +
                double(n) * double(host::ceil_div(m, c.tile)));
    }
    int64_t partial() const { return slices > 1 ? slices * count * m * n * 4 : 0; }
    bool cut(int z)  // into z slices, if they are that many and long enough
    {
        slice = int(host::ceil_div(steps, z));
        slices = z;
        return z == 1 || (slice >= 8 && host::ceil_div(steps, slice) == z && partial() < 270000000);
    }
};

// The tile of a launch with one or both, and their slices, by expected time: the longest tile, or
// all tiles' work shared by the CUs and the last tiles, which leave some idle; what they read, at
// 26 TB/s out of L2 and behind it; another launch for the sums of slices, and those to memory and
// back (2.5 TB/s).  Fitted to 190 passes of 64 to 12288 tokens through 64 x 64 to 5120 x 17408, each
// by all tiles and up to 32 slices: 0.7% from the best on average and 17% at most.
int plan(Plan* dx, Plan* dw)
{
    struct Choice {
        Plan plan;
        double alone, busy, work, sums;
        int64_t tiles;
    };
    const int cuts[] = {1, 2, 3, 4, 6, 8, 12, 16, 24, 32, 48, 64};
    constexpr int kCuts = sizeof(cuts) / sizeof(cuts[0]);
    const auto choices = [&](const Plan* of, const TurnedCost& c, Choice (&to)[kCuts]) {
        if (!of) {
            to[0] = Choice{};
            return 1;
        }
        int n = 0;
        for (const int z : cuts) {
            Plan p = *of;
            if (!p.cut(z))
                continue;
            const int64_t tiles = p.tiles(c) * p.slices;
            to[n++] = {p, p.alone(c), p.busy(c), tiles * p.busy(c) / 256,
                       p.slices > 1 ? 3.8 + 2.0 * double(p.partial()) / 2.5e6 : 0.0, tiles};
        }
        return n;
    };
    int best = 64;
    double least = 1e300;
    Plan one, other;
    Choice xs[kCuts], ws[kCuts];
    for (const TurnedCost& c : kTurnedCosts) {
        const double read = (dx ? dx->bytes(c) : 0.0) + (dw ? dw->bytes(c) : 0.0);
        const int nx = choices(dx, c, xs), nw = choices(dw, c, ws);
        for (int i = 0; i < nx; ++i)
            for (int j = 0; j < nw; ++j) {
                const Choice &x = xs[i], &w = ws[j];
                double us = std::max(x.alone, w.alone);
                if (x.tiles + w.tiles > 256) {
                    const double last = dx && dw ? std::min(x.busy, w.busy)
                                                 : std::max(x.busy, w.busy);
                    us = std::max(us, x.work + w.work + 0.97 * last);
                }
                us += read / 26e6 + x.sums + w.sums;
                if (us < least) {
                    least = us;
                    best = c.tile;
                    one = x.plan;
                    other = w.plan;
                }
            }
    }
    if (dx)
        *dx = one;
    if (dw)
        *dw = other;
    return best;
}

struct BackwardLayout {
    int64_t slopes = -1, dx_sums = -1, dw_sums = -1;
    TurnedPlace gate, up, x;
    int64_t total = 0;
    Plan dx, dw;
    int tile = 0;
};

BackwardLayout backward_layout(int64_t m, int64_t n, int64_t k, int64_t x_stride,
                               int64_t gate_stride, int64_t up_stride, bool dx, bool dw)
{
    BackwardLayout l;
    l.slopes = take(l.total, padded(m) * 2 * padded(n) * 2);
    if (dx) {
        const bool as_it_is = turnable(k, gate_stride) && gate_stride == up_stride;
        l.gate = turned_place(l.total, n, k, gate_stride, as_it_is);
        l.up = turned_place(l.total, n, k, up_stride, as_it_is);
        l.dx = Plan{m, k, 1, int(2 * padded(n) / kStep)};
    }
    if (dw) {
        l.x = turned_place(l.total, m, k, x_stride, turnable(k, x_stride));
        l.dw = Plan{n, k, 2, int(padded(m) / kStep)};
    }
    l.tile = plan(dx ? &l.dx : nullptr, dw ? &l.dw : nullptr);
    if (l.dx.partial())
        l.dx_sums = take(l.total, l.dx.partial());
    if (l.dw.partial())
        l.dw_sums = take(l.total, l.dw.partial());
    l.total = std::max<int64_t>(l.total, 256);
    return l;
}

uint32_t groups_for(int64_t work) { return uint32_t(std::min<int64_t>(host::ceil_div(work, 256), 8192)); }

// The copies of one launch.
struct Copies {
    Layouts of{};
    int64_t groups = 0;

    void add(const void* x, int64_t rows, int64_t cols, int64_t stride, uint8_t* out,
             int64_t out_rows, int64_t pitch)
    {
        of.of[of.count++] = Layout{static_cast<const uint16_t*>(x),
                                   rows,
                                   cols,
                                   stride,
                                   reinterpret_cast<uint16_t*>(out),
                                   out_rows,
                                   pitch,
                                   uint32_t(groups)};
        groups += host::ceil_div(out_rows * (pitch / 8), kPackLines);
    }
    void launch(hipStream_t st) const
    {
        if (of.count > 0)
            k_gated_pack<<<dim3(uint32_t(groups)), 256, 0, st>>>(of);
    }
};

// Where the products find a matrix that they turn, its copy added to the launch; k columns.
void turned_operand(const TurnedPlace& p, const void* x, int64_t rows, int64_t k, int64_t stride,
                    uint8_t* ws, Copies& copies, TurnedSource* to, int which)
{
    const auto* base = static_cast<const uint8_t*>(x);
    const uint8_t* copy = p.at < 0 ? base : ws + p.at;
    if (p.at >= 0)
        copies.add(base + p.from * stride * 2, p.rows, k, stride, ws + p.at, p.out_rows, p.pitch);
    to->base[which] = p.whole ? copy : base;
    to->tail[which] = copy;
    to->pitch = (p.whole ? p.pitch : stride) * 2;
    to->each = int(padded(rows) / kStep);
    to->full = p.whole ? to->each : int(rows / kStep);
}

template <typename Tile>
void launch_forward(const ForwardArgs& g, int slices, bool f32, bool save, hipStream_t st)
{
    auto* kernel = save ? (f32 ? k_gated_forward<Tile, true, true>
                               : k_gated_forward<Tile, false, true>)
                        : (f32 ? k_gated_forward<Tile, true, false>
                               : k_gated_forward<Tile, false, false>);
    const dim3 grid(uint32_t(host::ceil_div(g.m, Tile::kRows) *
                             host::ceil_div(g.n, Tile::kCols / 2)),
                    uint32_t(slices));
    kernel<<<grid, Tile::kThreads, 0, st>>>(g);
}

// The products that are planned, the one with the longer tiles first.
template <typename Tile>
void launch_products(ProductsArgs g, bool dx, bool dw, hipStream_t st)
{
    const auto groups = [](ProductArgs& p) {
        p.tiles = uint32_t(host::ceil_div(p.m, Tile::kRows) * host::ceil_div(p.n, Tile::kCols) *
                           p.count);
        return p.tiles * uint32_t(p.slices);
    };
    const uint32_t nx = dx ? groups(g.dx) : 0, nw = dw ? groups(g.dw) : 0;
    const bool dx_first = !dw || (dx && g.dx.slice >= g.dw.slice);
    g.dx_first = dx_first ? 0 : nw;
    g.dw_first = dx_first ? nx : 0;
    const auto launch = [&](uint32_t x, uint32_t w) {
        g.dx_end = g.dx_first + x;
        g.dw_end = g.dw_first + w;
        k_gated_products<Tile><<<dim3(x + w), Tile::kThreads, 0, st>>>(g);
    };
    if (nx >= 1024 && nw >= 1024) {
        // rounds enough to fill the chip alone, where the two would share its L2 for a while: 16384
        // tokens through 5120 x 17408 8.78 ms, in one launch 8.86
        g.dx_first = g.dw_first = 0;
        launch(nx, 0);
        launch(0, nw);
    } else {
        launch(nx, nw);
    }
    for (const ProductArgs* p : {&g.dx, &g.dw})
        if (p->partial)
            k_gated_join<<<dim3(groups_for(p->m * p->n * p->count)), 256, 0, st>>>(*p);
}

// The planned part of a product's arguments.
ProductArgs planned(const Plan& p, uint8_t* partial)
{
    ProductArgs g{};
    g.m = p.m;
    g.n = p.n;
    g.count = int(p.count);
    g.steps = p.steps;
    g.slice = p.slice;
    g.slices = p.slices;
    g.partial = reinterpret_cast<float*>(partial);
    return g;
}

struct Read {
    const void* p;
    size_t bytes;
};

}  // namespace

namespace host {

lt_err launch_zero(void* out, int item, int64_t m, int64_t n, int64_t stride, hipStream_t st)
{
    const ZeroArgs a{out, m, n, stride};
    if (item == 1)
        k_zero_rows<uint8_t><<<dim3(groups_for(m * n)), 256, 0, st>>>(a);
    else if (item == 2)
        k_zero_rows<uint16_t><<<dim3(groups_for(m * n)), 256, 0, st>>>(a);
    else
        k_zero_rows<uint32_t><<<dim3(groups_for(m * n)), 256, 0, st>>>(a);
    LT_TRY_HIP(hipGetLastError());
    return LT_OK;
}

}  // namespace host

extern "C" {

size_t lt_gated_saved_bytes(int64_t m, int64_t n)
{
    if (m < 0 || n < 0 || m >= kMost || n >= kMost)
        return 0;
    return size_t(m) * size_t(host::ceil_div(n, 8) * 8) * 6;
}

size_t lt_gated_forward_workspace_bytes(int64_t m, int64_t n, int64_t k, int64_t x_stride,
                                        int64_t gate_stride, int64_t up_stride)
{
    if (!valid_sizes(m, n, k))
        return 0;
    return size_t(forward_layout(m, n, k, x_stride, gate_stride, up_stride).total);
}

lt_err lt_gated_forward(const void* x, int64_t x_stride, const void* gate, int64_t gate_stride,
                        const void* up, int64_t up_stride, int activation, int64_t m, int64_t n,
                        int64_t k, void* out, int out_dtype, int64_t out_stride, void* saved,
                        void* workspace, size_t workspace_bytes, void* stream)
try {
    host::clear_error();
    if (!valid_sizes(m, n, k) || !valid_stride(m, n, out_stride) || !valid_stride(m, k, x_stride) ||
        !valid_stride(n, k, gate_stride) || !valid_stride(n, k, up_stride))
        return fail(LT_ERR_INVALID_ARG, "need 0 <= m, n, k < 2^21, fewer than 2^22 tiles of 64 x 64 "
                                        "in each matrix, and strides of a row's length or more");
    if (!valid_dtype(out_dtype))
        return fail(LT_ERR_INVALID_ARG, "out_dtype must be LT_DTYPE_F32 or LT_DTYPE_BF16");
    if (activation < LT_ACT_SILU || activation > LT_ACT_RELU)
        return fail(LT_ERR_INVALID_ARG, "unknown activation");
    if (m == 0 || n == 0)
        return LT_OK;
    if (!out || (k > 0 && (!x || !gate || !up)))
        return fail(LT_ERR_INVALID_ARG, "x, the weights and out must not be NULL");
    if (!host::aligned(x, 16) || !host::aligned(gate, 16) || !host::aligned(up, 16) ||
        !host::aligned(out, 16) || !host::aligned(saved, 16))
        return fail(LT_ERR_ALIGNMENT, "x, the weights, out and saved must be 16-byte aligned");
    const hipStream_t st = static_cast<hipStream_t>(stream);
    const size_t out_bytes = span_bytes(m, n, out_stride, out_dtype);
    const size_t saved_bytes = saved ? lt_gated_saved_bytes(m, n) : 0;
    const ForwardLayout l = forward_layout(m, n, k, x_stride, gate_stride, up_stride);
    const bool works =
        k > 0 && (l.x >= 0 || l.gate >= 0 || l.up >= 0 || l.partial >= 0);
    if (works && (!workspace || !host::aligned(workspace, 256) || workspace_bytes < size_t(l.total)))
        return fail(LT_ERR_WORKSPACE, "workspace must be 256-byte aligned and hold " +
                                          std::to_string(l.total) + " bytes");
    const size_t ws_bytes = works ? size_t(l.total) : 0;
    const Read read[] = {{x, span_bytes(m, k, x_stride, LT_DTYPE_BF16)},
                         {gate, span_bytes(n, k, gate_stride, LT_DTYPE_BF16)},
                         {up, span_bytes(n, k, up_stride, LT_DTYPE_BF16)}};
    for (const Read& r : read)
        if (host::overlaps(out, out_bytes, r.p, r.bytes) ||
            host::overlaps(saved, saved_bytes, r.p, r.bytes) ||
            host::overlaps(workspace, ws_bytes, r.p, r.bytes))
            return fail(LT_ERR_INVALID_ARG, "an array that is written overlaps x or a weight");
    if (host::overlaps(out, out_bytes, saved, saved_bytes) ||
        host::overlaps(out, out_bytes, workspace, ws_bytes) ||
        host::overlaps(saved, saved_bytes, workspace, ws_bytes))
        return fail(LT_ERR_INVALID_ARG, "out, saved and the workspace overlap");
    if (k == 0) {  // empty sums: act(0) * 0, and a = b = 0
        if (saved)
            if (lt_err e = host::launch_zero(saved, 1, 1, int64_t(saved_bytes), int64_t(saved_bytes),
                                             st))
                return e;
        return host::launch_zero(out, out_dtype == LT_DTYPE_F32 ? 4 : 2, m, n, out_stride, st);
    }
    const bool f32 = out_dtype == LT_DTYPE_F32;
    if (l.few) {
        FewArgs f{};
        f.w[0] = static_cast<const uint8_t*>(gate);
        f.w[1] = static_cast<const uint8_t*>(up);
        f.w_pitch[0] = gate_stride * 2;
        f.w_pitch[1] = up_stride * 2;
        f.x = static_cast<const uint8_t*>(x);
        f.x_pitch = x_stride * 2;
        f.m = m;
        f.n = n;
        f.bytes = k * 2;
        f.activation = activation;
        f.out = out;
        f.stride = out_stride;
        if (saved)
            f.saved = saved_layout(saved, m, n);
        launch_few(f, f32, saved != nullptr, st);
        LT_TRY_HIP(hipGetLastError());
        return LT_OK;
    }
    auto* ws = static_cast<uint8_t*>(workspace);
    if (works)
        if (lt_err e = host::workspace_written(ws, ws_bytes, st))
            return e;
    ForwardArgs g{};
    g.steps = int(padded(k) / kStep);
    g.m = m;
    g.n = n;
    g.activation = activation;
    g.out = out;
    g.stride = out_stride;
    if (saved)
        g.saved = saved_layout(saved, m, n);
    Copies copies;
    const auto operand = [&](const void* p, int64_t rows, int64_t stride, int64_t at,
                             const uint8_t** from, int64_t* pitch) {
        *from = static_cast<const uint8_t*>(p);
        *pitch = stride * 2;
        if (at < 0)
            return;
        copies.add(p, rows, k, stride, ws + at, rows, padded(k));
        *from = ws + at;
        *pitch = padded(k) * 2;
    };
    operand(x, m, x_stride, l.x, &g.x, &g.x_pitch);
    operand(gate, n, gate_stride, l.gate, &g.gate, &g.gate_pitch);
    operand(up, n, up_stride, l.up, &g.up, &g.up_pitch);
    copies.launch(st);
    g.slice = l.way.slice;
    if (l.partial >= 0)
        g.partial = reinterpret_cast<float*>(ws + l.partial);
    const bool keeps = saved && !g.partial;  // a cut sum's results are the last launch's
    if (l.way.tile == 256)
        launch_forward<Large16>(g, l.way.slices, f32, keeps, st);
    else if (l.way.tile == 128)
        launch_forward<Small16>(g, l.way.slices, f32, keeps, st);
    else
        launch_forward<Pair16>(g, l.way.slices, f32, keeps, st);
    if (g.partial) {
        auto* answer = saved ? (f32 ? k_gated_answer<true, true> : k_gated_answer<false, true>)
                             : (f32 ? k_gated_answer<true, false> : k_gated_answer<false, false>);
        answer<<<dim3(uint32_t(std::min<int64_t>(4096, host::ceil_div(m * n, 256)))), 256, 0, st>>>(
            g, l.way.slices);
    }
    LT_TRY_HIP(hipGetLastError());
    return LT_OK;
} catch (...) {
    return host::caught();
}

size_t lt_gated_backward_workspace_bytes(int64_t m, int64_t n, int64_t k, int64_t x_stride,
                                         int64_t gate_stride, int64_t up_stride, int dx, int dw)
{
    if (!valid_sizes(m, n, k))
        return 0;
    return size_t(
        backward_layout(m, n, k, x_stride, gate_stride, up_stride, dx != 0, dw != 0).total);
}

lt_err lt_gated_backward(const void* dh, int dh_dtype, int64_t dh_stride, const void* saved,
                         const void* x, int64_t x_stride, const void* gate, int64_t gate_stride,
                         const void* up, int64_t up_stride, int64_t m, int64_t n, int64_t k,
                         void* dx, int dx_dtype, int64_t dx_stride, void* dgate,
                         int64_t dgate_stride, void* dup, int64_t dup_stride, int grad_dtype,
                         void* workspace, size_t workspace_bytes, void* stream)
try {
    host::clear_error();
    const bool want_dw = dgate || dup;
    if (!valid_sizes(m, n, k) || !valid_stride(m, n, dh_stride) ||
        (want_dw && (!valid_stride(m, k, x_stride) || !valid_stride(n, k, dgate_stride) ||
                     !valid_stride(n, k, dup_stride))) ||
        (dx && (!valid_stride(n, k, gate_stride) || !valid_stride(n, k, up_stride) ||
                !valid_stride(m, k, dx_stride))))
        return fail(LT_ERR_INVALID_ARG, "need 0 <= m, n, k < 2^21, fewer than 2^22 tiles of 64 x 64 "
                                        "in each matrix, and strides of a row's length or more");
    if (!valid_dtype(dh_dtype) || !valid_dtype(dx_dtype) || !valid_dtype(grad_dtype))
        return fail(LT_ERR_INVALID_ARG, "dtypes must be LT_DTYPE_F32 or LT_DTYPE_BF16");
    if ((dgate != nullptr) != (dup != nullptr))
        return fail(LT_ERR_INVALID_ARG, "the weights' gradients come together");
    if (k == 0 || (!dx && !want_dw))
        return LT_OK;
    const bool empty = m == 0 || n == 0;
    if (!empty && (!dh || !saved || (dx && (!gate || !up)) || (want_dw && !x)))
        return fail(LT_ERR_INVALID_ARG, "dh, saved and the operands must not be NULL");
    if (!host::aligned(dh, dh_dtype == LT_DTYPE_BF16 ? 2 : 4) || !host::aligned(saved, 16) ||
        !host::aligned(x, 16) || !host::aligned(gate, 16) || !host::aligned(up, 16) ||
        !host::aligned(dx, 16) || !host::aligned(dgate, 16) || !host::aligned(dup, 16))
        return fail(LT_ERR_ALIGNMENT, "dh must be aligned to its elements, x, the weights, saved and "
                                      "the gradients to 16 bytes");
    const hipStream_t st = static_cast<hipStream_t>(stream);
    const BackwardLayout l = backward_layout(m, n, k, x_stride, gate_stride, up_stride,
                                             dx != nullptr, want_dw);
    const auto need = size_t(l.total);
    if (!empty && (!workspace || !host::aligned(workspace, 256) || workspace_bytes < need))
        return fail(LT_ERR_WORKSPACE, "workspace must be 256-byte aligned and hold " +
                                          std::to_string(need) + " bytes");
    std::vector<host::Range> ranges;
    const auto range = [&](const void* p, size_t bytes, bool written) {
        const auto lo = reinterpret_cast<uintptr_t>(p);
        if (p && bytes)
            ranges.push_back({lo, lo + bytes, written});
    };
    range(dx, span_bytes(m, k, dx_stride, dx_dtype), true);
    range(dgate, span_bytes(n, k, dgate_stride, grad_dtype), true);
    range(dup, span_bytes(n, k, dup_stride, grad_dtype), true);
    if (!empty) {
        range(dh, span_bytes(m, n, dh_stride, dh_dtype), false);
        range(saved, lt_gated_saved_bytes(m, n), false);
        range(workspace, need, true);
        if (want_dw)
            range(x, span_bytes(m, k, x_stride, LT_DTYPE_BF16), false);
        if (dx) {
            range(gate, span_bytes(n, k, gate_stride, LT_DTYPE_BF16), false);
            range(up, span_bytes(n, k, up_stride, LT_DTYPE_BF16), false);
        }
    }
    const std::string overlap = host::overlap(ranges);
    if (!overlap.empty())
        return fail(LT_ERR_INVALID_ARG, overlap);
    if (empty) {  // empty sums
        if (dx && m > 0)
            return host::launch_zero(dx, dx_dtype == LT_DTYPE_F32 ? 4 : 2, m, k, dx_stride, st);
        if (want_dw && n > 0) {
            const int item = grad_dtype == LT_DTYPE_F32 ? 4 : 2;
            if (lt_err e = host::launch_zero(dgate, item, n, k, dgate_stride, st))
                return e;
            return host::launch_zero(dup, item, n, k, dup_stride, st);
        }
        return LT_OK;
    }
    auto* ws = static_cast<uint8_t*>(workspace);
    if (lt_err e = host::workspace_written(ws, need, st))
        return e;
    const int64_t half = padded(n), tokens = padded(m);
    auto* slopes = reinterpret_cast<uint16_t*>(ws + l.slopes);
    ProductsArgs g{};
    g.dx = planned(l.dx, l.dx_sums < 0 ? nullptr : ws + l.dx_sums);
    g.dw = planned(l.dw, l.dw_sums < 0 ? nullptr : ws + l.dw_sums);
    Copies copies;
    if (dx) {
        turned_operand(l.gate, gate, n, k, gate_stride, ws, copies, &g.dx.b, 0);
        turned_operand(l.up, up, n, k, up_stride, ws, copies, &g.dx.b, 1);
        g.dx.b_cols = l.gate.whole ? padded(k) : k;
        g.dx.out[0] = dx;
        g.dx.stride[0] = dx_stride;
        g.dx.f32 = dx_dtype == LT_DTYPE_F32;
    }
    if (want_dw) {
        turned_operand(l.x, x, m, k, x_stride, ws, copies, &g.dw.b, 0);
        g.dw.b.base[1] = g.dw.b.base[0];
        g.dw.b.tail[1] = g.dw.b.tail[0];
        g.dw.b_cols = l.x.whole ? padded(k) : k;
        g.dw.out[0] = dgate;
        g.dw.out[1] = dup;
        g.dw.stride[0] = dgate_stride;
        g.dw.stride[1] = dup_stride;
        g.dw.f32 = grad_dtype == LT_DTYPE_F32;
    }
    g.dx.a = g.dw.a = ws + l.slopes;
    g.dx.a_pitch = g.dw.a_pitch = 4 * half;
    const auto own = uint32_t(host::ceil_div(tokens * (half / 8), 256));
    const SlopeArgs s{dh,   dh_stride, saved_layout(const_cast<void*>(saved), m, n), m, n, slopes,
                      half, tokens,    copies.of, own};
    const dim3 blocks(own + uint32_t(copies.groups));
    if (dh_dtype == LT_DTYPE_F32)
        k_gated_slopes<true><<<blocks, 256, 0, st>>>(s);
    else
        k_gated_slopes<false><<<blocks, 256, 0, st>>>(s);
    if (l.tile == 256)
        launch_products<Large16>(g, dx != nullptr, want_dw, st);
    else if (l.tile == 128)
        launch_products<Small16>(g, dx != nullptr, want_dw, st);
    else
        launch_products<Tiny16>(g, dx != nullptr, want_dw, st);
    LT_TRY_HIP(hipGetLastError());
    return LT_OK;
} catch (...) {
    return host::caught();
}

}  // extern "C"
