// fp8.hip -- matrix products in 8-bit floating point (e4m3) with a power-of-two scale for each
// block of 128 values, and the quantizer that makes their operands.
//
// A matrix is stored as codes, row by row, and for each row and each 128 columns the exponent e
// of a scale 2^e: value = code * 2^e, e the least with max |x| <= 448 * 2^e.  Powers of two
// are what the matrix instruction applies by itself, exactly and at no cost: sums stay in its
// accumulators from the first value to the last, where any other scale would need every 128
// products' sums multiplied and added apart.  Scaling by them is exact, so a value is rounded
// once, to four significant bits.
//
// Both operands of a product have the summed index contiguous, so a training step needs each of
// its matrices in the layouts of its products: x and dy by rows (forward, input gradient) and
// transposed, quantized along the tokens (weight gradient); the weight with one scale for each
// 128 x 128 block, whose codes are then the same in both layouts.  The quantizer writes both
// from one read.

#include "host.h"
#include "tiles.h"

#include <algorithm>
#include <string>
#include <vector>

namespace {

using host::fail;
using namespace tiles;

constexpr int kGroup = 128;

int64_t code_pitch(int64_t cols) { return host::ceil_div(cols, kGroup) * kGroup; }
int64_t scale_pitch(int64_t cols) { return host::ceil_div(host::ceil_div(cols, kGroup), 4) * 4; }

__device__ inline float load_value(const float* p) { return *p; }
__device__ inline float load_value(const uint16_t* p) { return __uint_as_float(uint32_t(*p) << 16); }

__device__ inline uint16_t bf16_bits(float x)
{
    return __builtin_bit_cast(uint16_t, (__bf16)x);  // to nearest even; a NaN becomes quiet
}

// ------------------------------------------------------------- quantizer

// Biased exponent of the scale for a group whose largest |x| has these bits, and the scale.
// A group with an infinity or a NaN has the NaN scale (255), and NaN codes.
struct Scale {
    uint32_t biased;
    float power;  // 2^e, or NaN
};

__device__ inline Scale scale_of(uint32_t top)
{
    Scale s;
    if (top >= 0x7F800000u)
        return {255u, __builtin_nanf("")};
    // 448 = 1.75 * 2^8; subnormals and what is below 2^-118 take the least exponent, -126
    int e = int(top >> 23) - 127 - 8 + ((top & 0x7FFFFFu) > 0x600000u ? 1 : 0);
    e = max(e, -126);
    e = top == 0u ? 0 : e;
    s.biased = uint32_t(e + 127);
    s.power = __uint_as_float(uint32_t(127 + e) << 23);
    return s;
}

// Four codes of values divided by a power of two, in the conversion itself.
typedef short s16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

__device__ inline uint32_t pack_codes(float a, float b, float c, float d, float power)
{
    s16x2 w = {0, 0};
    w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w, a, b, power, false);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w, c, d, power, true);
    return __builtin_bit_cast(uint32_t, w);
}

__device__ inline uint32_t pack_codes(uint32_t ab, uint32_t cd, float power)
{
    s16x2 w = {0, 0};
    w = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(w, __builtin_bit_cast(bf16x2, ab), power, false);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(w, __builtin_bit_cast(bf16x2, cd), power, true);
    return __builtin_bit_cast(uint32_t, w);
}

struct QuantizeArgs {
    const void* x;
    int64_t rows, cols, stride;  // elements; stride of x's rows
    uint8_t *codes, *scales;     // by rows, or null
    uint8_t *codes_t, *scales_t; // of the transpose, or null
    int64_t pitch, scale_pitch, pitch_t, scale_pitch_t;
    int across;                  // blocks of 128 columns
};

constexpr int kQuantizeThreads = 256;

// One block of 128 x 128 by a workgroup: thread t holds rows 4 (t / 16) + 64 h + r (h < 2,
// r < 4) and columns 8 (t % 16) .. + 7, so that a row's 128 columns are 16 neighbouring lanes,
// and four rows of a column are one word of the transpose.  Bound by HBM: x is read once, each
// layout of the codes written once, in whole lines: bf16 8192 x 11008 into both layouts 89 us,
// 4.1 TB/s; an fp32 weight of 11008 x 2048 31 us, 4.3 TB/s.
template <typename T, bool SQUARE>
__global__ __launch_bounds__(kQuantizeThreads) void k_fp8_quantize(QuantizeArgs a)
{
    constexpr int kTurnPitch = kGroup + 4;
    __shared__ __align__(16) uint8_t turned[kGroup * kTurnPitch];
    __shared__ uint32_t top_of[16][kGroup];  // of 8 rows of each column; [0] of all rows at last
    const int t = threadIdx.x, q = t >> 4, l = t & 15;
    const int64_t r0 = int64_t(blockIdx.x / a.across) * kGroup;
    const int64_t c0 = int64_t(blockIdx.x % a.across) * kGroup;
    const T* x = static_cast<const T*>(a.x);
    const bool whole = c0 + kGroup <= a.cols;
    float v[2][4][8];
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int64_t row = r0 + 4 * q + 64 * h + r, col = c0 + 8 * l;
            const T* p = x + row * a.stride + col;
            if (row >= a.rows) {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    v[h][r][e] = 0.0f;
            } else if (whole) {
                if constexpr (sizeof(T) == 2) {
                    const i32x4 w = load_any(p);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        v[h][r][2 * e] = __uint_as_float(uint32_t(w[e]) << 16);
                        v[h][r][2 * e + 1] = __uint_as_float(uint32_t(w[e]) & 0xFFFF0000u);
                    }
                } else {
                    const f32x4 w0 = __builtin_bit_cast(f32x4, load_any(p));
                    const f32x4 w1 = __builtin_bit_cast(f32x4, load_any(p + 4));
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        v[h][r][e] = w0[e];
                        v[h][r][4 + e] = w1[e];
                    }
                }
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    v[h][r][e] = col + e < a.cols ? load_value(p + e) : 0.0f;
            }
        }

    const auto magnitude = [](float f) { return __float_as_uint(f) & 0x7FFFFFFFu; };
    uint32_t block_top = 0;
    if constexpr (SQUARE) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int r = 0; r < 4; ++r)
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    block_top = max(block_top, magnitude(v[h][r][e]));
#pragma unroll
        for (int o = 32; o >= 1; o >>= 1)
            block_top = max(block_top, uint32_t(__shfl_xor(int(block_top), o, 64)));
        if ((t & 63) == 0)
            top_of[0][t >> 6] = block_top;
        __syncthreads();
        block_top = max(max(top_of[0][0], top_of[0][1]), max(top_of[0][2], top_of[0][3]));
    }

    // by rows
    if (a.codes) {
        const int group = int(c0 / kGroup);
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                uint32_t top = block_top;
                if constexpr (!SQUARE) {
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        top = max(top, magnitude(v[h][r][e]));
#pragma unroll
                    for (int o = 8; o >= 1; o >>= 1)
                        top = max(top, uint32_t(__shfl_xor(int(top), o, 64)));
                }
                const Scale s = scale_of(top);
                const int64_t row = r0 + 4 * q + 64 * h + r;
                if (row >= a.rows)
                    continue;
                const float(&w)[8] = v[h][r];
                *reinterpret_cast<uint2*>(a.codes + row * a.pitch + c0 + 8 * l) =
                    make_uint2(pack_codes(w[0], w[1], w[2], w[3], s.power),
                               pack_codes(w[4], w[5], w[6], w[7], s.power));
                uint8_t* to = a.scales + row * a.scale_pitch + group;
                if (l == 0)
                    *to = uint8_t(s.biased);
                else if (group + 1 == a.across && group + l < a.scale_pitch)
                    to[l] = 127;  // the last word's unused bytes
            }
    }

    // the transpose
    if (a.codes_t) {
        Scale s[8];
        if constexpr (SQUARE) {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                s[e] = scale_of(block_top);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                uint32_t top = 0;
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        top = max(top, magnitude(v[h][r][e]));
                top_of[q][8 * l + e] = top;
            }
            __syncthreads();
            if (t < kGroup) {
                uint32_t top = 0;
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    top = max(top, top_of[i][t]);
                top_of[0][t] = top;
            }
            __syncthreads();
#pragma unroll
            for (int e = 0; e < 8; ++e)
                s[e] = scale_of(top_of[0][8 * l + e]);
        }
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int e = 0; e < 8; ++e)
                *reinterpret_cast<uint32_t*>(turned + (8 * l + e) * kTurnPitch + 64 * h + 4 * q) =
                    pack_codes(v[h][0][e], v[h][1][e], v[h][2][e], v[h][3][e], s[e].power);
        __syncthreads();
        for (int i = t; i < kGroup * 8; i += kQuantizeThreads) {
            const int64_t col = c0 + i / 8;
            if (col >= a.cols)
                continue;
            const auto* from =
                reinterpret_cast<const uint32_t*>(turned + i / 8 * kTurnPitch + i % 8 * 16);
            *reinterpret_cast<uint4*>(a.codes_t + col * a.pitch_t + r0 + i % 8 * 16) =
                make_uint4(from[0], from[1], from[2], from[3]);
        }
        const int group = int(r0 / kGroup), groups = int((a.rows + kGroup - 1) / kGroup);
        if (t < kGroup && c0 + t < a.cols) {
            const Scale st = scale_of(SQUARE ? block_top : top_of[0][t]);
            uint8_t* to = a.scales_t + (c0 + t) * a.scale_pitch_t + group;
            *to = uint8_t(st.biased);
            if (group + 1 == groups)
                for (int i = 1; group + i < a.scale_pitch_t; ++i)
                    to[i] = 127;
        }
    }
}

// By rows only: a group is 16 lanes, a wave four groups of one row.  A block of 128 x 128 to a
// workgroup would leave most CUs idle for a prompt (fp32 1237 x 2011, 160 blocks: 5.8 us here,
// 10.4 there).
template <typename T>
__global__ __launch_bounds__(kQuantizeThreads) void k_fp8_quantize_rows(QuantizeArgs a)
{
    const int l = int(threadIdx.x) & 15;
    const int64_t words = a.scale_pitch / 4;  // of four groups
    const int64_t unit = int64_t(blockIdx.x) * (kQuantizeThreads / 64) + (threadIdx.x >> 6);
    const int64_t row = unit / words;
    if (row >= a.rows)
        return;
    const int64_t group = unit % words * 4 + (threadIdx.x >> 4 & 3);
    const int64_t col = group * kGroup + 8 * l;
    const T* p = static_cast<const T*>(a.x) + row * a.stride + col;
    float v[8];
    if (col + 8 <= a.cols) {
        constexpr int kLine = 16 / sizeof(T);
#pragma unroll
        for (int c = 0; c < 8; c += kLine) {
            const i32x4 w = load_any(p + c);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if constexpr (sizeof(T) == 2) {
                    v[2 * e] = __uint_as_float(uint32_t(w[e]) << 16);
                    v[2 * e + 1] = __uint_as_float(uint32_t(w[e]) & 0xFFFF0000u);
                } else {
                    v[c + e] = __int_as_float(w[e]);
                }
            }
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            v[e] = col + e < a.cols ? load_value(p + e) : 0.0f;
    }
    uint32_t top = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e)
        top = max(top, __float_as_uint(v[e]) & 0x7FFFFFFFu);
#pragma unroll
    for (int o = 8; o >= 1; o >>= 1)
        top = max(top, uint32_t(__shfl_xor(int(top), o, 64)));
    const Scale s = scale_of(top);  // a group past the last column is zeros: 127
    if (l == 0)
        a.scales[row * a.scale_pitch + group] = uint8_t(s.biased);
    if (group * kGroup < a.cols)
        *reinterpret_cast<uint2*>(a.codes + row * a.pitch + col) =
            make_uint2(pack_codes(v[0], v[1], v[2], v[3], s.power),
                       pack_codes(v[4], v[5], v[6], v[7], s.power));
}

// ------------------------------------------------------------- products

struct ProductArgs {
    const uint8_t *a, *a_scales, *b, *b_scales;
    int64_t m, n;              // rows of a and of b
    int64_t pitch, scale_pitch;
    int steps;                 // of 128 summed values
    int slice;                 // steps of one slice of the sum (gridDim.y slices), whole words
    void* out;
    int64_t stride;            // of out's rows, elements
    float* partial;            // several slices: [slice][m][n]
};

// Results to out, or one slice's sums to the workspace.
template <bool F32>
struct ProductWriter {
    static constexpr bool kTurned = false;
    static constexpr int kSlots = 8;
    void* out;
    int64_t stride, rows, cols;  // from the tile's origin on
    __device__ inline void fetch(int, int, int) {}
    __device__ inline void turn(int, int, const float (&)[8]) {}
    __device__ inline void store_one(int row, int col, float v)
    {
        if (row >= rows || col >= cols)
            return;
        const int64_t at = row * stride + col;
        if constexpr (F32)
            static_cast<float*>(out)[at] = v;
        else
            static_cast<uint16_t*>(out)[at] = bf16_bits(v);
    }
    __device__ inline void store(int row, int col, float (&v)[8], int)
    {
        typedef uint16_t u16x8 __attribute__((ext_vector_type(8)));
        if (row >= rows)
            return;
        if (col + 8 > cols) {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                store_one(row, col + e, v[e]);
            return;
        }
        const int64_t at = row * stride + col;
        if constexpr (F32) {
            float* p = static_cast<float*>(out) + at;
            store_any(p, f32x4{v[0], v[1], v[2], v[3]});
            store_any(p + 4, f32x4{v[4], v[5], v[6], v[7]});
        } else {
            u16x8 b;
#pragma unroll
            for (int e = 0; e < 8; ++e)
                b[e] = bf16_bits(v[e]);
            store_any(static_cast<uint16_t*>(out) + at, b);
        }
    }
};

// One tile of the result, or of one slice's sums.  16384 cubed 2.6 to 2.8 PFLOP/s on random codes
// and 3.3 on zeros: what bounds the first is power, the second the copies into LDS (tiles.h).
// A tile of 256 costs some 10 us beside its 1.0 to 1.4 us a step, most of it every CU's result
// leaving at once at the end of a round: 8192 x 11008 x 2048 1.9 PFLOP/s.
template <typename Tile, bool F32>
__global__ __launch_bounds__(Tile::kThreads, Tile::kWavesPerSimd) void k_fp8_product(ProductArgs g)
{
    __shared__ __align__(1024) uint8_t lds[Tile::kLdsBytes + Fp8<Tile>::kLdsBytes];
    const int64_t unit = unit_of_workgroup(Tile::kRun);
    const TilePlace at = tile_place(int(unit), int((g.m + Tile::kRows - 1) / Tile::kRows),
                                    int((g.n + Tile::kCols - 1) / Tile::kCols));
    const int64_t r0 = int64_t(at.row) * Tile::kRows, c0 = int64_t(at.col) * Tile::kCols;
    const int first = int(blockIdx.y) * g.slice, steps = min(g.slice, g.steps - first);
    Tile tile;
    Fp8<Tile> mul;
    mul.scales_p = g.a_scales + r0 * g.scale_pitch + first;
    mul.scales_q = g.b_scales + c0 * g.scale_pitch + first;
    mul.pitch = g.scale_pitch;
    mul.limit_p = g.m - r0;
    mul.limit_q = g.n - c0;
    mul.words = (steps + 3) / 4;
    mul.lds = lds + Tile::kLdsBytes;
    product(mul, tile, g.a + r0 * g.pitch + int64_t(first) * kStepBytes, g.pitch, g.m - r0,
            g.b + c0 * g.pitch + int64_t(first) * kStepBytes, g.pitch, g.n - c0, steps, lds);
    ProductWriter<F32> w;
    w.rows = g.m - r0;
    w.cols = g.n - c0;
    if (g.partial) {
        ProductWriter<true> p;
        p.rows = w.rows;
        p.cols = w.cols;
        p.stride = g.n;
        p.out = g.partial + (int64_t(blockIdx.y) * g.m + r0) * g.n + c0;
        finish(tile, lds, p);
        return;
    }
    w.stride = g.stride;
    w.out = F32 ? static_cast<void*>(static_cast<float*>(g.out) + r0 * g.stride + c0)
                : static_cast<void*>(static_cast<uint16_t*>(g.out) + r0 * g.stride + c0);
    finish(tile, lds, w);
}

// out = the slices' sums, added in their order.
template <bool F32>
__global__ __launch_bounds__(256) void k_fp8_join(const float* __restrict__ partial, int slices,
                                                  int64_t m, int64_t n, void* out, int64_t stride)
{
    const int64_t all = m * n;
    for (int64_t e = int64_t(blockIdx.x) * 256 + threadIdx.x; e < all;
         e += int64_t(gridDim.x) * 256) {
        float s = partial[e];
        for (int i = 1; i < slices; ++i)
            s += partial[i * all + e];
        const int64_t to = e / n * stride + e % n;
        if constexpr (F32)
            static_cast<float*>(out)[to] = s;
        else
            static_cast<uint16_t*>(out)[to] = bf16_bits(s);
    }
}

// ------------------------------------------------------------- few tokens

// y for up to 16 T tokens, bound by reading the weight once: no LDS tiles, every lane loads its
// 32 bytes of the instruction's 16 weight rows straight from HBM.  The waves of a workgroup
// share R blocks of 16 rows and cut the sum.  x comes as
// codes, or (T = 1) as it is: a lane then quantizes the 32 values of its token that it
// multiplies, with the group's maximum from the other three lanes that hold the group, so that a
// single token is one launch and x never waits for a pass of its own.
struct FewArgs {
    const uint8_t *w, *w_scales;
    const void* x;               // codes, or values
    const uint8_t* x_scales;
    int64_t m, n, k;
    int64_t pitch, scale_pitch;  // of the weight's rows, and of x's codes
    int64_t x_stride;            // of x's values
    int steps;
    void* out;
    int64_t stride;
};

enum { kCodes, kF32, kBf16 };

struct FewToken {
    i32x8 codes;
    uint32_t scale;
};

// What a lane has of its token and one step, as loaded: 32 codes and their scale, or 32 values.
template <int X>
struct FewInput {
    static constexpr int kWords = X == kCodes ? 2 : (X == kBf16 ? 4 : 8);
    i32x4 w[kWords];
    uint32_t scale;
};

template <typename T>
__device__ inline void few_load(const T* row, int64_t k, int s, int q, i32x4* w)
{
    const int64_t at = int64_t(s) * kGroup + 32 * q;
    const T* p = row + at;
    constexpr int kWords = int(32 * sizeof(T) / 16);
    if (at + 32 <= k) {
#pragma unroll
        for (int c = 0; c < kWords; ++c)
            w[c] = load_any(p + c * int(16 / sizeof(T)));
        return;
    }
#pragma unroll
    for (int c = 0; c < kWords; ++c)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if constexpr (sizeof(T) == 2) {
                const int i = 8 * c + 2 * e;
                const uint32_t lo = at + i < k ? p[i] : 0u, hi = at + i + 1 < k ? p[i + 1] : 0u;
                w[c][e] = int(lo | hi << 16);
            } else {
                w[c][e] = at + 4 * c + e < k ? __float_as_int(p[4 * c + e]) : 0;
            }
        }
}

template <int X>
__device__ inline FewToken few_quantize(const FewInput<X>& in)
{
    FewToken f;
    if constexpr (X == kCodes) {
        f.codes = i32x8{in.w[0][0], in.w[0][1], in.w[0][2], in.w[0][3],
                        in.w[1][0], in.w[1][1], in.w[1][2], in.w[1][3]};
        f.scale = in.scale;
        return f;
    }
    constexpr int kWords = FewInput<X>::kWords;
    uint32_t top = 0;
    if constexpr (X == kBf16) {
        typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
        u16x2 most = {0, 0};  // a bf16's magnitude is its pattern without the sign
#pragma unroll
        for (int c = 0; c < kWords; ++c)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                most = __builtin_elementwise_max(
                    most, __builtin_bit_cast(u16x2, uint32_t(in.w[c][e]) & 0x7FFF7FFFu));
        top = uint32_t(max(most[0], most[1])) << 16;
    } else {
#pragma unroll
        for (int c = 0; c < kWords; ++c)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                top = max(top, uint32_t(in.w[c][e]) & 0x7FFFFFFFu);
    }
    top = max(top, uint32_t(__shfl_xor(int(top), 16, 64)));
    top = max(top, uint32_t(__shfl_xor(int(top), 32, 64)));
    const Scale scale = scale_of(top);
    f.scale = scale.biased;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        if constexpr (X == kBf16) {
            f.codes[e] = int(pack_codes(uint32_t(in.w[e / 2][e % 2 * 2]),
                                        uint32_t(in.w[e / 2][e % 2 * 2 + 1]), scale.power));
        } else {
            const i32x4 v = in.w[e];
            f.codes[e] = int(pack_codes(__int_as_float(v[0]), __int_as_float(v[1]),
                                        __int_as_float(v[2]), __int_as_float(v[3]), scale.power));
        }
    }
    return f;
}

// Step s of one token, as a lane needs it.
template <int X>
__device__ inline void few_input(const FewArgs& g, int64_t token, int s, int q, FewInput<X>& in)
{
    if constexpr (X == kCodes) {
        const auto* p = reinterpret_cast<const i32x4*>(static_cast<const uint8_t*>(g.x) +
                                                       token * g.pitch + int64_t(s) * kGroup +
                                                       32 * q);
        in.w[0] = p[0];
        in.w[1] = p[1];
        in.scale = g.x_scales[token * g.scale_pitch + s];
    } else if constexpr (X == kF32) {
        few_load(static_cast<const float*>(g.x) + token * g.x_stride, g.k, s, q,
                 in.w);
    } else {
        few_load(static_cast<const uint16_t*>(g.x) + token * g.x_stride, g.k, s, q,
                 in.w);
    }
}

__device__ inline i32x8 load_codes(const uint8_t* p)
{
    const i32x4 a = reinterpret_cast<const i32x4*>(p)[0], b = reinterpret_cast<const i32x4*>(p)[1];
    return i32x8{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
}

template <int T, int R, int X, bool F32>
__global__ __launch_bounds__(512) void k_fp8_few(FewArgs g)
{
    extern __shared__ float sums[];  // [wave][R][T][lane][4]
    const int lane = int(threadIdx.x) & 63, r = lane & 15, q = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x) >> 6);
    const int waves = int(blockDim.x) >> 6;
    const int64_t n0 = int64_t(blockIdx.x) * 16 * R;
    const uint8_t *w[R], *ws[R];
#pragma unroll
    for (int i = 0; i < R; ++i) {
        int64_t row = n0 + 16 * i + r;
        row = row < g.n ? row : g.n - 1;
        w[i] = g.w + row * g.pitch + 32 * q;
        ws[i] = g.w_scales + row * g.scale_pitch;
    }
    int64_t token[T];
#pragma unroll
    for (int t = 0; t < T; ++t) {
        token[t] = 16 * t + r;
        token[t] = token[t] < g.m ? token[t] : g.m - 1;
    }
    f32x4 acc[R][T] = {};
    // one step is under way while the one before is multiplied
    struct Loaded {
        i32x8 a[R];
        uint32_t as[R];
        FewInput<X> x[T];
    };
    const auto load = [&](int s, Loaded& in) {
#pragma unroll
        for (int i = 0; i < R; ++i) {
            in.a[i] = load_codes(w[i] + int64_t(s) * kGroup);
            in.as[i] = ws[i][s];
        }
#pragma unroll
        for (int t = 0; t < T; ++t)
            few_input(g, token[t], s, q, in.x[t]);
    };
    const auto multiply = [&](const Loaded& in) {
#pragma unroll
        for (int t = 0; t < T; ++t) {
            const FewToken f = few_quantize<X>(in.x[t]);
#pragma unroll
            for (int i = 0; i < R; ++i)
                acc[i][t] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(
                    in.a[i], f.codes, acc[i][t], 0, 0, 0, int(in.as[i]), 0, int(f.scale));
        }
    };
    // each wave has a run of neighbouring steps: its rows are read in long pieces
    const int first = g.steps * wave / waves, last = g.steps * (wave + 1) / waves;
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
    // the waves' sums, added in their order: acc[i][t][e] is row 16 i + 4 q + e, token 16 t + r
#pragma unroll
    for (int i = 0; i < R; ++i)
#pragma unroll
        for (int t = 0; t < T; ++t)
            *reinterpret_cast<f32x4*>(sums + (((wave * R + i) * T + t) * 64 + lane) * 4) =
                acc[i][t];
    __syncthreads();
    for (int e = threadIdx.x; e < R * T * 256; e += int(blockDim.x)) {
        float v = sums[e];
        for (int i = 1; i < waves; ++i)
            v += sums[i * R * T * 256 + e];
        const int l = e / 4 % 64, block = e / 256;
        const int64_t row = n0 + 16 * (block / T) + 4 * (l >> 4) + e % 4;
        const int64_t tok = 16 * (block % T) + (l & 15);
        if (row >= g.n || tok >= g.m)
            continue;
        const int64_t to = tok * g.stride + row;
        if constexpr (F32)
            static_cast<float*>(g.out)[to] = v;
        else
            static_cast<uint16_t*>(g.out)[to] = bf16_bits(v);
    }
}

// The same where a wave can hold its share of x: eight waves cut the sum, each with up to STEPS
// steps of 16 T tokens in its registers, and go through blocks of 16 rows together, the next
// block's codes under way while one is multiplied.  x is read (and quantized) once for a
// workgroup and not once for every 16 or 32 rows: 16 tokens through 5120 x 17408 28 us (3.2 TB/s
// of the weight), without 41; a token through 2048 x 11008 8.3 and 10.3.
constexpr int kHeldWaves = 8;

template <int STEPS, int T, int X, bool F32>
__global__ __launch_bounds__(64 * kHeldWaves) void k_fp8_few_held(FewArgs g)
{
    __shared__ float sums[2][kHeldWaves][T][256];
    const int lane = int(threadIdx.x) & 63, r = lane & 15, q = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x) >> 6);
    const int first = g.steps * wave / kHeldWaves;
    const int count = g.steps * (wave + 1) / kHeldWaves - first;
    const int64_t blocks = (g.n + 15) / 16;

    struct Rows {
        i32x8 codes[STEPS];
        uint32_t scale[STEPS];
    } even, odd;
    const auto load = [&](int64_t block, Rows& w) {
        int64_t row = block * 16 + r;
        row = row < g.n ? row : g.n - 1;
        const uint8_t* p = g.w + row * g.pitch + int64_t(first) * kGroup + 32 * q;
        const uint8_t* s = g.w_scales + row * g.scale_pitch + first;
#pragma unroll
        for (int i = 0; i < STEPS; ++i)
            if (i < count) {
                w.codes[i] = load_codes(p + i * kGroup);
                w.scale[i] = s[i];
            }
    };
    load(blockIdx.x, even);

    FewToken x[T][STEPS];
#pragma unroll
    for (int t = 0; t < T; ++t) {
        const int64_t token = 16 * t + r < g.m ? 16 * t + r : g.m - 1;
        FewInput<X> in[STEPS];
#pragma unroll
        for (int i = 0; i < STEPS; ++i)
            if (i < count)
                few_input(g, token, first + i, q, in[i]);
#pragma unroll
        for (int i = 0; i < STEPS; ++i)
            if (i < count)
                x[t][i] = few_quantize<X>(in[i]);
    }
    const auto multiply = [&](int64_t block, const Rows& w, int turn) {
#pragma unroll
        for (int t = 0; t < T; ++t) {
            f32x4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int i = 0; i < STEPS; ++i)
                if (i < count)
                    acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(
                        w.codes[i], x[t][i].codes, acc, 0, 0, 0, int(w.scale[i]), 0,
                        int(x[t][i].scale));
            // acc[e] is row 4 q + e, token 16 t + r
            *reinterpret_cast<f32x4*>(&sums[turn][wave][t][lane * 4]) = acc;
        }
        __syncthreads();  // and the other buffer's sums have been read
        const int e = threadIdx.x % 256, t = threadIdx.x / 256;
        if (t >= T)
            return;
        float v = sums[turn][0][t][e];
#pragma unroll
        for (int i = 1; i < kHeldWaves; ++i)
            v += sums[turn][i][t][e];
        const int64_t row = block * 16 + 4 * (e >> 6) + e % 4, tok = 16 * t + e / 4 % 16;
        if (row >= g.n || tok >= g.m)
            return;
        const int64_t to = tok * g.stride + row;
        if constexpr (F32)
            static_cast<float*>(g.out)[to] = v;
        else
            static_cast<uint16_t*>(g.out)[to] = bf16_bits(v);
    };
    for (int64_t b = blockIdx.x; b < blocks; b += 2 * int64_t(gridDim.x)) {
        const int64_t next = b + gridDim.x;
        if (next < blocks)
            load(next, odd);
        multiply(b, even, 0);
        if (next >= blocks)
            break;
        if (next + gridDim.x < blocks)
            load(next + gridDim.x, even);
        multiply(next, odd, 1);
    }
}

template <bool F32>
__global__ __launch_bounds__(256) void k_fp8_zero(int64_t m, int64_t n, void* out, int64_t stride)
{
    const int64_t all = m * n;
    for (int64_t e = int64_t(blockIdx.x) * 256 + threadIdx.x; e < all;
         e += int64_t(gridDim.x) * 256) {
        const int64_t to = e / n * stride + e % n;
        if constexpr (F32)
            static_cast<float*>(out)[to] = 0.0f;
        else
            static_cast<uint16_t*>(out)[to] = 0;
    }
}

// ---------------------------------------------------------------- host side

// Rows of codes stay within the 32-bit offsets of a tile's loads.
constexpr int64_t kMostSummed = int64_t(1) << 23;
// Workgroups of 256 threads in a launch: the grid counts threads in 32 bits.
constexpr int64_t kMostGroups = int64_t(1) << 24;

struct Way {
    int tile;    // 256, 128 or 64
    int slices;  // of the sum
    int slice;   // steps of each
};

// The largest tile that still leaves every CU a workgroup (2048 x 4096 x 4096: tiles of 128 38 us,
// of 256 50; 4096 x 4096 x 4096: 76 and 61; 128 x 4096 x 4096: of 64 14, of 128 18).  Where even
// the smallest does not, a long sum is cut as well, into slices of 512 values or more: with the
// pass that joins them 64 x 4096 x 4096 takes 18 us, in one piece 13; 64 x 4096 x 8192 17 and 25,
// 256 x 256 x 16384 21 and 36.
constexpr int kLongSum = 48;        // steps
constexpr int64_t kUncutSum = 512;  // values: up to here no workspace is looked at

Way way_of(int64_t m, int64_t n, int64_t k)
{
    const int steps = int(host::ceil_div(k, kGroup));
    Way w{64, 1, steps};
    int64_t tiles = 0;
    for (const int t : {256, 128, 64}) {
        w.tile = t;
        tiles = host::ceil_div(m, t) * host::ceil_div(n, t);
        if (tiles >= 256)
            return w;
    }
    if (steps < kLongSum)
        return w;
    const int words = int(host::ceil_div(steps, 4));
    const int want = int(std::min<int64_t>(words, host::ceil_div(512, std::max<int64_t>(tiles, 1))));
    const int per = int(host::ceil_div(words, std::max(want, 1)));
    w.slice = std::max(per, 1) * 4;
    w.slices = std::max(1, int(host::ceil_div(steps, w.slice)));
    if (w.slices == 1)
        w.slice = steps;
    return w;
}

bool valid_sizes(int64_t m, int64_t n, int64_t k)
{
    const int64_t most = int64_t(1) << 28;
    return m >= 0 && n >= 0 && k >= 0 && m < most && n < most && k < kMostSummed &&
           host::ceil_div(m, 256) * host::ceil_div(n, 256) < kMostGroups;
}

// The last element of a matrix has an address, with room to spare in 64 bits.
bool valid_stride(int64_t rows, int64_t cols, int64_t stride)
{
    return stride >= cols && stride <= (int64_t(1) << 46) / std::max<int64_t>(rows, 1);
}

// Bytes from the first to the last element of rows x cols, `stride` elements from row to row.
size_t span_bytes(int64_t rows, int64_t cols, int64_t stride, int dtype)
{
    if (rows == 0 || cols == 0)
        return 0;
    return size_t((rows - 1) * stride + cols) * (dtype == LT_DTYPE_BF16 ? 2 : 4);
}

template <typename Tile>
void launch_product(const ProductArgs& g, const Way& w, bool f32, hipStream_t st)
{
    const dim3 grid(uint32_t(host::ceil_div(g.m, Tile::kRows) * host::ceil_div(g.n, Tile::kCols)),
                    uint32_t(w.slices));
    if (f32)
        k_fp8_product<Tile, true><<<grid, Tile::kThreads, 0, st>>>(g);
    else
        k_fp8_product<Tile, false><<<grid, Tile::kThreads, 0, st>>>(g);
}

// Tokens that the kernel for few takes, and up to which it takes them unquantized.  With the
// quantizer's pass, 17 tokens through 2048 x 11008 take 12 us here and 14 by tiles, through
// 5120 x 17408 30 and 33; 32 through 2048 x 2048 8.2 and 10.4, through 2048 x 11008 14 and 14.  At
// 64 the tiles were faster, 21 us against 31.
constexpr int64_t kFewTokens = 32;
constexpr int64_t kFewValues = 16;

template <int T, int R, int X>
void launch_few_rows(const FewArgs& g, bool f32, hipStream_t st)
{
    // eight waves where four would not give every CU sixteen and the sum is long enough to cut
    const int64_t groups = host::ceil_div(g.n, 16 * R);
    const int waves = groups * 4 < 4096 && g.steps >= 8 ? 8 : 4;
    const size_t lds = size_t(waves) * R * T * 1024;
    auto* kernel = f32 ? k_fp8_few<T, R, X, true> : k_fp8_few<T, R, X, false>;
    kernel<<<dim3(uint32_t(groups)), 64 * waves, lds, st>>>(g);
}

// Two blocks of 16 rows share a token's codes where that leaves every CU two workgroups (a token
// through 2048 x 151936: 64 us, with one block 79; through 2048 x 2048 4.8, with two 5.8).
template <int T, int X>
void launch_few(const FewArgs& g, bool f32, hipStream_t st)
{
    if (g.n >= 32 * 512)
        launch_few_rows<T, 2, X>(g, f32, st);
    else
        launch_few_rows<T, 1, X>(g, f32, st);
}

template <int STEPS, int T, int X>
void launch_held(const FewArgs& g, bool f32, int cus, hipStream_t st)
{
    // two workgroups to a CU where they are small (16 tokens through 2048 x 151936 69 us, with one
    // 81), else one (5120 x 17408: 28 us, with two 34)
    const int64_t groups = std::min<int64_t>(host::ceil_div(g.n, 16), STEPS <= 2 ? 2 * cus : cus);
    auto* kernel = f32 ? k_fp8_few_held<STEPS, T, X, true> : k_fp8_few_held<STEPS, T, X, false>;
    kernel<<<dim3(uint32_t(groups)), 64 * kHeldWaves, 0, st>>>(g);
}

// x is held where its share fits a wave's registers: up to 8192 values of 16 tokens (5120 in
// fp32 on the way), 5120 of 32.  Kernels are for 2, 5 and 8 steps a wave: between, a length takes
// the next larger one's registers, and above 2048 values its one workgroup a CU.
template <int X>
void launch_few_tokens(const FewArgs& g, bool f32, int cus, hipStream_t st)
{
    const int each = int(host::ceil_div(g.steps, kHeldWaves));
    if constexpr (X == kCodes)
        if (g.m > 16) {
            if (each <= 2)
                launch_held<2, 2, X>(g, f32, cus, st);
            else if (each <= 5)
                launch_held<5, 2, X>(g, f32, cus, st);
            else
                launch_few<2, X>(g, f32, st);
            return;
        }
    if (each <= 2) {
        launch_held<2, 1, X>(g, f32, cus, st);
    } else if (each <= 5) {
        launch_held<5, 1, X>(g, f32, cus, st);
    } else {
        if constexpr (X != kF32)
            if (each <= 8) {
                launch_held<8, 1, X>(g, f32, cus, st);
                return;
            }
        launch_few<1, X>(g, f32, st);
    }
}

// The quantizer's launch, its arguments checked; x at any element's address.
lt_err launch_quantize(const void* x, int dtype, int64_t rows, int64_t cols, int64_t row_stride,
                       bool square, uint8_t* codes, uint8_t* scales, uint8_t* codes_t,
                       uint8_t* scales_t, hipStream_t st)
{
    QuantizeArgs a{x,
                   rows,
                   cols,
                   row_stride,
                   codes,
                   scales,
                   codes_t,
                   scales_t,
                   code_pitch(cols),
                   scale_pitch(cols),
                   code_pitch(rows),
                   scale_pitch(rows),
                   int(host::ceil_div(cols, kGroup))};
    const dim3 grid(uint32_t(host::ceil_div(rows, kGroup) * a.across));
    const int64_t by_rows = host::ceil_div(rows * (a.scale_pitch / 4), kQuantizeThreads / 64);
    if (!codes_t && !square && by_rows < kMostGroups) {
        auto* kernel = dtype == LT_DTYPE_BF16 ? k_fp8_quantize_rows<uint16_t>
                                              : k_fp8_quantize_rows<float>;
        kernel<<<dim3(uint32_t(by_rows)), kQuantizeThreads, 0, st>>>(a);
        LT_TRY_HIP(hipGetLastError());
        return LT_OK;
    }
    auto* kernel = dtype == LT_DTYPE_BF16
                       ? (square ? k_fp8_quantize<uint16_t, true> : k_fp8_quantize<uint16_t, false>)
                       : (square ? k_fp8_quantize<float, true> : k_fp8_quantize<float, false>);
    kernel<<<grid, kQuantizeThreads, 0, st>>>(a);
    LT_TRY_HIP(hipGetLastError());
    return LT_OK;
}

// Workspace of lt_fp8_linear where x is quantized apart: [codes][scales][matmul's].
struct LinearLayout {
    size_t scales, matmul, total;
};

LinearLayout linear_layout(int64_t m, int64_t n, int64_t k)
{
    LinearLayout l{0, 0, 256};
    if (m <= kFewValues)
        return l;
    l.scales = host::round_up(size_t(m) * size_t(code_pitch(k)), 256);
    l.matmul = l.scales + host::round_up(size_t(m) * size_t(scale_pitch(k)), 256);
    l.total = l.matmul + lt_fp8_matmul_workspace_bytes(m, n, k);
    return l;
}

}  // namespace

extern "C" {

int64_t lt_fp8_code_pitch(int64_t cols) { return cols < 0 ? 0 : code_pitch(cols); }

int64_t lt_fp8_scale_pitch(int64_t cols) { return cols < 0 ? 0 : scale_pitch(cols); }

lt_err lt_fp8_quantize(const void* x, int dtype, int64_t rows, int64_t cols, int64_t row_stride,
                       int square, uint8_t* codes, uint8_t* scales, uint8_t* codes_t,
                       uint8_t* scales_t, void* stream)
try {
    host::clear_error();
    if (dtype != LT_DTYPE_F32 && dtype != LT_DTYPE_BF16)
        return fail(LT_ERR_INVALID_ARG, "dtype must be LT_DTYPE_F32 or LT_DTYPE_BF16");
    const int64_t most = int64_t(1) << 31;
    if (rows < 0 || cols < 0 || rows >= most || cols >= most ||
        !valid_stride(rows, cols, row_stride) ||
        host::ceil_div(rows, kGroup) * host::ceil_div(cols, kGroup) >= kMostGroups)
        return fail(LT_ERR_INVALID_ARG, "need 0 <= rows, cols < 2^31, blocks of 128 x 128 < 2^24 "
                                        "and row_stride >= cols");
    if ((codes != nullptr) != (scales != nullptr) || (codes_t != nullptr) != (scales_t != nullptr))
        return fail(LT_ERR_INVALID_ARG, "codes come with their scales");
    if (rows == 0 || cols == 0)
        return LT_OK;
    if (!x || (!codes && !codes_t))
        return fail(LT_ERR_INVALID_ARG, "x and at least one layout of codes must be given");
    if (!host::aligned(x, 16) || !host::aligned(codes, 16) || !host::aligned(codes_t, 16) ||
        !host::aligned(scales, 4) || !host::aligned(scales_t, 4))
        return fail(LT_ERR_ALIGNMENT, "x and codes must be 16-byte aligned, scales 4-byte");
    std::vector<host::Range> ranges;
    const auto range = [&](const void* p, size_t bytes, bool written) {
        const auto lo = reinterpret_cast<uintptr_t>(p);
        if (p)
            ranges.push_back({lo, lo + bytes, written});
    };
    range(x, span_bytes(rows, cols, row_stride, dtype), false);
    range(codes, size_t(rows) * size_t(code_pitch(cols)), true);
    range(scales, size_t(rows) * size_t(scale_pitch(cols)), true);
    range(codes_t, size_t(cols) * size_t(code_pitch(rows)), true);
    range(scales_t, size_t(cols) * size_t(scale_pitch(rows)), true);
    const std::string overlap = host::overlap(ranges);
    if (!overlap.empty())
        return fail(LT_ERR_INVALID_ARG, overlap);
    return launch_quantize(x, dtype, rows, cols, row_stride, square != 0, codes, scales, codes_t,
                           scales_t, static_cast<hipStream_t>(stream));
} catch (...) {
    return host::caught();
}

size_t lt_fp8_matmul_workspace_bytes(int64_t m, int64_t n, int64_t k)
{
    if (!valid_sizes(m, n, k))
        return 0;
    if (m <= kFewTokens)
        return 256;
    const Way w = way_of(m, n, k);
    return std::max(size_t(256),
                    w.slices > 1 ? size_t(w.slices) * size_t(m) * size_t(n) * 4 : size_t(0));
}

lt_err lt_fp8_matmul(const uint8_t* a_codes, const uint8_t* a_scales, const uint8_t* b_codes,
                     const uint8_t* b_scales, int64_t m, int64_t n, int64_t k, void* out,
                     int out_dtype, int64_t out_stride, void* workspace, size_t workspace_bytes,
                     void* stream)
try {
    host::clear_error();
    if (!valid_sizes(m, n, k) || !valid_stride(m, n, out_stride))
        return fail(LT_ERR_INVALID_ARG, "need 0 <= m, n < 2^28, 0 <= k < 2^23 and out_stride >= n");
    if (out_dtype != LT_DTYPE_F32 && out_dtype != LT_DTYPE_BF16)
        return fail(LT_ERR_INVALID_ARG, "out_dtype must be LT_DTYPE_F32 or LT_DTYPE_BF16");
    if (m == 0 || n == 0)
        return LT_OK;
    if (!out || (k > 0 && (!a_codes || !a_scales || !b_codes || !b_scales)))
        return fail(LT_ERR_INVALID_ARG, "operands and out must not be NULL");
    if (!host::aligned(a_codes, 16) || !host::aligned(b_codes, 16) || !host::aligned(out, 16) ||
        !host::aligned(a_scales, 4) || !host::aligned(b_scales, 4))
        return fail(LT_ERR_ALIGNMENT, "codes and out must be 16-byte aligned, scales 4-byte");
    const hipStream_t st = static_cast<hipStream_t>(stream);
    const bool f32 = out_dtype == LT_DTYPE_F32;
    const Way w = way_of(m, n, k);
    const bool few = m <= kFewTokens;
    if (k > kUncutSum && !few) {
        const size_t need = lt_fp8_matmul_workspace_bytes(m, n, k);
        if (!workspace || !host::aligned(workspace, 256) || workspace_bytes < need)
            return fail(LT_ERR_WORKSPACE, "workspace must be 256-byte aligned and hold " +
                                              std::to_string(need) + " bytes");
    }
    const size_t out_bytes = span_bytes(m, n, out_stride, out_dtype);
    const size_t a_pitch = size_t(code_pitch(k)), a_scale_pitch = size_t(scale_pitch(k));
    if (host::overlaps(out, out_bytes, a_codes, size_t(m) * a_pitch) ||
        host::overlaps(out, out_bytes, b_codes, size_t(n) * a_pitch) ||
        host::overlaps(out, out_bytes, a_scales, size_t(m) * a_scale_pitch) ||
        host::overlaps(out, out_bytes, b_scales, size_t(n) * a_scale_pitch))
        return fail(LT_ERR_INVALID_ARG, "out overlaps an operand");
    if (k == 0) {  // an empty sum
        auto* join = f32 ? k_fp8_zero<true> : k_fp8_zero<false>;
        join<<<dim3(uint32_t(std::min<int64_t>(4096, host::ceil_div(m * n, 256)))), 256, 0, st>>>(
            m, n, out, out_stride);
        LT_TRY_HIP(hipGetLastError());
        return LT_OK;
    }
    if (few) {
        const FewArgs f{b_codes, b_scales, a_codes, a_scales, m, n, k, code_pitch(k),
                        scale_pitch(k), 0, int(host::ceil_div(k, kGroup)), out, out_stride};
        int cus;
        if (lt_err e = host::compute_units(&cus))
            return e;
        launch_few_tokens<kCodes>(f, f32, cus, st);
        LT_TRY_HIP(hipGetLastError());
        return LT_OK;
    }
    ProductArgs g{a_codes, a_scales,   b_codes, b_scales,   m,      n, code_pitch(k),
                  scale_pitch(k), int(host::ceil_div(k, kGroup)), w.slice, out, out_stride, nullptr};
    if (w.slices > 1) {
        g.partial = static_cast<float*>(workspace);
        if (lt_err e = host::workspace_written(
                workspace, size_t(w.slices) * size_t(m) * size_t(n) * 4, st))
            return e;
    }
    if (w.tile == 256)
        launch_product<Large>(g, w, f32, st);
    else if (w.tile == 128)
        launch_product<Small>(g, w, f32, st);
    else
        launch_product<Tiny>(g, w, f32, st);
    if (g.partial) {
        auto* join = f32 ? k_fp8_join<true> : k_fp8_join<false>;
        join<<<dim3(uint32_t(std::min<int64_t>(4096, host::ceil_div(m * n, 256)))), 256, 0, st>>>(
            g.partial, w.slices, m, n, out, out_stride);
    }
    LT_TRY_HIP(hipGetLastError());
    return LT_OK;
} catch (...) {
    return host::caught();
}

size_t lt_fp8_linear_workspace_bytes(int64_t m, int64_t n, int64_t k)
{
    return valid_sizes(m, n, k) ? linear_layout(m, n, k).total : 0;
}

lt_err lt_fp8_linear(const void* x, int dtype, int64_t x_stride, const uint8_t* w_codes,
                     const uint8_t* w_scales, int64_t m, int64_t n, int64_t k, void* out,
                     int out_dtype, int64_t out_stride, void* workspace, size_t workspace_bytes,
                     void* stream)
try {
    host::clear_error();
    if (!valid_sizes(m, n, k) || !valid_stride(m, n, out_stride) || !valid_stride(m, k, x_stride))
        return fail(LT_ERR_INVALID_ARG, "need 0 <= m, n < 2^28, 0 <= k < 2^23, x_stride >= k and "
                                        "out_stride >= n");
    if ((dtype != LT_DTYPE_F32 && dtype != LT_DTYPE_BF16) ||
        (out_dtype != LT_DTYPE_F32 && out_dtype != LT_DTYPE_BF16))
        return fail(LT_ERR_INVALID_ARG, "dtypes must be LT_DTYPE_F32 or LT_DTYPE_BF16");
    if (m == 0 || n == 0)
        return LT_OK;
    if (!out || (k > 0 && (!x || !w_codes || !w_scales)))
        return fail(LT_ERR_INVALID_ARG, "x, the weight and out must not be NULL");
    if (!host::aligned(x, dtype == LT_DTYPE_BF16 ? 2 : 4) || !host::aligned(w_codes, 16) ||
        !host::aligned(out, 16) || !host::aligned(w_scales, 4))
        return fail(LT_ERR_ALIGNMENT, "x must be aligned to its elements, codes and out to 16 "
                                      "bytes, scales to 4");
    if (k == 0)
        return lt_fp8_matmul(nullptr, nullptr, nullptr, nullptr, m, n, k, out, out_dtype,
                             out_stride, nullptr, 0, stream);
    const LinearLayout l = linear_layout(m, n, k);
    if (m > kFewValues && (!workspace || !host::aligned(workspace, 256) || workspace_bytes < l.total))
        return fail(LT_ERR_WORKSPACE, "workspace must be 256-byte aligned and hold " +
                                          std::to_string(l.total) + " bytes");
    const size_t out_bytes = span_bytes(m, n, out_stride, out_dtype);
    if (host::overlaps(out, out_bytes, x, span_bytes(m, k, x_stride, dtype)) ||
        host::overlaps(out, out_bytes, w_codes, size_t(n) * size_t(code_pitch(k))) ||
        host::overlaps(out, out_bytes, w_scales, size_t(n) * size_t(scale_pitch(k))))
        return fail(LT_ERR_INVALID_ARG, "out overlaps x or the weight");
    if (m <= kFewValues) {
        const FewArgs f{w_codes, w_scales, x, nullptr, m, n, k, code_pitch(k), scale_pitch(k),
                        x_stride, int(host::ceil_div(k, kGroup)), out, out_stride};
        const bool f32 = out_dtype == LT_DTYPE_F32;
        const hipStream_t st = static_cast<hipStream_t>(stream);
        int cus;
        if (lt_err e = host::compute_units(&cus))
            return e;
        if (dtype == LT_DTYPE_F32)
            launch_few_tokens<kF32>(f, f32, cus, st);
        else
            launch_few_tokens<kBf16>(f, f32, cus, st);
        LT_TRY_HIP(hipGetLastError());
        return LT_OK;
    }
    auto* ws = static_cast<uint8_t*>(workspace);
    if (lt_err e = host::workspace_written(ws, l.total, static_cast<hipStream_t>(stream)))
        return e;
    if (lt_err e = launch_quantize(x, dtype, m, k, x_stride, false, ws, ws + l.scales, nullptr,
                                   nullptr, static_cast<hipStream_t>(stream)))
        return e;
    return lt_fp8_matmul(ws, ws + l.scales, w_codes, w_scales, m, n, k, out, out_dtype, out_stride,
                         ws + l.matmul, l.total - l.matmul, stream);
} catch (...) {
    return host::caught();
}

}  // extern "C"
