// gated.h -- what the gated projections in bf16 (gated.hip) and in 8-bit integers (int8.hip)
// share: the activations, and products of few tokens with one or two weights.
#ifndef LAZYTRAIN_GATED_H
#define LAZYTRAIN_GATED_H

#include <algorithm>

#include "lazytrain.h"
#include "tiles.h"

namespace gated {

using tiles::f32x4;
using tiles::i32x4;

typedef uint16_t u16x8 __attribute__((ext_vector_type(8)));

__device__ inline uint16_t bf16_bits(float x)
{
    return __builtin_bit_cast(uint16_t, (__bf16)x);  // to nearest even; a NaN becomes quiet
}

// 1 / (1 + e^-z), from the hardware's power of two and reciprocal, one unit in the last place each:
// z * log2(e) is rounded before, which makes it |z| * 2^-24 relative.
__device__ inline float logistic(float z)
{
    return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(z * -1.44269504f));
}

// g Phi(g) through the complementary error function: 1 + erf(g / sqrt 2) cancels for negative g.
__device__ inline float normal_cdf(float g) { return 0.5f * erfcf(g * -0.70710678f); }

constexpr float kTanhLinear = 1.59576912f;   // 2 sqrt(2 / pi)
constexpr float kTanhCubic = 0.0713548163f;  // that times 0.044715

struct Silu {
    __device__ static inline float of(float g, float* slope)
    {
        const float s = logistic(g);
        *slope = s * __builtin_fmaf(g, 1.0f - s, 1.0f);
        return g * s;
    }
};

struct Gelu {
    __device__ static inline float of(float g, float* slope)
    {
        const float p = normal_cdf(g);
        *slope = __builtin_fmaf(
            g * 0.398942280f, __builtin_amdgcn_exp2f(g * g * -0.72134752f), p);  // g e^(-g^2/2)
        return g * p;
    }
};

struct GeluTanh {  // 0.5 g (1 + tanh(z / 2)) = g / (1 + e^-z)
    __device__ static inline float of(float g, float* slope)
    {
        const float s = logistic(g * __builtin_fmaf(kTanhCubic * g, g, kTanhLinear));
        // beyond 100 the second term is 0, and its factors might not fit
        const float c = fminf(fmaxf(g, -100.0f), 100.0f);
        *slope = __builtin_fmaf(c * (s * (1.0f - s)),
                                __builtin_fmaf(3.0f * kTanhCubic * c, c, kTanhLinear), s);
        return g * s;
    }
};

struct Relu {
    __device__ static inline float of(float g, float* slope)
    {
        *slope = g <= 0.0f ? 0.0f : 1.0f;
        return g <= 0.0f ? 0.0f : g;
    }
};

// The activation and its derivative of N values.  `kind` is the same for a whole launch: a branch,
// not a kernel for each, and one for all N, whose chains of instructions then overlap.
template <int N>
__device__ inline void activate(int kind, const float (&g)[N], float (&y)[N], float (&slope)[N])
{
    const auto all = [&](auto act) {
#pragma unroll
        for (int e = 0; e < N; ++e)
            y[e] = act.of(g[e], &slope[e]);
    };
    if (kind == LT_ACT_SILU)
        all(Silu());
    else if (kind == LT_ACT_GELU)
        all(Gelu());
    else if (kind == LT_ACT_GELU_TANH)
        all(GeluTanh());
    else
        all(Relu());
}

template <int N>
__device__ inline void activate(int kind, const float (&g)[N], float (&y)[N])
{
    float unused[N];
    activate(kind, g, y, unused);
}

// Eight results of a row, wherever it begins; those from `left` on do not exist.
template <bool F32>
__device__ inline void store_row(void* out, int64_t at, const float (&v)[8], int64_t left)
{
    if (left >= 8) {
        if constexpr (F32) {
            float* p = static_cast<float*>(out) + at;
            tiles::store_any(p, f32x4{v[0], v[1], v[2], v[3]});
            tiles::store_any(p + 4, f32x4{v[4], v[5], v[6], v[7]});
        } else {
            u16x8 b;
#pragma unroll
            for (int e = 0; e < 8; ++e)
                b[e] = bf16_bits(v[e]);
            tiles::store_any(static_cast<uint16_t*>(out) + at, b);
        }
        return;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e)
        if (e < left) {
            if constexpr (F32)
                static_cast<float*>(out)[at + e] = v[e];
            else
                static_cast<uint16_t*>(out)[at + e] = bf16_bits(v[e]);
        }
}

// ------------------------------------------------------------- few tokens

// Instructions of 16 rows x 16 tokens: a lane holds 16 bytes of row or token l % 16, and ends
// with rows 4 (l / 16) + e of token l % 16.
struct FewBf16 {
    typedef f32x4 Acc;
    __device__ static inline Acc mul(i32x4 w, i32x4 x, Acc c)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(tiles::bf16x8, w),
                                                       __builtin_bit_cast(tiles::bf16x8, x), c, 0,
                                                       0, 0);
    }
};

struct FewInt8 {
    typedef i32x4 Acc;
    __device__ static inline Acc mul(i32x4 w, i32x4 x, Acc c)
    {
        return __builtin_amdgcn_mfma_i32_16x16x64_i8(w, x, c, 0, 0, 0);
    }
};

struct FewArgs {
    const uint8_t* w[2];    // one or two weights, rows of k values
    int64_t w_pitch[2];     // bytes
    const uint8_t* x;
    int64_t x_pitch;
    const float* w_scales[2];  // integers
    const float* x_scales;
    int64_t m, n;
    int64_t bytes;          // of a row's values
    int activation;
    void* out;
    int64_t stride;
};

constexpr int kFewStep = 128;  // bytes of every row

// 32 bytes of a row from byte `at` on; what lies behind its end is 0 (WHOLE: nothing does).
template <bool WHOLE>
__device__ inline void few_load(const uint8_t* row, int64_t at, int64_t bytes, i32x4 (&v)[2])
{
    if (WHOLE || at + 32 <= bytes) {
        v[0] = tiles::load_any(row + at);
        v[1] = tiles::load_any(row + at + 16);
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

// Results for up to 16 tokens, 16 rows of each of the B weights to a workgroup, bound by
// reading the weights once: no LDS tiles, every lane loads its bytes of the instruction's rows
// straight from HBM, and the waves cut the sum into runs of neighbouring steps.
template <typename Mul, int B, bool F32>
__global__ __launch_bounds__(512) void k_few(FewArgs g)
{
    extern __shared__ f32x4 few_sums[];  // [wave][B][lane], of 16 bytes
    constexpr bool kInt = std::is_same<Mul, FewInt8>::value;
    typedef typename Mul::Acc Acc;
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
    Acc acc[B] = {};
    struct Loaded {
        i32x4 w[B][2], x[2];
    };
    const auto load = [&](int s, Loaded& in) {
        const int64_t at = int64_t(s) * kFewStep + 32 * q;
#pragma unroll
        for (int b = 0; b < B; ++b)
            few_load<kInt>(w[b], at, g.bytes, in.w[b]);
        few_load<kInt>(x, at, g.bytes, in.x);
    };
    const auto multiply = [&](const Loaded& in) {
#pragma unroll
        for (int c = 0; c < 2; ++c)
#pragma unroll
            for (int b = 0; b < B; ++b)
                acc[b] = Mul::mul(in.w[b][c], in.x[c], acc[b]);
    };
    const int steps = int((g.bytes + kFewStep - 1) / kFewStep);
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
        few_sums[(wave * B + b) * 64 + lane] = __builtin_bit_cast(f32x4, acc[b]);
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
        if constexpr (kInt) {
            int s = 0;
            for (int i = 0; i < waves; ++i)
                s += __float_as_int(from[i * B * 256]);
            v[b] = float(s) * g.x_scales[tok] * g.w_scales[b][row];
        } else {
            float s = from[0];
            for (int i = 1; i < waves; ++i)
                s += from[i * B * 256];
            v[b] = s;
        }
    }
    float y = v[0];
    if constexpr (B == 2) {
        const float u[1] = {v[0]};
        float a[1];
        activate(g.activation, u, a);
        y = a[0] * v[1];
    }
    if constexpr (F32)
        static_cast<float*>(g.out)[tok * g.stride + row] = y;
    else
        static_cast<uint16_t*>(g.out)[tok * g.stride + row] = bf16_bits(y);
}

// Above these, tiles: 32 tokens in two passes of the instruction took 30 us through 2048 x 11008
// (bf16, gated), 48 by tiles 19; in integers 14 and 11.
constexpr int64_t kFewTokens = 16;

template <typename Mul, int B>
void launch_few(const FewArgs& g, bool f32, hipStream_t st)
{
    const int64_t steps = (g.bytes + kFewStep - 1) / kFewStep;
    const int waves = steps >= 8 ? 8 : 4;
    auto* kernel = f32 ? k_few<Mul, B, true> : k_few<Mul, B, false>;
    kernel<<<dim3(uint32_t((g.n + 15) / 16)), 64 * waves, size_t(waves) * B * 1024, st>>>(g);
}

// ------------------------------------------------------------- tiles

struct Way {
    int tile;    // 256, 128 or 64
    int slices;  // of the sum
    int slice;   // steps of each
};

// What a tile costs a CU, in microseconds: each step, and beside its steps.
struct Cost {
    int tile;
    double step, rest;
};

constexpr Cost kCosts[] = {{256, 1.33, 14.0}, {128, 0.5, 2.0}, {64, 0.18, 0.6}};
constexpr Cost kPairCosts[] = {{256, 1.33, 14.0}, {128, 0.5, 2.0}, {64, 0.29, 1.0}};

// The tile and the slices of the sum that a launch is expected to end first with.  The CU with the
// most tiles sets its time; a tile costs so many microseconds a step and beside its steps, and
// slices another launch and their sums' way to memory and back (4 TB/s).  Fitted to products of 16
// to 8192 rows, 1024 to 5120 summed values and 1024 to 17408 columns in both types, where the
// choice is within 10% of the best tile but for a few (23% at most); the largest tile wherever it
// gives every CU one was up to twice as slow (1536 x 2048 x 11008 in integers 61 us, by tiles of
// 128 45; 768 x 2048 x 11008 gated in bf16 92 and 75; 3500 x 4096 x 1024 28 and 20).
// `pair`: a tile's columns are two weights'; such sums are not cut.
inline Way way_of(int64_t m, int64_t n, int64_t count, int steps, bool pair)
{
    Way best{64, 1, steps};
    if (steps <= 0)
        return best;
    double least = 1e300;
    for (const Cost& c : pair ? kPairCosts : kCosts) {
        const int64_t wide = pair && c.tile > 64 ? c.tile / 2 : c.tile;
        const int64_t tiles = (m + c.tile - 1) / c.tile * ((n + wide - 1) / wide) * count;
        const int most_slices = pair ? 1 : std::min(64, std::max(1, steps / 8));
        for (int z = 1; z <= most_slices; ++z) {
            const int slice = (steps + z - 1) / z, slices = (steps + slice - 1) / slice;
            const double sums = double(slices) * double(m) * double(n) * double(count) * 4;
            if (z > 1 && (slice < 8 || slices != z || sums > 2.7e8))
                continue;
            const double most = double((tiles * slices + 255) / 256);
            const double us =
                most * (c.step * slice + c.rest) + (z > 1 ? 5.0 + 2.0 * sums / 4e6 : 0.0);
            if (us < least) {
                least = us;
                best = Way{c.tile, slices, slice};
            }
        }
    }
    return best;
}

}  // namespace gated

#endif
