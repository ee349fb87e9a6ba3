// gated.h -- what the gated projections in bf16 (gated.hip) and in 8-bit integers (int8.hip)
// share: the activations, stores, and how a product is cut into tiles and slices.
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
// z * log2(e) is rounded before, and log2(e) is a float 0.23 * 2^-24 off, which makes it 1.23 |z| *
// 2^-24 relative.
__device__ inline float logistic(float z)
{
    return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(z * -1.44269504f));
}

// Phi(-s) = e^(-s^2/2) t P(t) for s >= 0 with t = 1 / (1 + 0.35 s): the function beside the power
// falls slowly and smoothly, and P, of degree 8, is its fit with the least largest relative error on
// 0 <= s <= 14.5 (least squares, reweighted by the errors): 5.8e-8 with these coefficients, which
// are floats, 3.2e-8 before.  In fp32 within (1.12 s^2 + 15) * 2^-24, mostly the power's argument
// (a square, a constant 0.23 * 2^-24 off and a product); 0 from 13.2 on, where s Phi(-s) is below
// 2e-38.  4096
// x 2048 x 11008 in integers 228 us, with the library's erfc 279; kept in bf16 346 and 386.
__device__ inline float tail(float s, float power)
{
    const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(0.35f, s, 1.0f));
    float p = -0.0291580297f;
    p = __builtin_fmaf(p, t, 0.144031614f);
    p = __builtin_fmaf(p, t, -0.255840391f);
    p = __builtin_fmaf(p, t, 0.159321249f);
    p = __builtin_fmaf(p, t, -0.0232133921f);
    p = __builtin_fmaf(p, t, 0.105552927f);
    p = __builtin_fmaf(p, t, 0.119821183f);
    p = __builtin_fmaf(p, t, 0.139863536f);
    p = __builtin_fmaf(p, t, 0.139621302f);
    return p * t * power;
}

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
        const float power = __builtin_amdgcn_exp2f(g * g * -0.72134752f);  // e^(-g^2/2)
        const float below = tail(fabsf(g), power);
        const float p = g < 0.0f ? below : 1.0f - below;  // no difference where it would cancel
        *slope = __builtin_fmaf(g * 0.398942280f, power, p);
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

// Tokens of an instruction.  Above these, tiles: 32 tokens in two passes of the instruction took 30
// us through 2048 x 11008 (bf16, gated), by tiles 19; in integers 14 and 11.
constexpr int64_t kFewTokens = 16;

// ------------------------------------------------------------- tiles

struct Way {
    int tile;    // 256, 128 or 64
    int slices;  // of the sum
    int slice;   // steps of each
};

// What a tile costs, in microseconds: a step of one that has a CU to itself, of one among as many
// as a CU takes, and what is beside the steps.  `places`: how many that is.
struct Cost {
    int tile, places;
    double alone, full, rest;
};

constexpr Cost kCosts[] = {{256, 1, 1.27, 1.27, 18.5}, {128, 2, 0.59, 0.52, 2.4},
                           {64, 4, 0.44, 0.28, 0.8}};
constexpr Cost kPairCosts[] = {{256, 1, 1.37, 1.37, 14.5}, {128, 2, 0.62, 0.57, 1.3},
                               {64, 3, 0.51, 0.42, 0.5}};

// The tile and the slices of the sum that a launch is expected to end first with.  The CU with the
// most tiles sets the time of the steps; the weights come at 6.2 TB/s (those that the last cache
// holds count in) where all CUs have as much to read, and later the more that differs; slices cost
// another launch and their sums' way to memory and back (5.8 TB/s).  Fitted to 628 products of 32 to
// 8192 rows, 768 to 17408 columns and 1024 to 17408 summed values in both types, each by all tiles
// and up to 24 slices: the choice is 0.6% from the best on average, 7% or more for 20 of them and 23%
// at most.  Without the reading and the rounds that share a CU it was 5% and up to twice as long: 512
// x 5120 x 5120 gated in bf16 103 us for 67, 128 x 17408 x 5120 in integers 64 for 38; without slices
// of a pair's sums 64 x 11008 x 2048 gated in bf16 53 for 23.
// `pair`: a tile's columns are two weights'.
inline Way way_of(int64_t m, int64_t n, int steps, bool pair)
{
    Way best{64, 1, steps};
    if (steps <= 0)
        return best;
    const int weights = pair ? 2 : 1, most_slices = std::min(24, std::max(1, steps / 8));
    const double reading = double(n) * steps * tiles::kStepBytes * weights / 6.2e6;
    double least = 1e300;
    for (const Cost& c : pair ? kPairCosts : kCosts) {
        const int64_t wide = pair && c.tile > 64 ? c.tile / 2 : c.tile;
        const int64_t tiles = (m + c.tile - 1) / c.tile * ((n + wide - 1) / wide);
        for (int z = 1; z <= most_slices; ++z) {
            const int slice = (steps + z - 1) / z, slices = (steps + slice - 1) / slice;
            const double sums = double(slices) * double(m) * double(n) * weights * 4;
            if (z > 1 && (slice < 8 || slices != z || sums > 2.7e8))
                continue;
            const int64_t groups = tiles * slices, each = (groups + 255) / 256;
            const double step =
                std::max(c.alone * double((each + c.places - 1) / c.places), c.full * double(each));
            const double apart = double(each * 256) / double(groups) - 1.0;
            const double us = std::max(step * slice + c.rest * double(each),
                                       reading * (1.0 + 0.68 * apart)) +
                              (z > 1 ? 6.7 + 2.0 * sums / 5.8e6 : 0.0);
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
