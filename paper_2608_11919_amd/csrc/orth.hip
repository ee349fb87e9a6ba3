// orth.hip -- Newton-Schulz orthogonalisation of a list of matrices, and the Muon step.
//
// X_0 = U / ||U||_F; five times (ns_steps) A = X X^T, B = b A + c A A, X = a X + B X, on the
// side of the smaller dimension (A = X^T X and X B where there are more rows than columns).
// The singular values of X_0 lie in [0, 1], those of every later X in [0, 1.203]: the
// polynomial's largest value on [0, 1.203] is f(0.5545) = 1.2024.  Hence |A| <= 1.446 and
// |B| <= 2.81, and powers of two place every operand in fp16's range: X times 2^15, A and B
// times 2^14.
//
// Products take fp16 operands and sum in fp32.  fp16 has three bits more than bf16 at the
// same rate.  The linear term a X reads X as a sum of two fp16 numbers: directions whose
// singular values are far below the largest grow by a factor of a in every step, and one
// fp16 number loses them against the large ones.  Simulated for Gaussian matrices of 64 to
// 1024 rows: 1.2e-3 to 2.0e-3 off in 2-norm (bf16 operands: 1.1e-2 to 1.6e-2); for eight strong
// directions over noise 1.3e-4 (one fp16 X: 1.4e-2, bf16: 0.12).
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

namespace {

using host::fail;
using host::Guard;
using host::round_up;
using namespace tiles;

constexpr float kA = 3.4445f, kB = -4.7750f, kC = 2.0315f;
constexpr float kScaleX = 32768.0f;               // X is stored times 2^15
constexpr float kGramOut = 1.0f / 65536.0f;       // (2^15)^2 -> 2^14
constexpr float kSquareOut = kC / 16384.0f;       // (2^14)^2 -> 2^14
constexpr float kUpdateOut = 1.0f / 16384.0f;     // 2^14 * 2^15 -> 2^15
constexpr int kTile = 128;                        // output tile, and what sizes are padded to
constexpr int kThreads = 256;
constexpr int kPrep = 64;                         // tile of the transposing pass

struct Matrix {
    const void* src;           // the matrix, or the Muon step's update in fp32
    _Float16 *h[2], *t[2], *l[2];
    _Float16 *a, *b;
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
    for (int64_t e = e0 + threadIdx.x; e < e1; e += kThreads) {
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

template <typename T>
__global__ __launch_bounds__(kThreads) void k_orth_prepare(Gate gate,
                                                           const int64_t* __restrict__ prefix,
                                                           const Matrix* __restrict__ mats,
                                                           int first, int n)
{
    __shared__ _Float16 turned[kPrep][kPrep + 2];
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
    const int c = int(threadIdx.x) & 63;
    for (int r = int(threadIdx.x) >> 6; r < kPrep; r += kThreads / 64) {
        const int row = r0 + r, col = c0 + c;
        float x = 0.0f;
        if (row < m.rows && col < m.cols)
            x = float(double(load_value(src + int64_t(row) * m.cols + col)) * by);
        const _Float16 hi = _Float16(x);
        const int64_t at = int64_t(row) * m.cp + col;
        m.h[0][at] = hi;
        m.l[0][at] = _Float16(x - float(hi));
        turned[c][r] = hi;
    }
    __syncthreads();
    for (int q = int(threadIdx.x) >> 6; q < kPrep; q += kThreads / 64)
        m.t[0][int64_t(c0 + q) * m.rp + r0 + c] = turned[q][c];
}

// ------------------------------------------------------------- products

// One 128 x 128 output tile by four waves of 64 x 64; a lane ends with
// acc[i][j][r] = C[64 * (wave / 2) + 16 i + lane % 16][64 * (wave % 2) + 16 j + 4 (lane / 16) + r]
// (the operands are swapped in the instruction, so that a lane holds consecutive columns).
struct TileAcc {
    f32x4 v[4][4];
};

__device__ inline void tile_step(const uint8_t* p, const uint8_t* q, int wave, int lane,
                                 TileAcc& acc)
{
    i32x4 a[4][2], b[4][2];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        read_chunks(p, 64 * (wave >> 1) + 16 * i, lane, a[i]);
        read_chunks(q, 64 * (wave & 1) + 16 * i, lane, b[i]);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j)
            acc.v[i][j] = Half::mul<0>(b[j], a[i], acc.v[i][j]);
}

// P and Q: the tiles' first rows; steps >= 1 of 128 bytes.
__device__ inline void tile_product(const _Float16* P, int64_t pitch_p, const _Float16* Q,
                                    int64_t pitch_q, int steps, uint8_t* lds, TileAcc& acc)
{
    constexpr int kHalf = 2 * kTile * kStepBytes;
    const int lane = int(threadIdx.x) & 63;
    const int wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x) >> 6);
    TileLoad<kTile, kThreads> load_p, load_q;
    load_p.init(pitch_p * 2, kTile);
    load_q.init(pitch_q * 2, kTile);
    const auto* p = reinterpret_cast<const uint8_t*>(P);
    const auto* q = reinterpret_cast<const uint8_t*>(Q);
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j)
            acc.v[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    load_p.issue(p, lds);
    load_q.issue(q, lds + kTile * kStepBytes);
    for (int s = 0; s < steps; ++s) {
        uint8_t* now = lds + (s & 1) * kHalf;
        uint8_t* next = lds + (~s & 1) * kHalf;
        wait_loads();
        __syncthreads();  // the step's tiles are in place, and no wave reads the other buffer
        if (s + 1 < steps) {
            load_p.issue(p + int64_t(s + 1) * kStepBytes, next);
            load_q.issue(q + int64_t(s + 1) * kStepBytes, next + kTile * kStepBytes);
        }
        tile_step(now, now + kTile * kStepBytes, wave, lane, acc);
    }
}

// A = X X^T (or X^T X), or B = b A + c A A: symmetric, tiles on and above the diagonal, each
// stored on both sides.
template <bool SQUARE>
__global__ __launch_bounds__(kThreads) void k_orth_gram(Gate gate,
                                                        const int64_t* __restrict__ prefix,
                                                        const Matrix* __restrict__ mats, int first,
                                                        int n, int from)
{
    __shared__ __align__(1024) uint8_t lds[4 * kTile * kStepBytes];
    if (!descriptors_ok(gate) || !step_applies(gate))
        return;
    const int64_t unit = prefix[first] + blockIdx.x;
    const int k = find_matrix(prefix, first, n, unit);
    const Matrix& m = mats[k];
    const bool wide = m.rows <= m.cols;
    const int side = wide ? m.rp : m.cp, inner = SQUARE ? side : (wide ? m.cp : m.rp);
    // the tile's place in the upper triangle, row by row
    const int count = side / kTile;
    int left = int(unit - prefix[k]), ti = 0;
    while (left >= count - ti) {
        left -= count - ti;
        ++ti;
    }
    const int tj = ti + left;
    const _Float16* x = SQUARE ? m.a : (wide ? m.h[from] : m.t[from]);
    TileAcc acc;
    tile_product(x + int64_t(ti) * kTile * inner, inner, x + int64_t(tj) * kTile * inner, inner,
                 inner / 64, lds, acc);
    const int lane = int(threadIdx.x) & 63, wave = int(threadIdx.x) >> 6;
    _Float16* out = SQUARE ? m.b : m.a;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int row = ti * kTile + 64 * (wave >> 1) + 16 * i + (lane & 15);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int col = tj * kTile + 64 * (wave & 1) + 16 * j + 4 * (lane >> 4);
            const int64_t at = int64_t(row) * side + col;
            typedef _Float16 half4 __attribute__((ext_vector_type(4)));
            half4 v, old = {};
            if constexpr (SQUARE)
                old = *reinterpret_cast<const half4*>(m.a + at);
#pragma unroll
            for (int r = 0; r < 4; ++r)
                v[r] = _Float16(SQUARE ? kSquareOut * acc.v[i][j][r] + kB * float(old[r])
                                       : kGramOut * acc.v[i][j][r]);
            *reinterpret_cast<half4*>(out + at) = v;
            if (ti != tj) {
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    out[int64_t(col + r) * side + row] = v[r];
            }
        }
    }
}

enum Final { kNext, kOutF32, kOutBf16, kWeights };

// X' = a X + B X (or a X + X B): the next X, or where it goes.
template <int FINAL>
__global__ __launch_bounds__(kThreads) void k_orth_update(Gate gate,
                                                          const int64_t* __restrict__ prefix,
                                                          const Matrix* __restrict__ mats,
                                                          int first, int n, int from, float decay)
{
    __shared__ __align__(1024) uint8_t lds[4 * kTile * kStepBytes];
    if (!descriptors_ok(gate))
        return;
    const bool applies = step_applies(gate);
    if (!applies && FINAL != kWeights)
        return;
    const int64_t unit = prefix[first] + blockIdx.x;
    const int k = find_matrix(prefix, first, n, unit);
    const Matrix& m = mats[k];
    const bool wide = m.rows <= m.cols;
    const int across = m.cp / kTile, tile = int(unit - prefix[k]);
    const int r0 = tile / across * kTile, c0 = tile % across * kTile;
    const int lane = int(threadIdx.x) & 63, wave = int(threadIdx.x) >> 6;
    TileAcc acc;
    if (applies) {
        const int inner = wide ? m.rp : m.cp;
        const _Float16* P = (wide ? m.b : m.h[from]) + int64_t(r0) * inner;
        const _Float16* Q = (wide ? m.t[from] : m.b) + int64_t(c0) * inner;
        tile_product(P, inner, Q, inner, inner / 64, lds, acc);
    } else if (!m.wb) {
        return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int row = r0 + 64 * (wave >> 1) + 16 * i + (lane & 15);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int col = c0 + 64 * (wave & 1) + 16 * j + 4 * (lane >> 4);
            const int64_t at = int64_t(row) * m.cp + col;
            typedef _Float16 half4 __attribute__((ext_vector_type(4)));
            float v[4] = {};
            if (applies) {
                const half4 h = *reinterpret_cast<const half4*>(m.h[from] + at);
                const half4 l = *reinterpret_cast<const half4*>(m.l[from] + at);
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    v[r] = kUpdateOut * acc.v[i][j][r] + kA * (float(h[r]) + float(l[r]));
            }
            if constexpr (FINAL == kNext) {
                half4 h, l;
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    h[r] = _Float16(v[r]);
                    l[r] = _Float16(v[r] - float(h[r]));
                    m.t[from ^ 1][int64_t(col + r) * m.rp + row] = h[r];
                }
                *reinterpret_cast<half4*>(m.h[from ^ 1] + at) = h;
                *reinterpret_cast<half4*>(m.l[from ^ 1] + at) = l;
            } else {
                if (row >= m.rows)
                    continue;
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    if (col + r >= m.cols)
                        continue;
                    const int64_t to = int64_t(row) * m.cols + col + r;
                    const float o = v[r] * (1.0f / kScaleX);
                    if constexpr (FINAL == kOutF32) {
                        static_cast<float*>(m.out)[to] = o;
                    } else if constexpr (FINAL == kOutBf16) {
                        static_cast<uint16_t*>(m.out)[to] = bf16_bits(o);
                    } else {
                        float w = m.w[to];
                        if (applies) {
                            w = __builtin_fmaf(-m.rate, o, w * decay);
                            m.w[to] = w;
                        }
                        if (m.wb)
                            m.wb[to] = bf16_bits(w);
                    }
                }
            }
        }
    }
}

// ---------------------------------------------------------------- host side

// The workspace: [tag][prefixes][momentum descriptors][matrices][square sums][partials] and
// the region that the batches share.
constexpr int64_t kBatchElems = int64_t(1) << 27;  // padded elements of a batch of several

enum { kPreUnits, kPrePrep, kPreGram, kPreTile, kPrefixes };

struct Plan {
    size_t prefix[kPrefixes], momentum, mats, header, squares, partials, region, total;
    std::vector<int> batch;  // first matrix of each batch, and the list's length
};

int64_t padded(int64_t x) { return int64_t(round_up(size_t(x), kTile)); }

int64_t units_of(int64_t numel, int64_t span) { return (numel + span - 1) / span; }

// Bytes of a matrix in the region: X in three layouts twice, A and B, the Muon step's update.
struct Place {
    size_t h[2], t[2], l[2], a, b, u, bytes;
};

Place place(int64_t rows, int64_t cols, bool muon)
{
    Place p;
    const size_t x = round_up(size_t(padded(rows)) * size_t(padded(cols)) * 2, 256);
    const size_t side = size_t(std::min(padded(rows), padded(cols)));
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
    p.a = take(side * side * 2);
    p.b = take(side * side * 2);
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
    int64_t units = 0, elems = 0;
    size_t region = 0, bytes = 0;
    for (int k = 0; k < K; ++k) {
        if (rows[k] == 0 || cols[k] == 0) {
            if (p.batch.empty())
                p.batch.push_back(k);
            continue;
        }
        units += units_of(rows[k] * cols[k], span);
        const int64_t n = padded(rows[k]) * padded(cols[k]);
        if (p.batch.empty() || (elems > 0 && elems + n > kBatchElems)) {
            p.batch.push_back(k);
            elems = 0;
            bytes = 0;
        }
        elems += n;
        bytes += place(rows[k], cols[k], muon).bytes;
        region = std::max(region, bytes);
    }
    p.batch.push_back(K);
    p.region = p.partials + round_up(sizeof(double) * size_t(units), 256);
    p.total = round_up(p.region + region, 256);
    return p;
}

// Sizes a call can take: rows and columns in [0, 2^23), so that 128 rows of the widest matrix
// stay within the 32-bit offsets of a tile's loads.
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
        uint8_t* at = ws + p.region;
        for (int k = p.batch[b]; k < p.batch[b + 1]; ++k) {
            const int64_t numel = c.rows[k] * c.cols[k];
            Matrix& m = mats[k];
            int64_t prep = 0, gram = 0, tile = 0;
            if (numel > 0) {
                const Place x = place(c.rows[k], c.cols[k], c.muon);
                for (int i = 0; i < 2; ++i) {
                    m.h[i] = reinterpret_cast<_Float16*>(at + x.h[i]);
                    m.t[i] = reinterpret_cast<_Float16*>(at + x.t[i]);
                    m.l[i] = reinterpret_cast<_Float16*>(at + x.l[i]);
                }
                m.a = reinterpret_cast<_Float16*>(at + x.a);
                m.b = reinterpret_cast<_Float16*>(at + x.b);
                m.partial = partial;
                m.square = reinterpret_cast<double*>(ws + p.squares) + k;
                m.rows = int32_t(c.rows[k]);
                m.cols = int32_t(c.cols[k]);
                m.rp = int32_t(padded(c.rows[k]));
                m.cp = int32_t(padded(c.cols[k]));
                m.units = int32_t(units_of(numel, c.span));
                fill(k, m, momentum[c.muon ? k : 0], reinterpret_cast<float*>(at + x.u));
                partial += m.units;
                at += x.bytes;
                const int64_t side = std::min(m.rp, m.cp) / kTile;
                prep = int64_t(m.rp / kPrep) * (m.cp / kPrep);
                gram = side * (side + 1) / 2;
                tile = int64_t(m.rp / kTile) * (m.cp / kTile);
            }
            pre[kPreUnits][k + 1] = pre[kPreUnits][k] + m.units;
            pre[kPrePrep][k + 1] = pre[kPrePrep][k] + prep;
            pre[kPreGram][k + 1] = pre[kPreGram][k] + gram;
            pre[kPreTile][k + 1] = pre[kPreTile][k] + tile;
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
    const hipStream_t st = c.st;
    for (size_t b = 0; b + 1 < p.batch.size(); ++b) {
        const int first = p.batch[b], n = p.batch[b + 1] - first;
        const auto blocks = [&](int i) { return pre[i][first + n] - pre[i][first]; };
        if (n == 0 || blocks(kPreTile) == 0)
            continue;
        const dim3 tiles_(uint32_t(blocks(kPreTile))), grams(uint32_t(blocks(kPreGram)));
        if (lt_err e = begin(gate, dev[kPreUnits], d_momentum, d_mats, first, n,
                             pre[kPreUnits][first], blocks(kPreUnits)))
            return e;
        k_orth_norm<<<dim3(uint32_t(n)), kThreads, 0, st>>>(gate, d_mats, first);
        const bool wide_src = c.muon || c.in_dtype == LT_DTYPE_F32;
        auto* prep = wide_src ? k_orth_prepare<float> : k_orth_prepare<uint16_t>;
        prep<<<dim3(uint32_t(blocks(kPrePrep))), kThreads, 0, st>>>(gate, dev[kPrePrep], d_mats,
                                                                    first, n);
        auto* last = c.muon ? k_orth_update<kWeights>
                            : (c.out_dtype == LT_DTYPE_F32 ? k_orth_update<kOutF32>
                                                           : k_orth_update<kOutBf16>);
        for (int s = 0; s < c.ns_steps; ++s) {
            const int from = s & 1;
            k_orth_gram<false><<<grams, kThreads, 0, st>>>(gate, dev[kPreGram], d_mats, first, n,
                                                           from);
            k_orth_gram<true><<<grams, kThreads, 0, st>>>(gate, dev[kPreGram], d_mats, first, n,
                                                          from);
            auto* update = s + 1 < c.ns_steps ? k_orth_update<kNext> : last;
            update<<<tiles_, kThreads, 0, st>>>(gate, dev[kPreTile], d_mats, first, n, from,
                                                decay);
        }
        LT_TRY_HIP(hipGetLastError());
    }
    return LT_OK;
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
{
    return valid_sizes(rows, cols, n_matrices)
               ? make_plan(rows, cols, n_matrices, false, kSquareUnit).total
               : 0;
}

lt_err lt_orthogonalize(const void* const* matrices, int in_dtype, void* const* out, int out_dtype,
                        const int64_t* rows, const int64_t* cols, int n_matrices, int ns_steps,
                        void* workspace, size_t workspace_bytes, void* stream)
{
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
            const Matrix* mats, int first, int n, int64_t, int64_t units) {
            auto* squares = in_dtype == LT_DTYPE_F32 ? k_orth_squares<float>
                                                     : k_orth_squares<uint16_t>;
            squares<<<dim3(uint32_t(units)), kThreads, 0, c.st>>>(gate, prefix, mats, first, n);
            LT_TRY_HIP(hipGetLastError());
            return LT_OK;
        });
}

size_t lt_muon_workspace_bytes(const int64_t* rows, const int64_t* cols, int n_matrices,
                               int block_size)
{
    return valid_sizes(rows, cols, n_matrices) && host::valid_block_size(block_size)
               ? make_plan(rows, cols, n_matrices, true, host::momentum_unit(block_size)).total
               : 0;
}

lt_err lt_muon_step(float* const* params, const void* const* grads, int grad_dtype,
                    int8_t* const* m_codes, float* const* m_absmax, uint16_t* const* params_bf16,
                    const int64_t* rows, const int64_t* cols, int n_matrices, int block_size,
                    int code_map, double lr, double momentum, int nesterov, double weight_decay,
                    double update_rms, int ns_steps, const float* coef, const int32_t* status,
                    const void* step_state, void* workspace, size_t workspace_bytes, void* stream)
{
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
            const Matrix*, int first, int n, int64_t first_unit, int64_t units) {
            return host::launch_momentum(gate.guard, prefix, momenta, first, n, first_unit, units,
                                         grad_dtype, block_size, code_map, s, coef, status,
                                         step_state, c.st);
        });
}

}  // extern "C"
