// momentum.hip -- the momentum pass of the Muon step: decode, update, the update's
// direction with its sum of squares, requantize.  Part of library.hip (it uses the code
// tables and the loads of lazytrain.hip).
//
// Per element, in fp32 with every product and sum rounded: g = grad * coef,
// m1 = beta * m0 + rest * g, u = beta * m1 + rest * g (Nesterov) or m1.  Per block: the new
// absmax and codes as the 8-bit AdamW step stores a first moment.  u goes to the workspace in
// fp32: its norm is known only when all of it is, so it is read once more either way, and the
// orthogonalisation reads it there.  The pass is bound by HBM: 2 or 4 bytes of gradient, a
// code read and written, 4 bytes of u (67.6M elements with bf16 gradients, block 4096: 115 to
// 133 us, 4.1 to 4.7 TB/s).

namespace {

constexpr int kMomentumSpan = 4096;  // elements of a unit, where a block is no longer
constexpr int kMomentumHeld = kMomentumSpan / (kThreads * kGranule);  // granules a lane keeps

struct MomentumIn {
    float g[8];
    uint32_t m[2];
};

template <typename GT>
__device__ inline void momentum_load(const host::MomentumTensor& d, int64_t at, int nv,
                                     MomentumIn& in)
{
    if (nv >= kGranule) {
        if constexpr (sizeof(GT) == 2) {
            const uint4 q = load16(static_cast<const uint16_t*>(d.g) + at);
            in.g[0] = bf16_lo(q.x); in.g[1] = bf16_hi(q.x);
            in.g[2] = bf16_lo(q.y); in.g[3] = bf16_hi(q.y);
            in.g[4] = bf16_lo(q.z); in.g[5] = bf16_hi(q.z);
            in.g[6] = bf16_lo(q.w); in.g[7] = bf16_hi(q.w);
        } else {
            load8f(static_cast<const float*>(d.g) + at, nv, in.g);
        }
        const uint2 m = load8(d.mq + at);
        in.m[0] = m.x;
        in.m[1] = m.y;
        return;
    }
    in.m[0] = in.m[1] = 0u;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const bool ok = e < nv;
        if constexpr (sizeof(GT) == 2)
            in.g[e] = ok ? bf16_lo(gp(static_cast<const uint16_t*>(d.g))[at + e]) : 0.0f;
        else
            in.g[e] = ok ? gp(static_cast<const float*>(d.g))[at + e] : 0.0f;
        if (ok)
            in.m[e >> 2] |= uint32_t(uint8_t(gp(d.mq)[at + e])) << (8 * (e & 3));
    }
}

template <int MAP>
__device__ inline void momentum_new(const MomentumIn& in, float step, float coef,
                                    const host::MomentumScalars& s, const dyn::LdsTables& tab,
                                    float (&m1)[8], float (&cg)[8])
{
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const uint32_t b = (in.m[e >> 2] >> (8 * (e & 3))) & 0xFFu;
        const float m0 = MAP == kMapLinear ? float(int8_t(b)) * step : tab.dm[b] * step;
        cg[e] = (in.g[e] * coef) * s.rest;
        m1[e] = m0 * s.beta + cg[e];  // contraction is off: product and sum round apart
    }
}

template <int MAP>
__device__ inline void momentum_store(int8_t* mq, int64_t at, int nv, const float (&m1)[8],
                                      float inv, bool ok, const dyn::LdsTables& tab)
{
    uint32_t p[2] = {0u, 0u};
    if (ok) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            uint32_t c;
            if constexpr (MAP == kMapLinear) {
                c = uint32_t(int(fminf(fmaxf(rintf(m1[e] * inv), -127.0f), 127.0f))) & 0xFFu;
            } else {
                c = dyn::encode<dyn::kBaseM, dyn::kTopM>(tab.em, fabsf(m1[e]) * inv);
                c |= m1[e] < 0.0f ? 0x80u : 0u;
            }
            p[e >> 2] |= c << (8 * (e & 3));
        }
    }
    if (nv >= kGranule) {
        *reinterpret_cast<uint2*>(mq + at) = make_uint2(p[0], p[1]);
        return;
    }
    for (int e = 0; e < nv; ++e)
        gp(mq)[at + e] = int8_t(p[e >> 2] >> (8 * (e & 3)));
}

template <typename GT, int MAP>
__global__ __launch_bounds__(kThreads) void k_muon_momentum(
    WsGuard guard, const int64_t* __restrict__ prefix,
    const host::MomentumTensor* __restrict__ desc, int first, int n, int64_t first_unit, int B,
    int64_t span, host::MomentumScalars s, const float* __restrict__ coef_ptr,
    const int32_t* __restrict__ status_ptr, const uint8_t* __restrict__ state)
{
    __shared__ uint32_t top[kMomentumSpan / 64];  // |m1|'s largest pattern, by block
    __shared__ double squares[kThreads / 64];
    __shared__ __align__(16) uint8_t dyn_lds[MAP == kMapDynamic ? sizeof(dyn::LdsTables) : 16];
    const dyn::LdsTables& tab = *reinterpret_cast<const dyn::LdsTables*>(dyn_lds);

    dyn::TableCopy<kThreads> tables;
    if constexpr (MAP == kMapDynamic)
        tables.load();
    StepScalars run = {};
    run.state = state;
    float coef;
    if (!step_runs(guard, run, coef_ptr, status_ptr, &coef))
        return;
    const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
    if (t < kMomentumSpan / 64)
        top[t] = 0u;
    if constexpr (MAP == kMapDynamic)
        tables.store(dyn_lds);
    else
        __syncthreads();

    const int64_t unit = first_unit + blockIdx.x;
    const int k = first + find_tensor_wave(prefix + first, n, unit, lane);
    const host::MomentumTensor d = desc[k];
    const int64_t in_matrix = unit - prefix[k];
    const int64_t e0 = in_matrix * span;
    const int len = int(i64min(span, d.numel - e0));
    const int64_t blk0 = e0 / B;
    const int n_gran = (len + kGranule - 1) / kGranule;

    // pass 1: the new momentum, the update, block maxima
    float held[kMomentumHeld][8];
    double sq = 0.0;
#pragma unroll 1
    for (int gi = t, r = 0; gi < ((n_gran + kThreads - 1) / kThreads) * kThreads;
         gi += kThreads, ++r) {
        const bool mine = gi < n_gran;
        const int o = kGranule * gi;
        const int b = mine ? o / B : 0;  // a granule lies within one block
        float m1[8] = {}, cg[8];
        if (mine) {
            const int nv = min(kGranule, len - o);
            const float a = gp(d.ma)[blk0 + b];
            MomentumIn in;
            momentum_load<GT>(d, e0 + o, nv, in);
            momentum_new<MAP>(in, MAP == kMapLinear ? a / 127.0f : a, coef, s, tab, m1, cg);
            float u[8];
            float most = 0.0f;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                m1[e] = e < nv ? m1[e] : 0.0f;
                u[e] = s.nesterov ? m1[e] * s.beta + cg[e] : m1[e];
                u[e] = e < nv ? u[e] : 0.0f;
                sq += double(u[e]) * double(u[e]);
                // NaN patterns lie above infinity's, so a maximum of patterns keeps them
                most = __uint_as_float(max(__float_as_uint(most), __float_as_uint(fabsf(m1[e]))));
            }
            store8f(d.u + e0 + o, nv, u);
            atomicMax(&top[b], __float_as_uint(most));
        }
        if (r == 0) {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                held[0][e] = m1[e];
        } else if (r == 1) {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                held[1][e] = m1[e];
        }
    }
    static_assert(kMomentumHeld == 2, "the passes keep two granules");
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1)
        sq += __shfl_xor(sq, o, 64);
    if (lane == 0)
        squares[wave] = sq;
    __syncthreads();
    if (t == 0)
        d.partial[in_matrix] = (squares[0] + squares[1]) + (squares[2] + squares[3]);

    // pass 2: requantize (the first two granules of a lane from registers)
#pragma unroll 1
    for (int gi = t, r = 0; gi < n_gran; gi += kThreads, ++r) {
        const int o = kGranule * gi;
        const int nv = min(kGranule, len - o), b = o / B;
        const float amax = __uint_as_float(top[b]);
        const float inv = (MAP == kMapLinear ? 127.0f : 1.0f) / amax;
        const bool ok = isfinite(amax) && isfinite(inv);
        float m1[8], cg[8];
        if (r < kMomentumHeld) {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                m1[e] = r == 0 ? held[0][e] : held[1][e];
        } else {
            const float a = gp(d.ma)[blk0 + b];
            MomentumIn in;
            momentum_load<GT>(d, e0 + o, nv, in);
            momentum_new<MAP>(in, MAP == kMapLinear ? a / 127.0f : a, coef, s, tab, m1, cg);
        }
        momentum_store<MAP>(d.mq, e0 + o, nv, m1, inv, ok, tab);
    }
    __syncthreads();  // every old scale has been read
    const int blocks = (len + B - 1) / B;
    for (int b = t; b < blocks; b += kThreads) {
        const float amax = __uint_as_float(top[b]);
        const float inv = (MAP == kMapLinear ? 127.0f : 1.0f) / amax;
        gp(d.ma)[blk0 + b] = isfinite(amax) && isfinite(inv) ? amax : 0.0f;
    }
}

}  // namespace

namespace host {

int64_t momentum_unit(int block)
{
    return block >= kMomentumSpan ? block : int64_t(kMomentumSpan / block) * block;
}

lt_err launch_momentum(const Guard& guard, const int64_t* prefix, const MomentumTensor* desc,
                       int first, int n, int64_t first_unit, int64_t units, int grad_dtype,
                       int block, int code_map, const MomentumScalars& s, const float* coef,
                       const int32_t* status, const void* step_state, hipStream_t st)
{
    if (units == 0)
        return LT_OK;
    const WsGuard g{guard.at, guard.tag};
    const bool dynamic = code_map == LT_MAP_DYNAMIC;
    auto* kernel = grad_dtype == LT_DTYPE_BF16
                       ? (dynamic ? k_muon_momentum<uint16_t, kMapDynamic>
                                  : k_muon_momentum<uint16_t, kMapLinear>)
                       : (dynamic ? k_muon_momentum<float, kMapDynamic>
                                  : k_muon_momentum<float, kMapLinear>);
    kernel<<<dim3(uint32_t(units)), kThreads, 0, st>>>(
        g, prefix, desc, first, n, first_unit, block, momentum_unit(block), s, coef, status,
        static_cast<const uint8_t*>(step_state));
    LT_HIP(hipGetLastError());
    return LT_OK;
}

}  // namespace host
