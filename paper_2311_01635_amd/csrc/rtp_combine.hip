// Weighted combination of what a token's k experts give, and its gradients (rtp_combine_fwd, rtp_combine_bwd).
//
// Bound: HBM, a fused multiply-add or two an element.  THREADS threads share a token (a wave where that is enough: no barrier) and go
// along its row eight elements at a time, with the loads of K slots in flight together, past the caches (8192 tokens of 2 x 4096 33 us,
// 6.1 TB/s; through them 35.5), and those of the weights beside them.  K is the number of slots, rounded up to a
// power of two, or chunks of 8.
#include "rtp_block_kernels.h"
#include "rtp_elem.h"
#include <algorithm>

namespace rtp {

constexpr int CT = 256;

template <rtp_dtype DT, int K, int THREADS>
__global__ __launch_bounds__(CT) void combine_fwd_kernel(CombineArgs p)
{
    using E = typename Elem<DT>::t;
    constexpr int ROWS = CT / THREADS;
    for (int64_t t = (int64_t)blockIdx.x * ROWS + threadIdx.x / THREADS; t < p.T; t += (int64_t)gridDim.x * ROWS) {
        const E *yk = (const E *)p.Yk + t * p.k * p.ld_yk;
        E *y = (E *)p.Y + t * p.ld_y;
        for (int64_t i = threadIdx.x % THREADS * 8; i < p.D; i += THREADS * 8) {
            float v[8] = {};
            for (int j0 = 0; j0 < p.k; j0 += K) {
                float w[K];
                Eight<DT> x[K];
#pragma unroll
                for (int j = 0; j < K; ++j) { // (a slot without weight is fetched too: its weight is on its way as well)
                    if (j0 + j < p.k) x[j].template load<true>(yk + (j0 + j) * p.ld_yk + i, p.D - i);
                    w[j] = j0 + j >= p.k ? 0.0f : p.weights ? p.weights[t * p.k + j0 + j] : 1.0f;
                }
#pragma unroll
                for (int j = 0; j < K; ++j) {
                    if (w[j] == 0.0f) continue;
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] = fmaf(w[j], x[j].get(e), v[e]);
                }
            }
            Eight<DT> o;
            o.set(v);
            o.store(y + i, p.D - i);
        }
    }
}

// dY is read once for K slots; the K dot products stay in registers along the row.
template <rtp_dtype DT, int K, int THREADS>
__global__ __launch_bounds__(CT) void combine_bwd_kernel(CombineArgs p)
{
    using E = typename Elem<DT>::t;
    constexpr int ROWS = CT / THREADS, WAVES = THREADS / 64;
    __shared__ float part[WAVES][K];
    const int tid = threadIdx.x % THREADS;
    for (int64_t t = (int64_t)blockIdx.x * ROWS + threadIdx.x / THREADS; t < p.T; t += (int64_t)gridDim.x * ROWS) {
        const E *dy = (const E *)p.dY + t * p.ld_y;
        for (int j0 = 0; j0 < p.k; j0 += K) {
            float w[K], dot[K];
#pragma unroll
            for (int j = 0; j < K; ++j) {
                w[j] = j0 + j >= p.k ? 0.0f : p.weights ? p.weights[t * p.k + j0 + j] : 1.0f;
                dot[j] = 0.0f;
            }
            const E *yk = (const E *)p.Yk + (t * p.k + j0) * p.ld_yk;
            E *dyk = (E *)p.dYk + (t * p.k + j0) * p.ld_dyk;
            for (int64_t i = tid * 8; i < p.D; i += THREADS * 8) {
                Eight<DT> g, x[K];
                g.load(dy + i, p.D - i);
                if (p.dweights) {
#pragma unroll
                    for (int j = 0; j < K; ++j)
                        if (j0 + j < p.k) x[j].template load<true>(yk + j * p.ld_yk + i, p.D - i);
                }
#pragma unroll
                for (int j = 0; j < K; ++j) {
                    if (j0 + j >= p.k) continue;
                    if (p.dweights) {
#pragma unroll
                        for (int e = 0; e < 8; ++e) dot[j] = fmaf(g.get(e), x[j].get(e), dot[j]);
                    }
                    if (p.dYk) {
                        float o[8];
#pragma unroll
                        for (int e = 0; e < 8; ++e) o[e] = w[j] == 0.0f ? 0.0f : w[j] * g.get(e);
                        Eight<DT> d;
                        d.set(o);
                        d.store(dyk + j * p.ld_dyk + i, p.D - i);
                    }
                }
            }
            if (!p.dweights) continue;
#pragma unroll
            for (int j = 0; j < K; ++j) dot[j] = wave_sum(dot[j]);
            if (WAVES == 1) {
                if (tid == 0) {
#pragma unroll
                    for (int j = 0; j < K; ++j)
                        if (j0 + j < p.k) p.dweights[t * p.k + j0 + j] = dot[j];
                }
            } else {
                if ((tid & 63) == 0) {
#pragma unroll
                    for (int j = 0; j < K; ++j) part[tid / 64][j] = dot[j];
                }
                __syncthreads();
                if (tid < K && j0 + tid < p.k) {
                    float v = 0.0f;
#pragma unroll
                    for (int i = 0; i < WAVES; ++i) v += part[i][tid];
                    p.dweights[t * p.k + j0 + tid] = v;
                }
                __syncthreads();
            }
        }
    }
}

// A wave a token while a row is one eight a lane, else the workgroup: the shorter a thread's way along its row, the better the
// memory is kept busy.  (A wave: 8192 tokens of 2 x 4096 38.6 us instead of 35.5, gradients of 4099 of 8 x 2048 64.3 instead of 51.1.)
template <rtp_dtype DT, int K, bool BWD>
static hipError_t launch(const CombineArgs &a, hipStream_t s)
{
    const bool wide = a.D > 512;
    const unsigned grid = (unsigned)std::min<int64_t>(wide ? a.T : (a.T + CT / 64 - 1) / (CT / 64), 1 << 20);
    if (BWD) {
        if (wide) combine_bwd_kernel<DT, K, CT><<<grid, CT, 0, s>>>(a);
        else combine_bwd_kernel<DT, K, 64><<<grid, CT, 0, s>>>(a);
    } else {
        if (wide) combine_fwd_kernel<DT, K, CT><<<grid, CT, 0, s>>>(a);
        else combine_fwd_kernel<DT, K, 64><<<grid, CT, 0, s>>>(a);
    }
    return hipGetLastError();
}
template <rtp_dtype DT, bool BWD>
static hipError_t by_slots(const CombineArgs &a, hipStream_t s)
{
    if (a.k == 1) return launch<DT, 1, BWD>(a, s);
    if (a.k == 2) return launch<DT, 2, BWD>(a, s);
    if (a.k <= 4) return launch<DT, 4, BWD>(a, s);
    return launch<DT, 8, BWD>(a, s);
}
template <bool BWD>
static hipError_t by_type(const CombineArgs &a, hipStream_t s)
{
    if (a.dtype == RTP_F32) return by_slots<RTP_F32, BWD>(a, s);
    if (a.dtype == RTP_BF16) return by_slots<RTP_BF16, BWD>(a, s);
    return by_slots<RTP_F16, BWD>(a, s);
}
hipError_t launch_combine_fwd(const CombineArgs &a, hipStream_t s) { return by_type<false>(a, s); }
hipError_t launch_combine_bwd(const CombineArgs &a, hipStream_t s) { return by_type<true>(a, s); }

} // namespace rtp
