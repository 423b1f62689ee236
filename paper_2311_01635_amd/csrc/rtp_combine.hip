// Weighted combination of what a token's k experts give, and its gradients (rtp_combine_fwd, rtp_combine_bwd).
#include "rtp_block_kernels.h"
#include "rtp_elem.h"
#include <algorithm>

namespace rtp {

constexpr int CT = 256;

template <rtp_dtype DT>
__global__ __launch_bounds__(CT) void combine_fwd_row_kernel(CombineArgs p)
{
    using E = typename Elem<DT>::t;
    for (int64_t t = blockIdx.x; t < p.T; t += gridDim.x) {
        const E *yk = (const E *)p.Yk + t * p.k * p.ld_yk;
        E *y = (E *)p.Y + t * p.ld_y;
        for (int64_t i = threadIdx.x; i < p.D; i += CT) {
            float v = 0.0f;
            for (int j = 0; j < p.k; ++j) {
                const float w = p.weights ? p.weights[t * p.k + j] : 1.0f;
                if (w != 0.0f) v = fmaf(w, (float)yk[j * p.ld_yk + i], v);
            }
            y[i] = (E)v;
        }
    }
}

template <rtp_dtype DT>
__global__ __launch_bounds__(CT) void combine_bwd_row_kernel(CombineArgs p)
{
    using E = typename Elem<DT>::t;
    __shared__ float part[CT / 64];
    for (int64_t t = blockIdx.x; t < p.T; t += gridDim.x) {
        const E *dy = (const E *)p.dY + t * p.ld_y;
        for (int j = 0; j < p.k; ++j) {
            const float w = p.weights ? p.weights[t * p.k + j] : 1.0f;
            const E *yk = (const E *)p.Yk + (t * p.k + j) * p.ld_yk;
            E *dyk = (E *)p.dYk + (t * p.k + j) * p.ld_dyk;
            float dot = 0.0f;
            for (int64_t i = threadIdx.x; i < p.D; i += CT) {
                const float g = (float)dy[i];
                if (p.dweights) dot = fmaf(g, (float)yk[i], dot);
                if (p.dYk) dyk[i] = w == 0.0f ? (E)0.0f : (E)(w * g);
            }
            if (!p.dweights) continue;
            dot = wave_sum(dot);
            if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = dot;
            __syncthreads();
            if (threadIdx.x == 0) {
                float v = part[0];
                for (int i = 1; i < CT / 64; ++i) v += part[i];
                p.dweights[t * p.k + j] = v;
            }
            __syncthreads();
        }
    }
}

hipError_t launch_combine_fwd(const CombineArgs &a, hipStream_t s)
{
    const unsigned grid = (unsigned)std::min<int64_t>(a.T, 1 << 20);
    if (a.dtype == RTP_F32) combine_fwd_row_kernel<RTP_F32><<<grid, CT, 0, s>>>(a);
    else if (a.dtype == RTP_BF16) combine_fwd_row_kernel<RTP_BF16><<<grid, CT, 0, s>>>(a);
    else combine_fwd_row_kernel<RTP_F16><<<grid, CT, 0, s>>>(a);
    return hipGetLastError();
}

hipError_t launch_combine_bwd(const CombineArgs &a, hipStream_t s)
{
    const unsigned grid = (unsigned)std::min<int64_t>(a.T, 1 << 20);
    if (a.dtype == RTP_F32) combine_bwd_row_kernel<RTP_F32><<<grid, CT, 0, s>>>(a);
    else if (a.dtype == RTP_BF16) combine_bwd_row_kernel<RTP_BF16><<<grid, CT, 0, s>>>(a);
    else combine_bwd_row_kernel<RTP_F16><<<grid, CT, 0, s>>>(a);
    return hipGetLastError();
}

} // namespace rtp
