// Element types of the kernels around a unit, and what their rows are read and written with.
#pragma once
#include "../../include/rtp.h"
#include <hip/hip_runtime.h>

namespace rtp {

template <rtp_dtype D> struct Elem;
template <> struct Elem<RTP_F32> { using t = float; };
template <> struct Elem<RTP_BF16> { using t = __bf16; };
template <> struct Elem<RTP_F16> { using t = _Float16; };

// sum over the wave, in every lane
__device__ __forceinline__ float wave_sum(float v)
{
#pragma unroll
    for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o);
    return v;
}

} // namespace rtp
