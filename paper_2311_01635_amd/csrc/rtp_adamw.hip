// One AdamW step over many tensors (rtp_adamw_step), and the moments as numbers (rtp_adamw_moments).
#include "rtp_block_kernels.h"
#include "rtp_elem.h"
#include <algorithm>

namespace rtp {

constexpr int AT = RTP_ADAMW_BLOCK; // a thread an element of a block

// ---- moments in 8 bits -----------------------------------------------------------------------
// A code, shifted to where an fp32 has exponent and mantissa, is that number times a power of two, denormal ones included: reading
// is a shift and a scaling, writing a scaling, an addition of random bits below the last kept one, and a shift.
constexpr int TOP_M = 14, TOP_V = 30; // exponent code of the binade of a block's largest element (one above is for a carry)

__device__ __forceinline__ float unpack(unsigned mag, int E, int top)
{
    return E == 255 ? __builtin_nanf("") : ldexpf(__uint_as_float(mag << 20), E - top);
}
__device__ __forceinline__ unsigned pack(float a, int E, int top, unsigned rnd16)
{
    return (__float_as_uint(ldexpf(a, top - E)) + (rnd16 << 4)) >> 20;
}

// 32 random bits of the seed and an element's place, and 16 more
__device__ __forceinline__ unsigned hash(unsigned place, unsigned seed)
{
    unsigned x = place * 0x9E3779B1u + seed;
    x = (x ^ x >> 15) * 0xB504F333u;
    x = (x ^ x >> 16) * 0x243F6A89u;
    return x ^ x >> 15;
}
__device__ __forceinline__ unsigned hash_more(unsigned x) { return x * 0x9E3779B1u >> 16; }

// a float between two neighbours of a 16-bit type goes to the upper with the probability of its place between them
__device__ __forceinline__ float round_random(float v, rtp_dtype t, unsigned rnd16)
{
    const unsigned u = __float_as_uint(v);
    if ((u & 0x7F800000u) == 0x7F800000u) return v;
    if (t == RTP_BF16) return __uint_as_float((u + rnd16) & 0xFFFF0000u);
    if (fabsf(v) >= 6.103515625e-05f) return __uint_as_float((u + (rnd16 >> 3)) & 0xFFFFE000u);
    // below 2^-14 fp16's spacing is 2^-24
    const float n = floorf(ldexpf(fabsf(v), 24) + ldexpf((float)rnd16, -16));
    return copysignf(ldexpf(n, -24), v);
}

template <rtp_moments MO>
__global__ __launch_bounds__(AT) void adamw_block_kernel(AdamwArgs p)
{
    __shared__ float high[2][AT / 64];
    const rtp_adamw_scalars h = p.sc_dev ? *p.sc_dev : p.sc;
    const float scale = p.scale ? *p.scale : 1.0f;
    if (!(fabsf(scale) < INFINITY)) return;
    for (int64_t chunk = blockIdx.x; chunk < p.chunks; chunk += gridDim.x) {
        const AdamwEntry &e = p.entries[p.owner[chunk]];
        const int64_t first = (chunk - e.chunk) * ADAMW_CHUNK;
        for (int b = 0; b < ADAMW_CHUNK_BLOCKS && first + b * RTP_ADAMW_BLOCK < e.numel; ++b) {
            const int64_t i = first + b * RTP_ADAMW_BLOCK + threadIdx.x, block = e.block + i / RTP_ADAMW_BLOCK;
            const int64_t place = e.block * RTP_ADAMW_BLOCK + i;
            const bool on = i < e.numel;
            const float g = on ? e.grad[i] * scale : 0.0f;
            float m, v;
            if (MO == RTP_MOMENTS_F32) {
                m = on ? ((const float *)p.m)[place] : 0.0f;
                v = on ? ((const float *)p.v)[place] : 0.0f;
            } else {
                const unsigned mc = ((const uint8_t *)p.m)[place], vc = ((const uint8_t *)p.v)[place];
                m = unpack(mc & 127, max((int)p.exps[block * 2], 1), TOP_M);
                m = mc & 128 ? -m : m;
                v = unpack(vc, max((int)p.exps[block * 2 + 1], 1), TOP_V);
                if (!on) m = v = 0.0f;
            }
            m = h.beta1 * m + h.one_minus_beta1 * g;
            v = h.beta2 * v + h.one_minus_beta2 * (g * g);
            const unsigned rnd = hash((unsigned)place, h.seed);
            if (on) {
                float w = e.master ? e.master[i] : e.dtype == RTP_F32 ? ((const float *)e.param)[i] :
                          e.dtype == RTP_BF16 ? (float)((const __bf16 *)e.param)[i] : (float)((const _Float16 *)e.param)[i];
                w = w * (1.0f - h.lr * e.weight_decay) - h.step_size * (m / (sqrtf(v) * h.root_scale + h.eps));
                if (e.master) e.master[i] = w;
                else if (e.dtype != RTP_F32) w = round_random(w, (rtp_dtype)e.dtype, hash_more(rnd));
                if (e.dtype == RTP_F32) ((float *)e.param)[i] = w;
                else if (e.dtype == RTP_BF16) ((__bf16 *)e.param)[i] = (__bf16)w;
                else ((_Float16 *)e.param)[i] = (_Float16)w;
            }
            if (MO == RTP_MOMENTS_F32) {
                if (on) { ((float *)p.m)[place] = m; ((float *)p.v)[place] = v; }
            } else {
                // (magnitudes as integers are in the order of their values, NaN above all)
                unsigned a = __float_as_uint(m) & 0x7FFFFFFFu, c = __float_as_uint(v) & 0x7FFFFFFFu;
#pragma unroll
                for (int o = 32; o; o >>= 1) { a = max(a, (unsigned)__shfl_xor((int)a, o)); c = max(c, (unsigned)__shfl_xor((int)c, o)); }
                __syncthreads();
                if ((threadIdx.x & 63) == 0) { high[0][threadIdx.x >> 6] = __uint_as_float(a); high[1][threadIdx.x >> 6] = __uint_as_float(c); }
                __syncthreads();
                for (int k = 0; k < AT / 64; ++k) { a = max(a, __float_as_uint(high[0][k])); c = max(c, __float_as_uint(high[1][k])); }
                const int Em = max((int)(a >> 23), 1), Ev = max((int)(c >> 23), 1);
                ((uint8_t *)p.m)[place] = (uint8_t)(pack(fabsf(m), Em, TOP_M, rnd & 0xFFFF) | (__float_as_uint(m) >> 31 << 7));
                ((uint8_t *)p.v)[place] = (uint8_t)max(pack(v, Ev, TOP_V, rnd >> 16), v > 0.0f ? 1u : 0u);
                if (threadIdx.x == 0) { p.exps[block * 2] = (uint8_t)Em; p.exps[block * 2 + 1] = (uint8_t)Ev; }
            }
        }
    }
}

template <rtp_moments MO, rtp_dtype DT>
__global__ __launch_bounds__(AT) void adamw_moments_kernel(const void *m, const void *v, const uint8_t *exps, int64_t blocks, void *m_out, void *v_out)
{
    using O = typename Elem<DT>::t;
    for (int64_t b = blockIdx.x; b < blocks; b += gridDim.x) {
        const int64_t i = b * RTP_ADAMW_BLOCK + threadIdx.x;
        float x, y;
        if (MO == RTP_MOMENTS_F32) {
            x = ((const float *)m)[i];
            y = ((const float *)v)[i];
        } else {
            const unsigned mc = ((const uint8_t *)m)[i];
            x = unpack(mc & 127, max((int)exps[b * 2], 1), TOP_M);
            x = mc & 128 ? -x : x;
            y = unpack(((const uint8_t *)v)[i], max((int)exps[b * 2 + 1], 1), TOP_V);
        }
        ((O *)m_out)[i] = (O)x;
        ((O *)v_out)[i] = (O)y;
    }
}

hipError_t launch_adamw(rtp_moments moments, const AdamwArgs &a, hipStream_t s)
{
    const unsigned grid = (unsigned)std::min<int64_t>(a.chunks, 1 << 20);
    if (moments == RTP_MOMENTS_F32) adamw_block_kernel<RTP_MOMENTS_F32><<<grid, AT, 0, s>>>(a);
    else adamw_block_kernel<RTP_MOMENTS_8BIT><<<grid, AT, 0, s>>>(a);
    return hipGetLastError();
}

hipError_t launch_adamw_moments(rtp_moments moments, rtp_dtype out, const void *m, const void *v, const uint8_t *exps, int64_t blocks,
                                void *m_out, void *v_out, hipStream_t s)
{
    const unsigned grid = (unsigned)std::min<int64_t>(blocks, 1 << 20);
    const bool f = out == RTP_F32;
    if (moments == RTP_MOMENTS_F32) {
        if (f) adamw_moments_kernel<RTP_MOMENTS_F32, RTP_F32><<<grid, AT, 0, s>>>(m, v, exps, blocks, m_out, v_out);
        else adamw_moments_kernel<RTP_MOMENTS_F32, RTP_BF16><<<grid, AT, 0, s>>>(m, v, exps, blocks, m_out, v_out);
    } else {
        if (f) adamw_moments_kernel<RTP_MOMENTS_8BIT, RTP_F32><<<grid, AT, 0, s>>>(m, v, exps, blocks, m_out, v_out);
        else adamw_moments_kernel<RTP_MOMENTS_8BIT, RTP_BF16><<<grid, AT, 0, s>>>(m, v, exps, blocks, m_out, v_out);
    }
    return hipGetLastError();
}

} // namespace rtp
