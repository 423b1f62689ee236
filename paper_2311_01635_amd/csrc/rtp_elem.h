// Element types of the kernels around a unit, and how their rows are read and written.
#pragma once
#include "../../include/rtp.h"
#include <hip/hip_runtime.h>

namespace rtp {

template <rtp_dtype D> struct Elem;
template <> struct Elem<RTP_F32> { using t = float; };
template <> struct Elem<RTP_BF16> { using t = __bf16; };
template <> struct Elem<RTP_F16> { using t = _Float16; };

// N neighbouring elements (8 or 4) as they are in memory.  Rows may begin anywhere (an odd length, a column of a wider matrix): the
// hardware reads and writes 16 bytes at any address of an element, and a row that begins off 16 bytes costs the lines it
// touches, no path of its own.  What is left of a row behind its last whole N goes element by element (`n` of them).
template <rtp_dtype D, int N> struct Some {
    using t = typename Elem<D>::t;
    static constexpr int WORDS = sizeof(t) * N / 4;
    typedef uint32_t Raw __attribute__((ext_vector_type(WORDS), aligned(sizeof(t))));
    struct { uint32_t w[WORDS]; } raw;

    // ONCE: past the caches, for what nobody reads again soon.  (Stores always are: rows that a launch writes are longer than
    // the caches before their reader comes, and it is gentler on what the launch reads: norm of 4096 x 4096 43 -> 41 us.)
    template <bool ONCE = false> __device__ __forceinline__ void load(const t *p, int64_t n)
    {
        if (n >= N) {
            const Raw v = ONCE ? __builtin_nontemporal_load((const Raw *)p) : *(const Raw *)p;
#pragma unroll
            for (int i = 0; i < WORDS; ++i) raw.w[i] = v[i];
        } else {
#pragma unroll
            for (int i = 0; i < WORDS; ++i) raw.w[i] = 0;
#pragma unroll
            for (int i = 0; i < N - 1; ++i)
                if (i < n) {
                    if (sizeof(t) == 4) raw.w[i % WORDS] = ((const uint32_t *)p)[i];
                    else raw.w[i / 2] |= (uint32_t)((const uint16_t *)p)[i] << (i & 1) * 16;
                }
        }
    }
    __device__ __forceinline__ void store(t *p, int64_t n) const
    {
        if (n >= N) {
            Raw v;
#pragma unroll
            for (int i = 0; i < WORDS; ++i) v[i] = raw.w[i];
            __builtin_nontemporal_store(v, (Raw *)p);
        } else {
#pragma unroll
            for (int i = 0; i < N - 1; ++i)
                if (i < n) {
                    if (sizeof(t) == 4) ((uint32_t *)p)[i] = raw.w[i % WORDS];
                    else ((uint16_t *)p)[i] = (uint16_t)(raw.w[i / 2] >> (i & 1) * 16);
                }
        }
    }
    __device__ __forceinline__ float get(int i) const
    {
        if constexpr (D == RTP_F32) return __uint_as_float(raw.w[i % WORDS]);
        const uint32_t h = raw.w[i / 2];
        if (D == RTP_BF16) return __uint_as_float(i & 1 ? h & 0xFFFF0000u : h << 16);
        return (float)__builtin_bit_cast(_Float16, (uint16_t)(i & 1 ? h >> 16 : h));
    }
    // (rounded to nearest, once)
    __device__ __forceinline__ void set(const float (&v)[N])
    {
#pragma unroll
        for (int i = 0; i < WORDS; ++i) {
            if constexpr (D == RTP_F32) {
                raw.w[i] = __float_as_uint(v[i % N]);
            } else {
                const uint32_t lo = __builtin_bit_cast(uint16_t, (t)v[2 * i % N]), hi = __builtin_bit_cast(uint16_t, (t)v[(2 * i + 1) % N]);
                raw.w[i] = lo | hi << 16;
            }
        }
    }
};

template <rtp_dtype D> using Eight = Some<D, 8>;
template <rtp_dtype D> using Four = Some<D, 4>;

// v of the lane that a data-parallel-primitive control names; every lane has one
template <int CTRL> __device__ __forceinline__ float dpp(float v)
{
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xF, 0xF, true));
}
constexpr int DPP_XOR1 = 0xB1, DPP_XOR2 = 0x4E, DPP_HALF_MIRROR = 0x141, DPP_MIRROR = 0x140; // within 2, 4, 8 and 16 lanes

// sum over the wave, in every lane: within rows of 16 lanes by operand modifiers of the additions, then the four rows
__device__ __forceinline__ float wave_sum(float v)
{
    v += dpp<DPP_XOR1>(v);
    v += dpp<DPP_XOR2>(v);
    v += dpp<DPP_HALF_MIRROR>(v);
    v += dpp<DPP_MIRROR>(v);
    const int i = __float_as_int(v);
    const float a = __int_as_float(__builtin_amdgcn_readlane(i, 0)), b = __int_as_float(__builtin_amdgcn_readlane(i, 16));
    const float c = __int_as_float(__builtin_amdgcn_readlane(i, 32)), d = __int_as_float(__builtin_amdgcn_readlane(i, 48));
    return (a + b) + (c + d);
}
// the largest over the wave, in every lane (a scalar)
__device__ __forceinline__ uint32_t wave_umax(uint32_t v)
{
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, DPP_XOR1, 0xF, 0xF, true));
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, DPP_XOR2, 0xF, 0xF, true));
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, DPP_HALF_MIRROR, 0xF, 0xF, true));
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, DPP_MIRROR, 0xF, 0xF, true));
    const uint32_t a = __builtin_amdgcn_readlane(v, 0), b = __builtin_amdgcn_readlane(v, 16);
    const uint32_t c = __builtin_amdgcn_readlane(v, 32), d = __builtin_amdgcn_readlane(v, 48);
    return max(max(a, b), max(c, d));
}

} // namespace rtp
