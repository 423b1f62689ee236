// One AdamW step over many tensors (rtp_adamw_step), and the moments as numbers (rtp_adamw_moments).
#include "rtp_block_kernels.h"
#include "rtp_elem.h"
#include <algorithm>
#include <type_traits>

namespace rtp {

// Bound: HBM, 12 to 30 bytes a parameter that are read and written once.  With 8-bit moments the arithmetic is as long: at 6 TB/s a
// parameter's 12 bytes leave a compute unit time for 79 instructions a wave, and the hash, the update and two
// conversions are about 70 of them.  A wave takes four blocks of 256, a lane four neighbours of each: their 16 loads are sent
// before the first is waited for (past the caches: 752 -> 706 us for 135M with fp32 moments and masters, 5.7 TB/s), a block's largest
// element is a reduction within the wave, and nothing needs a barrier.  135M with 8-bit moments: 295 us, 5.5 TB/s; a thread an
// element, blocks of 256 threads: 1400.
constexpr int AT = 256, AB = 4; // threads, blocks of a wave
static_assert(AT / 64 * AB == ADAMW_CHUNK_BLOCKS, "a workgroup is a chunk");

// ---- moments in 8 bits -----------------------------------------------------------------------
// A code, shifted to where an fp32 has exponent and mantissa, is that number times a power of two, denormal ones included: reading
// is a shift and a scaling, writing a scaling, an addition of random bits below the last kept one, and a shift.
constexpr int TOP_M = 14, TOP_V = 30; // exponent code of the binade of a block's largest element (one above is for a carry)

// byte k of a word of codes; `scale` = E - TOP
__device__ __forceinline__ float unpack_m(uint32_t word, int k, int scale)
{
    return ldexpf(__uint_as_float((uint32_t)((int32_t)(word << (24 - 8 * k)) >> 4) & 0x87F00000u), scale);
}
__device__ __forceinline__ float unpack_v(uint32_t word, int k, int scale)
{
    return ldexpf(__uint_as_float((word >> 8 * k & 255u) << 20), scale);
}
__device__ __forceinline__ uint32_t pack(float a, int scale, uint32_t rnd16)
{
    return (__float_as_uint(ldexpf(a, scale)) + (rnd16 << 4)) >> 20;
}

// 32 random bits of the seed and an element's place (x = place * PLACE + seed), and 16 more
constexpr uint32_t PLACE = 0x9E3779B1u;
__device__ __forceinline__ uint32_t hash(uint32_t x)
{
    x = (x ^ x >> 15) * 0xB504F333u;
    x = (x ^ x >> 16) * 0x243F6A89u;
    return x ^ x >> 15;
}
__device__ __forceinline__ uint32_t hash_more(uint32_t x) { return x * 0x9E3779B1u >> 16; }

// A float between two neighbours of a 16-bit type goes to the upper with the probability of its place between them.  (Infinities have no
// bits below to carry; NaN, which may, are let through.)
template <rtp_dtype D> __device__ __forceinline__ float round_random(float v, uint32_t rnd16)
{
    const uint32_t u = __float_as_uint(v);
    if (D == RTP_BF16) return __uint_as_float((u + (v != v ? 0u : rnd16)) & 0xFFFF0000u);
    if (!(fabsf(v) < INFINITY)) return v;
    if (fabsf(v) >= 6.103515625e-05f) return __uint_as_float((u + (rnd16 >> 3)) & 0xFFFFE000u);
    // below 2^-14 fp16's spacing is 2^-24
    const float n = floorf(ldexpf(fabsf(v), 24) + ldexpf((float)rnd16, -16));
    return copysignf(ldexpf(n, -24), v);
}

// beta x + (1 - beta) y with each product and the sum rounded by itself, as a step written out in fp32 operations does.  A fused
// multiply-add is as near to 64 bits, but its half a unit decides a code's random rounding now and then, and the next steps go on from
// the code: two programs that step the same state have to round alike.  (Two instructions an element: 295 us instead of 294.)
__device__ __forceinline__ float decayed(float beta, float x, float one_minus_beta, float y)
{
#pragma clang fp contract(off)
    return beta * x + one_minus_beta * y;
}

// (a pointer out of the table is one into device memory: without the word for it the accesses are the flat ones, which wait for LDS too)
template <class T> __device__ __forceinline__ T *global(T *p)
{
    return (T *)(__attribute__((address_space(1))) T *)(uintptr_t)p;
}

// Blocks [first, first + AB) of a tensor's, as many as it has.  FULL: all of them, whole.
template <rtp_moments MO, rtp_dtype D, bool MASTER, bool FULL>
__device__ __forceinline__ void adamw_blocks(const AdamwArgs &p, const AdamwEntry &e, const int64_t first, const rtp_adamw_scalars &h, const float scale)
{
    using P = typename Elem<D>::t;
    constexpr bool BYTE = MO == RTP_MOMENTS_8BIT, RANDOM = D != RTP_F32 && !MASTER;
    const int i = (threadIdx.x & 63) * 4; // this lane's place in a block
    const int64_t from = first * RTP_ADAMW_BLOCK, place = e.block * RTP_ADAMW_BLOCK + from;
    const int total = FULL ? AB * RTP_ADAMW_BLOCK : (int)min(e.numel - from, (int64_t)AB * RTP_ADAMW_BLOCK);
    P *const param = global((P *)e.param) + from;
    const float *const grad = global(e.grad) + from;
    float *const copy = global(e.master) + from, *const pm = (float *)p.m + place, *const pv = (float *)p.v + place;
    uint8_t *const qm = (uint8_t *)p.m + place, *const qv = (uint8_t *)p.v + place;
    uint16_t *const exps = (uint16_t *)p.exps + e.block + first;
    const float keep = 1.0f - h.lr * e.weight_decay;
    Four<RTP_F32> g[AB], master[AB], fm[AB], fv[AB];
    Four<D> w[AB];
    uint32_t bm[AB], bv[AB], ex[AB];
#pragma unroll
    for (int b = 0; b < AB; ++b) {
        const int at = b * RTP_ADAMW_BLOCK;
        if (!FULL && at >= total) break;
        const int n = FULL ? 4 : total - at - i;
        g[b].template load<true>(grad + at + i, n);
        if (MASTER) master[b].template load<true>(copy + at + i, n);
        else w[b].template load<true>(param + at + i, n);
        if (BYTE) {
            bm[b] = *(const uint32_t *)(qm + at + i);
            bv[b] = *(const uint32_t *)(qv + at + i);
            ex[b] = exps[b];
        } else {
            fm[b].template load<true>(pm + at + i, 4);
            fv[b].template load<true>(pv + at + i, 4);
        }
    }
#pragma unroll
    for (int b = 0; b < AB; ++b) {
        const int at = b * RTP_ADAMW_BLOCK;
        if (!FULL && at >= total) break;
        const int n = FULL ? 4 : total - at - i;
        float m[4], v[4], o[4];
        if (BYTE) {
            const int x = __builtin_amdgcn_readfirstlane(ex[b]), em = max(x & 255, 1), ev = max(x >> 8, 1);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                m[k] = unpack_m(bm[b], k, em - TOP_M);
                v[k] = unpack_v(bv[b], k, ev - TOP_V);
                if (!FULL && k >= n) m[k] = v[k] = 0.0f; // behind the tensor
            }
            if (em == 255 || ev == 255) {
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    if (em == 255) m[k] = __builtin_nanf("");
                    if (ev == 255) v[k] = __builtin_nanf("");
                }
            }
        } else {
#pragma unroll
            for (int k = 0; k < 4; ++k) { m[k] = fm[b].get(k); v[k] = fv[b].get(k); }
        }
        uint32_t rnd[4], top_m = 0, top_v = 0;
        const uint32_t x = (uint32_t)(place + at + i) * PLACE + h.seed;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const float gr = g[b].get(k) * scale;
            m[k] = decayed(h.beta1, m[k], h.one_minus_beta1, gr);
            v[k] = decayed(h.beta2, v[k], h.one_minus_beta2, gr * gr);
            if (BYTE || RANDOM) rnd[k] = hash(x + k * PLACE);
            // the hardware's root and reciprocal, 1 ulp each (a second moment below 2^-126 counts as zero here)
            const float d = m[k] * __builtin_amdgcn_rcpf(fmaf(__builtin_amdgcn_sqrtf(v[k]), h.root_scale, h.eps));
            o[k] = fmaf(-h.step_size, d, keep * (MASTER ? master[b].get(k) : w[b].get(k)));
            if (BYTE) {
                // (magnitudes as integers are in the order of their values, NaN above all)
                top_m = max(top_m, __float_as_uint(m[k]) & 0x7FFFFFFFu);
                top_v = max(top_v, __float_as_uint(v[k]) & 0x7FFFFFFFu);
            }
        }
        if (MASTER) {
            // (fp16: the compiler would round the update to it by itself, and not what the master holds)
#pragma unroll
            for (int k = 0; k < 4; ++k) asm("" : "+v"(o[k]));
            master[b].set(o);
            master[b].store(copy + at + i, n);
        }
        if (RANDOM) {
#pragma unroll
            for (int k = 0; k < 4; ++k) o[k] = round_random<D>(o[k], hash_more(rnd[k]));
        }
        w[b].set(o);
        w[b].store(param + at + i, n);
        if (BYTE) {
            const int Em = max((int)(wave_umax(top_m) >> 23), 1), Ev = max((int)(wave_umax(top_v) >> 23), 1);
            uint32_t cm = 0, cv = 0;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const uint32_t sign = __float_as_uint(m[k]) >> 31 << 7;
                cm |= (pack(fabsf(m[k]), TOP_M - Em, rnd[k] & 0xFFFF) & 127u | sign) << 8 * k;
                // (a second moment that is there does not vanish)
                cv |= (max(pack(v[k], TOP_V - Ev, rnd[k] >> 16), min(__float_as_uint(v[k]), 1u)) & 255u) << 8 * k;
            }
            *(uint32_t *)(qm + at + i) = cm;
            *(uint32_t *)(qv + at + i) = cv;
            if (i == 0) exps[b] = (uint16_t)(Em | Ev << 8);
        } else {
            fm[b].set(m);
            fv[b].set(v);
            fm[b].store(pm + at + i, n);
            fv[b].store(pv + at + i, n);
        }
    }
}

template <rtp_moments MO>
__global__ __launch_bounds__(AT) void adamw_kernel(AdamwArgs p)
{
    const rtp_adamw_scalars h = p.sc_dev ? *p.sc_dev : p.sc;
    const float scale = p.scale ? *p.scale : 1.0f;
    if (!(fabsf(scale) < INFINITY)) return;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    for (int64_t chunk = blockIdx.x; chunk < p.chunks; chunk += gridDim.x) {
        const AdamwEntry &e = p.entries[p.owner[chunk]];
        const int64_t first = (chunk - e.chunk) * ADAMW_CHUNK_BLOCKS + wave * AB;
        const bool full = (first + AB) * RTP_ADAMW_BLOCK <= e.numel;
        if (first * RTP_ADAMW_BLOCK >= e.numel) continue;
        auto blocks = [&](auto dtype, auto master) {
            if (full) adamw_blocks<MO, decltype(dtype)::value, decltype(master)::value, true>(p, e, first, h, scale);
            else adamw_blocks<MO, decltype(dtype)::value, decltype(master)::value, false>(p, e, first, h, scale);
        };
        using std::false_type;
        using std::true_type;
        if (e.dtype == RTP_F32) blocks(std::integral_constant<rtp_dtype, RTP_F32>{}, false_type{});
        else if (e.dtype == RTP_BF16 && e.master) blocks(std::integral_constant<rtp_dtype, RTP_BF16>{}, true_type{});
        else if (e.dtype == RTP_BF16) blocks(std::integral_constant<rtp_dtype, RTP_BF16>{}, false_type{});
        else if (e.master) blocks(std::integral_constant<rtp_dtype, RTP_F16>{}, true_type{});
        else blocks(std::integral_constant<rtp_dtype, RTP_F16>{}, false_type{});
    }
}

// Moments as numbers.  Bound: HBM.  A thread takes eight neighbours, a block 32 threads (16 to a thread left holes of 16 bytes in what a
// store instruction writes: 278 us instead of 129 for 135M of 8 bits).
template <rtp_moments MO, rtp_dtype DT>
__global__ __launch_bounds__(AT) void adamw_moments_kernel(const void *m, const void *v, const uint8_t *exps, int64_t blocks, void *m_out, void *v_out)
{
    using O = typename Elem<DT>::t;
    const int64_t b = (int64_t)blockIdx.x * (AT / 32) + threadIdx.x / 32, i = b * RTP_ADAMW_BLOCK + threadIdx.x % 32 * 8;
    if (b >= blocks) return;
    float x[8], y[8];
    if (MO == RTP_MOMENTS_F32) {
        Eight<RTP_F32> em, ev;
        em.load<true>((const float *)m + i, 8);
        ev.load<true>((const float *)v + i, 8);
#pragma unroll
        for (int k = 0; k < 8; ++k) { x[k] = em.get(k); y[k] = ev.get(k); }
    } else {
        const uint2 cm = *(const uint2 *)((const uint8_t *)m + i), cv = *(const uint2 *)((const uint8_t *)v + i);
        const uint32_t ex = ((const uint16_t *)exps)[b];
        const int em = max((int)(ex & 255), 1), ev = max((int)(ex >> 8), 1);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            x[k] = em == 255 ? __builtin_nanf("") : unpack_m(k < 4 ? cm.x : cm.y, k % 4, em - TOP_M);
            y[k] = ev == 255 ? __builtin_nanf("") : unpack_v(k < 4 ? cv.x : cv.y, k % 4, ev - TOP_V);
        }
    }
    Eight<DT> e;
    e.set(x);
    e.store((O *)m_out + i, 8);
    e.set(y);
    e.store((O *)v_out + i, 8);
}

hipError_t launch_adamw(rtp_moments moments, const AdamwArgs &a, hipStream_t s)
{
    const unsigned grid = (unsigned)std::min<int64_t>(a.chunks, 1 << 20);
    if (moments == RTP_MOMENTS_F32) adamw_kernel<RTP_MOMENTS_F32><<<grid, AT, 0, s>>>(a);
    else adamw_kernel<RTP_MOMENTS_8BIT><<<grid, AT, 0, s>>>(a);
    return hipGetLastError();
}

hipError_t launch_adamw_moments(rtp_moments moments, rtp_dtype out, const void *m, const void *v, const uint8_t *exps, int64_t blocks,
                                void *m_out, void *v_out, hipStream_t s)
{
    const unsigned grid = (unsigned)((blocks + AT / 32 - 1) / (AT / 32));
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
