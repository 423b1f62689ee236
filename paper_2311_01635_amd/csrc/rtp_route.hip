// Routing to experts (rtp_route_fwd, rtp_route_bwd).
#include "rtp_block_kernels.h"
#include "rtp_elem.h"
#include <algorithm>
#include <cmath>

namespace rtp {

// Bound: the arithmetic of the choice (a row of 256 is 1 KB; its eight largest are eight rounds of comparisons).  LANES lanes share
// a row, eight or sixteen neighbouring experts each, 64 / LANES rows to a wave: a round is then a maximum over a lane's keys, one over
// LANES lanes, and the lowest lane that has it, with no barrier and little LDS.  Keys are 32-bit integers in the order of what they
// stand for.  Where the choice is of scores (a bias, groups), they are scores in 32 bits; a row in which two of them that
// matter are closer than 32 bits can tell apart is decided again in 64 bits by its whole wave.
constexpr int RW = 4; // waves of a workgroup

struct RouteArgs {
    rtp_route_desc d;
    const void *logits;
    const float *bias;
    int32_t *ids;
    float *weights;
    const int32_t *ids_in;
    const float *dweights;
    void *dlogits;
};

// log of a sigmoid, without the underflow of the sigmoid itself
__device__ __forceinline__ float log_sigmoid(float l) { return fminf(l, 0.0f) - log1pf(expf(-fabsf(l))); }

// LDS operations of a wave are in order; this keeps the compiler from moving them past one another
__device__ __forceinline__ void wave_fence() { __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront"); }

// ---- over LANES neighbouring lanes, in each of them ----------------------------------------------
template <int CTRL> __device__ __forceinline__ uint32_t dpp(uint32_t v)
{
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xF, 0xF, true);
}
// f(own, other half's) for halves of 16 and of 32 lanes: the two results of a swap of a value with itself are both halves
template <int HALF, class F> __device__ __forceinline__ uint32_t with_other_half(uint32_t v, F f)
{
    const auto r = HALF == 16 ? __builtin_amdgcn_permlane16_swap(v, v, false, false) : __builtin_amdgcn_permlane32_swap(v, v, false, false);
    return f((uint32_t)r[0], (uint32_t)r[1]);
}
template <int LANES, class F> __device__ __forceinline__ uint32_t over(uint32_t v, F f)
{
    if (LANES >= 2) v = f(v, dpp<DPP_XOR1>(v));
    if (LANES >= 4) v = f(v, dpp<DPP_XOR2>(v));
    if (LANES >= 8) v = f(v, dpp<DPP_HALF_MIRROR>(v));
    if (LANES >= 16) v = f(v, dpp<DPP_MIRROR>(v));
    if (LANES >= 32) v = with_other_half<16>(v, f);
    if (LANES >= 64) v = with_other_half<32>(v, f);
    return v;
}
template <int LANES> __device__ __forceinline__ uint32_t over_max(uint32_t v)
{
    return over<LANES>(v, [](uint32_t a, uint32_t b) { return max(a, b); });
}
template <int LANES> __device__ __forceinline__ float over_fmax(float v)
{
    return __uint_as_float(over<LANES>(__float_as_uint(v), [](uint32_t a, uint32_t b) { return __float_as_uint(fmaxf(__uint_as_float(a), __uint_as_float(b))); }));
}
template <int LANES> __device__ __forceinline__ float over_sum(float v)
{
    return __uint_as_float(over<LANES>(__float_as_uint(v), [](uint32_t a, uint32_t b) { return __float_as_uint(__uint_as_float(a) + __uint_as_float(b)); }));
}

// ---- keys: 0 is out of the choice (taken, of another group, not there), 1 closed, then numbers in their order, NaN last ------
constexpr uint32_t KEY_OUT = 0, KEY_CLOSED = 1, KEY_NAN = 0xFFFFFFFFu;
__device__ __forceinline__ uint32_t key_of(float v)
{
    if (v != v) return KEY_NAN;
    if (v == -INFINITY) return KEY_CLOSED;
    const uint32_t u = __float_as_uint(v == 0.0f ? 0.0f : v); // (-0 and 0 are equal)
    return u ^ ((int32_t)u < 0 ? 0xFFFFFFFFu : 0x80000000u);
}
__device__ __forceinline__ float value_of(uint32_t key) { return __uint_as_float(key & 0x80000000u ? key ^ 0x80000000u : ~key); }

// ---- one row in 64 bits, by a whole wave ------------------------------------------------------------
// The same order as finite doubles.  Beside a NaN logit every softmax is NaN: such choices are alike.
constexpr double ROW_OUT = -4e300, ROW_CLOSED = -1e300, ROW_NAN = 1e300;

__device__ __forceinline__ double wave_max(double v)
{
#pragma unroll
    for (int o = 32; o; o >>= 1) v = fmax(v, __shfl_xor(v, o));
    return v;
}
__device__ __forceinline__ double wave_add(double v)
{
#pragma unroll
    for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o);
    return v;
}

template <class L>
__device__ __forceinline__ void choose_in_64_bits(const rtp_route_desc &d, const L *l, const float *bias, double *key, double *group, int *slot_id, float *slot_l)
{
    const int lane = threadIdx.x & 63, E = d.E, G = d.groups, len = E / G;
    const bool softmax = d.score == RTP_SCORE_SOFTMAX;
    double top = -INFINITY, sum = 0.0;
    if (softmax) {
        bool nan = false;
        for (int e = lane; e < E; e += 64) {
            const double v = (double)(float)l[e];
            nan |= v != v;
            top = fmax(top, v);
        }
        top = wave_max(top);
        if (__any(nan)) top = NAN;
        if (top == -INFINITY) top = 0.0;
        for (int e = lane; e < E; e += 64) sum += exp((double)(float)l[e] - top);
        sum = wave_add(sum);
    }
    wave_fence();
    for (int e = lane; e < E; e += 64) {
        const double v = (double)(float)l[e];
        const double c = v == -INFINITY ? v : (softmax ? exp(v - top) / sum : 1.0 / (1.0 + exp(-v))) + (bias ? (double)bias[e] : 0.0);
        key[e] = v != v ? ROW_NAN : c != c ? 0.0 : fmin(fmax(c, ROW_CLOSED), 0.5 * ROW_NAN);
    }
    wave_fence();
    if (G > 1) {
        if (lane < G) { // a group's score
            double a = ROW_OUT, b = ROW_OUT;
            for (int i = 0; i < len; ++i) {
                const double v = key[lane * len + i];
                b = fmax(b, fmin(a, v));
                a = fmax(a, v);
            }
            group[lane] = d.group_top == 2 && b > ROW_CLOSED ? a + b : a;
        }
        wave_fence();
        for (int g = 0; g < G; ++g) {
            int before = 0;
            for (int o = 0; o < G; ++o) before += group[o] > group[g] || (group[o] == group[g] && o < g);
            if (before >= d.kept_groups)
                for (int i = lane; i < len; i += 64) key[g * len + i] = ROW_OUT;
        }
        wave_fence();
    }
    for (int j = 0; j < d.k; ++j) {
        double best = ROW_OUT;
        int at = E;
        for (int e = lane; e < E; e += 64)
            if (key[e] > best) { best = key[e]; at = e; }
#pragma unroll
        for (int o = 32; o; o >>= 1) {
            const double b = __shfl_xor(best, o);
            const int a = __shfl_xor(at, o);
            if (b > best || (b == best && a < at)) { best = b; at = a; }
        }
        wave_fence();
        if (lane == 0) {
            slot_id[j] = at;
            slot_l[j] = (float)l[at];
            key[at] = ROW_OUT;
        }
        wave_fence();
    }
}

// SCORED: the choice is of scores.  EPL: experts of a lane.
template <rtp_dtype DT, int LANES, int EPL, bool SCORED>
__global__ __launch_bounds__(64 * RW) void route_fwd_kernel(RouteArgs p)
{
    using L = typename Elem<DT>::t;
    constexpr int ROWS = 64 / LANES, SLOTS = ROWS * (LANES * EPL < RTP_ROUTE_MAX_TOP ? LANES * EPL : RTP_ROUTE_MAX_TOP);
    // a wave's keys in 64 bits and group scores, or its rows' in 32 bits
    __shared__ double big[SCORED ? RW : 1][SCORED ? RTP_ROUTE_MAX_EXPERTS + RTP_ROUTE_MAX_GROUPS : 1];
    __shared__ int slot_id[RW][SLOTS];
    __shared__ float slot_l[RW][SLOTS];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, seg = lane / LANES, l = lane % LANES;
    const int E = p.d.E, k = p.d.k, G = p.d.groups, len = E / G;
    const bool softmax = p.d.score == RTP_SCORE_SOFTMAX;
    int *const ids = slot_id[wave] + seg * k;
    float *const ls = slot_l[wave] + seg * k;
    const int left = E - l * EPL; // of this lane's experts that there are
    for (int64_t row0 = ((int64_t)blockIdx.x * RW + wave) * ROWS; row0 < p.d.T; row0 += (int64_t)gridDim.x * RW * ROWS) {
        const int64_t row = min(row0 + seg, p.d.T - 1);
        const L *const logits = (const L *)p.logits + row * p.d.ld;
        float v[EPL];
#pragma unroll
        for (int i = 0; i < EPL; i += 8) {
            Eight<DT> x;
            if (left > i) x.load(logits + l * EPL + i, left - i);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[i + e] = i + e < left ? x.get(e) : -INFINITY;
        }
        // sum over the row, which the scores of a softmax divide by
        float top = -INFINITY, sum = 1.0f;
        if (softmax && (SCORED || !p.d.renormalise)) {
#pragma unroll
            for (int e = 0; e < EPL; ++e) top = fmaxf(top, v[e]);
            top = over_fmax<LANES>(top);
            if (top == -INFINITY) top = 0.0f;
            sum = 0.0f;
#pragma unroll
            for (int e = 0; e < EPL; ++e) sum += expf(v[e] - top);
            sum = over_sum<LANES>(sum);
        }
        uint32_t key[EPL];
        bool unsure = false;
        if (SCORED) {
            const float inv = 1.0f / sum;
#pragma unroll
            for (int e = 0; e < EPL; ++e) {
                const float b = p.bias && e < left ? p.bias[l * EPL + e] : 0.0f;
                const float c = (softmax ? expf(v[e] - top) * inv : 1.0f / (1.0f + expf(-v[e]))) + b;
                unsure |= e < left && (!(fabsf(c) < INFINITY) || v[e] == INFINITY) && v[e] != -INFINITY;
                key[e] = v[e] == -INFINITY ? KEY_CLOSED : key_of(c);
            }
        } else {
#pragma unroll
            for (int e = 0; e < EPL; ++e) key[e] = key_of(v[e]);
        }
#pragma unroll
        for (int e = 0; e < EPL; ++e)
            if (e >= left) key[e] = KEY_OUT;
        // Two numbers closer than this may be in the other order.  A score is off by 2^-19 of itself at most (the 22 roundings of a
        // sum of 1024 terms, the exponential and the quotient 3 more, and by a denormal), a choice by half a step of the row's largest
        // on top: four times that.
        float close = 0x1p-126f;
        if (SCORED && p.bias) {
            float most = 0.0f;
#pragma unroll
            for (int e = 0; e < EPL; ++e)
                if (key[e] > KEY_CLOSED) most = fmaxf(most, fabsf(value_of(key[e])));
            close = 0x1p-17f * (softmax ? 1.0f / sum : 1.0f) + 0x1p-22f * over_fmax<LANES>(most);
        }
        auto apart = [&](float a) { return p.bias ? close : 0x1p-17f * a + close; };
        if (SCORED && G > 1) {
            uint32_t *const keys = (uint32_t *)big[wave] + seg * E;
            float *const group = (float *)(big[wave] + RTP_ROUTE_MAX_EXPERTS / 2) + seg * G;
            wave_fence();
#pragma unroll
            for (int e = 0; e < EPL; ++e)
                if (e < left) keys[l * EPL + e] = key[e];
            wave_fence();
            // S lanes to a group
            int S = LANES;
            while (S > 1 && S * G > LANES) S >>= 1;
            for (int g0 = 0; g0 < G; g0 += LANES / S) {
                const int g = g0 + l / S;
                uint32_t a = KEY_OUT, b = KEY_OUT;
                if (g < G)
                    for (int i = l % S; i < len; i += S) {
                        const uint32_t x = keys[g * len + i];
                        b = max(b, min(a, x));
                        a = max(a, x);
                    }
                for (int o = 1; o < S; o <<= 1) {
                    const uint32_t c = __shfl_xor(a, o), d = __shfl_xor(b, o);
                    b = max(max(b, d), min(a, c));
                    a = max(a, c);
                }
                if (g < G && l % S == 0)
                    group[g] = a <= KEY_CLOSED ? -INFINITY : value_of(a) + (p.d.group_top == 2 && b > KEY_CLOSED ? value_of(b) : 0.0f);
            }
            wave_fence();
            for (int g0 = 0; g0 < G; g0 += LANES / S) {
                const int g = g0 + l / S;
                if (g >= G) continue;
                const float mine = group[g];
                int before = 0;
                for (int o = 0; o < G; ++o) {
                    const float other = group[o];
                    before += other > mine || (other == mine && o < g);
                    unsure |= o != g && mine > -INFINITY && fabsf(other - mine) < 2.0f * apart(mine);
                }
                if (before >= p.d.kept_groups)
                    for (int i = l % S; i < len; i += S) keys[g * len + i] = KEY_OUT;
            }
            wave_fence();
#pragma unroll
            for (int e = 0; e < EPL; ++e)
                if (e < left) key[e] = keys[l * EPL + e];
        }
        uint32_t last = 0;
        for (int j = 0; j < k + (SCORED ? 1 : 0); ++j) {
            uint32_t best = KEY_OUT;
#pragma unroll
            for (int e = 0; e < EPL; ++e) best = max(best, key[e]);
            const uint32_t most = over_max<LANES>(best);
            if (SCORED) {
                if (j > 0 && most > KEY_CLOSED) unsure |= value_of(last) - value_of(most) < apart(value_of(last));
                last = most;
                if (j == k) break;
            }
            // the lowest lane that has it, and its first key of that value
            const uint64_t have = __ballot(best == most);
            const uint64_t mine = LANES == 64 ? have : have >> (seg * LANES) & ((1ull << (LANES & 63)) - 1);
            if (l == __ffsll((unsigned long long)mine) - 1) {
                int at = 0;
                float x = 0.0f;
#pragma unroll
                for (int e = EPL - 1; e >= 0; --e)
                    if (key[e] == most) { at = e; x = v[e]; }
#pragma unroll
                for (int e = 0; e < EPL; ++e)
                    if (e == at) key[e] = KEY_OUT;
                ids[j] = l * EPL + at;
                ls[j] = x;
            }
        }
        if (SCORED) {
            uint64_t again = __ballot(unsure);
            while (again) {
                const int s = (__ffsll((unsigned long long)again) - 1) / LANES;
                again &= LANES == 64 ? 0 : ~(((1ull << (LANES & 63)) - 1) << (s * LANES));
                const int64_t r = min(row0 + s, p.d.T - 1);
                choose_in_64_bits<L>(p.d, (const L *)p.logits + r * p.d.ld, p.bias, big[wave], big[wave] + RTP_ROUTE_MAX_EXPERTS,
                                     slot_id[wave] + s * k, slot_l[wave] + s * k);
            }
        }
        wave_fence();
        if (row0 + seg < p.d.T) {
            // renormalised: a softmax over the chosen logits, or over log sigmoid of them (what the sum over all experts or a tiny sigmoid
            // would divide by cancels)
            float m = -INFINITY, z = 0.0f;
            if (p.d.renormalise) {
                for (int j = 0; j < k; ++j) m = fmaxf(m, softmax ? ls[j] : log_sigmoid(ls[j]));
                if (m == -INFINITY) m = 0.0f;
                for (int j = 0; j < k; ++j) z += ls[j] == -INFINITY ? 0.0f : expf((softmax ? ls[j] : log_sigmoid(ls[j])) - m);
            }
            for (int j = l; j < k; j += LANES) {
                const float x = ls[j];
                float s = p.d.renormalise ? expf((softmax ? x : log_sigmoid(x)) - m) / z : softmax ? expf(x - top) / sum : 1.0f / (1.0f + expf(-x));
                if (x == -INFINITY) s = 0.0f;
                p.ids[row * k + j] = ids[j];
                p.weights[row * k + j] = p.d.scale * s;
            }
        }
        wave_fence();
    }
}

template <rtp_dtype DT, rtp_dtype GT>
__global__ __launch_bounds__(64 * RW) void route_bwd_wave_kernel(RouteArgs p)
{
    using L = typename Elem<DT>::t;
    using G = typename Elem<GT>::t;
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, E = p.d.E, k = p.d.k;
    const bool softmax = p.d.score == RTP_SCORE_SOFTMAX;
    const float scale = p.d.scale;
    for (int64_t row = (int64_t)blockIdx.x * RW + w; row < p.d.T; row += (int64_t)gridDim.x * RW) {
        const L *l = (const L *)p.logits + row * p.d.ld;
        G *out = (G *)p.dlogits + row * p.d.ld_grad;
        const int32_t *ids = p.ids_in + row * k;
        const float *a = p.dweights + row * k;
        auto logit = [&](int j) { // of a slot that has a part in the gradient, else -infinity
            const int e = ids[j];
            return (unsigned)e < (unsigned)E ? (float)l[e] : -INFINITY;
        };
        auto lg = [&](float v) { return softmax ? v : log_sigmoid(v); };
        float m = -INFINITY, z = 0.0f, dot = 0.0f;
        if (p.d.renormalise) { // (NaN: the maximum passes it over, the sums do not)
            for (int j = 0; j < k; ++j) m = fmaxf(m, lg(logit(j)));
            if (m == -INFINITY) m = 0.0f;
            for (int j = 0; j < k; ++j) {
                const float v = logit(j), x = v == -INFINITY ? 0.0f : expf(lg(v) - m);
                z += x;
                dot += x == 0.0f ? 0.0f : x * a[j];
            }
            dot /= z > 0.0f ? z : 1.0f;
        } else if (softmax) {
            for (int e = lane; e < E; e += 64) m = fmaxf(m, (float)l[e]);
#pragma unroll
            for (int o = 32; o; o >>= 1) m = fmaxf(m, __shfl_xor(m, o));
            if (m == -INFINITY) m = 0.0f;
            for (int e = lane; e < E; e += 64) z += expf((float)l[e] - m);
            z = wave_sum(z);
            for (int j = 0; j < k; ++j) {
                const float v = logit(j);
                dot += v == -INFINITY ? 0.0f : expf(v - m) / z * a[j];
            }
        }
        for (int e = lane; e < E; e += 64) {
            const float v = (float)l[e];
            float g = 0.0f, n = 0.0f; // sum of the slots' gradients, and how many name this expert
            for (int j = 0; j < k; ++j)
                if (ids[j] == e) { g += a[j]; n += 1.0f; }
            float d = 0.0f;
            if (v != -INFINITY) {
                const float sig = 1.0f / (1.0f + expf(-v));
                if (p.d.renormalise)
                    d = n == 0.0f ? 0.0f : expf(lg(v) - m) / z * (g - n * dot) * (softmax ? 1.0f : 1.0f - sig);
                else if (softmax)
                    d = expf(v - m) / z * (g - dot);
                else
                    d = n == 0.0f ? 0.0f : sig * (1.0f - sig) * g;
            }
            out[e] = (G)(scale * d);
        }
    }
}

template <class F>
static hipError_t by_type(rtp_dtype t, F f)
{
    if (t == RTP_F32) return f.template operator()<RTP_F32>();
    if (t == RTP_BF16) return f.template operator()<RTP_BF16>();
    return f.template operator()<RTP_F16>();
}

static unsigned route_grid(int64_t T, int rows = 1) { return (unsigned)std::min<int64_t>((T + RW * rows - 1) / (RW * rows), 1 << 20); }

struct RouteFwd {
    const RouteArgs &p;
    hipStream_t s;
    template <rtp_dtype DT, int LANES, int EPL> hipError_t launch()
    {
        const unsigned grid = route_grid(p.d.T, 64 / LANES);
        if (p.bias || p.d.groups > 1) route_fwd_kernel<DT, LANES, EPL, true><<<grid, 64 * RW, 0, s>>>(p);
        else route_fwd_kernel<DT, LANES, EPL, false><<<grid, 64 * RW, 0, s>>>(p);
        return hipGetLastError();
    }
    template <rtp_dtype DT> hipError_t operator()()
    {
        // eight experts a lane, sixteen where 64 lanes are not enough
        if (p.d.E <= 8) return launch<DT, 1, 8>();
        if (p.d.E <= 16) return launch<DT, 2, 8>();
        if (p.d.E <= 32) return launch<DT, 4, 8>();
        if (p.d.E <= 64) return launch<DT, 8, 8>();
        if (p.d.E <= 128) return launch<DT, 16, 8>();
        if (p.d.E <= 256) return launch<DT, 32, 8>();
        if (p.d.E <= 512) return launch<DT, 64, 8>();
        return launch<DT, 64, 16>();
    }
};

hipError_t launch_route_fwd(const rtp_route_desc &d, const void *logits, const float *bias, int32_t *ids, float *weights, hipStream_t s)
{
    const RouteArgs p{d, logits, bias, ids, weights, nullptr, nullptr, nullptr};
    return by_type(d.dtype, RouteFwd{p, s});
}

template <rtp_dtype DT> struct RouteBwdTo {
    const RouteArgs &p;
    hipStream_t s;
    template <rtp_dtype GT> hipError_t operator()()
    {
        route_bwd_wave_kernel<DT, GT><<<route_grid(p.d.T), 64 * RW, 0, s>>>(p);
        return hipGetLastError();
    }
};
struct RouteBwd {
    const RouteArgs &p;
    hipStream_t s;
    template <rtp_dtype DT> hipError_t operator()() { return by_type(p.d.grad_dtype, RouteBwdTo<DT>{p, s}); }
};

hipError_t launch_route_bwd(const rtp_route_desc &d, const void *logits, const int32_t *ids, const float *dweights, void *dlogits, hipStream_t s)
{
    const RouteArgs p{d, logits, nullptr, nullptr, nullptr, ids, dweights, dlogits};
    return by_type(d.dtype, RouteBwd{p, s});
}

} // namespace rtp
