// Routing to experts (rtp_route_fwd, rtp_route_bwd).
#include "rtp_block_kernels.h"
#include "rtp_elem.h"
#include <algorithm>
#include <cmath>

namespace rtp {

// Bound: latency and the instructions of the choice (a row of 256 is 1 KB; its eight largest are eight rounds of comparisons).  LANES lanes
// share a row, eight or sixteen neighbouring experts each, 64 / LANES rows to a wave: a round is then a maximum over a lane's keys, one
// over LANES lanes, and the lowest lane that has it, with no barrier and little LDS.  Keys are 32-bit integers in the order of what they
// stand for.  Where the choice is of scores (a bias, groups), they are scores in 32 bits; a row in which two of them that
// matter are closer than 32 bits can tell apart is decided again in 64 bits: the chosen are put in order among themselves, or, where
// it is in doubt who they are, the whole wave chooses again.
// 16384 tokens over 256 experts in 8 groups, 8 a token: 30 us (all rows in 64 bits, a wave a row: 117); 23 are the 32-bit choice, of
// which the groups 4, the rest the few rows in doubt (0.1 %), behind the last ones: 4 us to choose one again.  The path that does so is
// in the same kernel: its 123 registers (52 where the choice is of logits) and 36 KB of LDS leave four waves a SIMD to hide latency.
// Sixteen lanes of sixteen instead of 32 of eight: 34.  8192 over 8, two a token: 4.5 us, latency.
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

// f over the wave, in every lane
template <class F> __device__ __forceinline__ double over_wave(double v, F f)
{
    uint32_t lo = (uint32_t)__double2loint(v), hi = (uint32_t)__double2hiint(v);
    auto step = [&](uint32_t l, uint32_t h) {
        const double r = f(__hiloint2double((int)hi, (int)lo), __hiloint2double((int)h, (int)l));
        lo = (uint32_t)__double2loint(r);
        hi = (uint32_t)__double2hiint(r);
    };
    step(dpp<DPP_XOR1>(lo), dpp<DPP_XOR1>(hi));
    step(dpp<DPP_XOR2>(lo), dpp<DPP_XOR2>(hi));
    step(dpp<DPP_HALF_MIRROR>(lo), dpp<DPP_HALF_MIRROR>(hi));
    step(dpp<DPP_MIRROR>(lo), dpp<DPP_MIRROR>(hi));
#pragma unroll
    for (int half = 16; half <= 32; half *= 2) {
        const auto l = half == 16 ? __builtin_amdgcn_permlane16_swap(lo, lo, false, false) : __builtin_amdgcn_permlane32_swap(lo, lo, false, false);
        const auto h = half == 16 ? __builtin_amdgcn_permlane16_swap(hi, hi, false, false) : __builtin_amdgcn_permlane32_swap(hi, hi, false, false);
        lo = (uint32_t)l[0];
        hi = (uint32_t)h[0];
        step((uint32_t)l[1], (uint32_t)h[1]);
    }
    return __hiloint2double((int)hi, (int)lo);
}
__device__ __forceinline__ double wave_max(double v)
{
    return over_wave(v, [](double a, double b) { return fmax(a, b); });
}

// EACH: experts of a lane, neighbours, in registers.  (`key` and `group`: LDS, for groups alone.)
template <int EACH, class L>
__device__ __forceinline__ void choose_in_64_bits(const rtp_route_desc &d, const L *l, const float *bias, double *key, double *group, int *slot_id)
{
    const int lane = threadIdx.x & 63, E = d.E, G = d.groups, first = lane * EACH;
    const bool softmax = d.score == RTP_SCORE_SOFTMAX;
    double v[EACH], c[EACH], add[EACH];
#pragma unroll
    for (int e = 0; e < EACH; ++e) {
        v[e] = first + e < E ? (double)(float)l[first + e] : -INFINITY;
        add[e] = bias && first + e < E ? (double)bias[first + e] : 0.0;
    }
    double top = -INFINITY, sum = 0.0;
    if (softmax) {
        bool nan = false;
#pragma unroll
        for (int e = 0; e < EACH; ++e) {
            nan |= v[e] != v[e];
            top = fmax(top, v[e]);
        }
        top = wave_max(top);
        if (__any(nan)) top = NAN;
        if (top == -INFINITY) top = 0.0;
#pragma unroll
        for (int e = 0; e < EACH; ++e) sum += exp(v[e] - top);
        sum = over_wave(sum, [](double a, double b) { return a + b; });
    }
#pragma unroll
    for (int e = 0; e < EACH; ++e) {
        c[e] = v[e] == -INFINITY ? v[e] : (softmax ? exp(v[e] - top) / sum : 1.0 / (1.0 + exp(-v[e]))) + add[e];
        c[e] = v[e] != v[e] ? ROW_NAN : c[e] != c[e] ? 0.0 : fmin(fmax(c[e], ROW_CLOSED), 0.5 * ROW_NAN);
        if (first + e >= E) c[e] = ROW_OUT;
    }
    if (G > 1) {
        const int len = E / G;
        wave_fence();
#pragma unroll
        for (int e = 0; e < EACH; ++e)
            if (first + e < E) key[first + e] = c[e];
        wave_fence();
        int S = 64; // lanes to a group
        while (S * G > 64) S >>= 1;
        const int g = lane / S;
        double a = ROW_OUT, b = ROW_OUT;
        if (g < G) {
#pragma unroll 4
            for (int i = lane % S; i < len; i += S) {
                const double x = key[g * len + i];
                b = fmax(b, fmin(a, x));
                a = fmax(a, x);
            }
        }
        for (int o = 1; o < S; o <<= 1) {
            const double x = __shfl_xor(a, o), y = __shfl_xor(b, o);
            b = fmax(fmax(b, y), fmin(a, x));
            a = fmax(a, x);
        }
        if (d.group_top == 2 && b > ROW_CLOSED) a += b;
        if (g < G && lane % S == 0) group[g] = a;
        wave_fence();
        int before = 0;
#pragma unroll 4
        for (int o = 0; o < G; ++o) before += group[o] > a || (group[o] == a && o < g);
        if (g < G && before >= d.kept_groups)
            for (int i = lane % S; i < len; i += S) key[g * len + i] = ROW_OUT;
        wave_fence();
#pragma unroll
        for (int e = 0; e < EACH; ++e)
            if (first + e < E) c[e] = key[first + e];
    }
    for (int j = 0; j < d.k; ++j) {
        double best = c[0];
        int at = 0;
#pragma unroll
        for (int e = 1; e < EACH; ++e)
            if (c[e] > best) { best = c[e]; at = e; }
        // (a lane's experts are neighbours: the lowest lane has the lowest index)
        const double most = wave_max(best);
        if (lane == __ffsll((unsigned long long)__ballot(best == most)) - 1) {
            slot_id[j] = first + at;
#pragma unroll
            for (int e = 0; e < EACH; ++e)
                if (e == at) c[e] = ROW_OUT;
        }
    }
    wave_fence();
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
    __shared__ float slot_s[RW][SLOTS];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, seg = lane / LANES, l = lane % LANES;
    const int E = p.d.E, k = p.d.k, G = p.d.groups, len = E / G;
    const bool softmax = p.d.score == RTP_SCORE_SOFTMAX;
    int *const ids = slot_id[wave] + seg * k;
    float *const ss = slot_s[wave] + seg * k;
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
        bool unsure = false, disordered = false; // who is chosen, and in which order they are
        // Two numbers closer than `near` of themselves, or than `close`, may be in the other order.  A sigmoid is off by 2.5 2^-23 of
        // itself (exponential, sum, reciprocal), a softmax by as much, by |l - top| 2^-24, and by its sum, which is the same for all
        // of a row: 22 roundings for 1024 terms.  A choice is off by half a step of the row's largest on top; two of them by twice
        // all that.
        const float near = softmax ? 0x1p-17f : 0x1p-20f;
        float close = softmax ? 0x1p-90f : 0x1p-126f; // (a smaller exponential is off by more)
        if (SCORED) {
            const float inv = softmax ? 1.0f / sum : 1.0f;
            float most = 0.0f;
#pragma unroll
            for (int e = 0; e < EPL; ++e) {
                const float b = p.bias && e < left ? p.bias[l * EPL + e] : 0.0f;
                const float x = softmax ? expf(v[e] - top) * inv : __builtin_amdgcn_rcpf(1.0f + expf(-v[e]));
                const float c = v[e] == -INFINITY ? 0.0f : x + b;
                unsure |= !(fabsf(c) < INFINITY);
                most = fmaxf(most, fabsf(c));
                key[e] = v[e] == -INFINITY ? KEY_CLOSED : key_of(c);
            }
            if (p.bias) close = near * inv + 0x1p-22f * over_fmax<LANES>(most);
        } else {
#pragma unroll
            for (int e = 0; e < EPL; ++e) key[e] = key_of(v[e]);
        }
#pragma unroll
        for (int e = 0; e < EPL; ++e)
            if (e >= left) key[e] = KEY_OUT;
        auto apart = [&](float a) { return p.bias ? close : near * a + close; };
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
                }
                const bool out = before >= p.d.kept_groups;
                // (which of two kept groups is the better one does not matter: only one that is out, and as good as one that is not)
                if (out && mine > -INFINITY) {
                    int better = 0; // by more than what may be in the other order
                    for (int o = 0; o < G; ++o) better += group[o] - mine >= 2.0f * apart(mine);
                    unsure |= better < p.d.kept_groups;
                }
                if (out)
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
                if (j > 0 && most > KEY_CLOSED && value_of(last) - value_of(most) < apart(value_of(last))) {
                    // (the order of a softmax with a bias takes its sum in 64 bits, and that of vanishing ones is of equals)
                    if (j < k && (softmax ? !p.bias && value_of(most) > 0x1p-80f : true)) disordered = true;
                    else unsure = true;
                }
                last = most;
                if (j == k) break;
            }
            // the lowest lane that has it, and its first key of that value
            const uint64_t have = __ballot(best == most);
            const uint64_t mine = LANES == 64 ? have : have >> (seg * LANES) & ((1ull << (LANES & 63)) - 1);
            if (l == __ffsll((unsigned long long)mine) - 1) {
                int at = 0;
#pragma unroll
                for (int e = EPL - 1; e >= 0; --e)
                    if (key[e] == most) at = e;
#pragma unroll
                for (int e = 0; e < EPL; ++e)
                    if (e == at) key[e] = KEY_OUT;
                ids[j] = l * EPL + at;
            }
        }
        if (SCORED && disordered) { // the chosen among themselves: each counts the better ones
            double *const c = big[wave] + seg * k;
            int *const sorted = (int *)ss;
            wave_fence();
            for (int j = l; j < k; j += LANES) {
                const double x = (double)(float)logits[ids[j]];
                c[j] = x == -INFINITY ? ROW_CLOSED : softmax ? x : 1.0 / (1.0 + exp(-x)) + (p.bias ? (double)p.bias[ids[j]] : 0.0);
            }
            wave_fence();
            for (int j = l; j < k; j += LANES) {
                int better = 0;
                for (int o = 0; o < k; ++o) {
                    better += c[o] > c[j] || (c[o] == c[j] && ids[o] < ids[j]);
                    // (Logits stand for their softmax here, whose probabilities are above 2^-80, so that l - top is off by 2^-47 in 64
                    // bits, and two are in the order of their logits if these are 2^-44 apart.  Nearer ones may be equal there: the whole
                    // row says.)
                    unsure |= softmax && !p.bias && c[o] != c[j] && fabs(c[o] - c[j]) < 0x1p-44;
                }
                sorted[better] = ids[j];
            }
            wave_fence();
            for (int j = l; j < k; j += LANES) ids[j] = sorted[j];
            wave_fence();
        }
        if (SCORED) {
            uint64_t again = __ballot(unsure);
            while (again) {
                const int s = (__ffsll((unsigned long long)again) - 1) / LANES;
                again &= LANES == 64 ? 0 : ~(((1ull << (LANES & 63)) - 1) << (s * LANES));
                const int64_t r = min(row0 + s, p.d.T - 1);
                choose_in_64_bits<(LANES * EPL + 63) / 64>(p.d, (const L *)p.logits + r * p.d.ld, p.bias, big[wave], big[wave] + RTP_ROUTE_MAX_EXPERTS, slot_id[wave] + s * k);
            }
        }
        wave_fence();
        // weights: lane l has slots l, l + LANES, ..., and all of a row's lanes see its k numbers in LDS
        auto exchange = [&](auto number) {
            wave_fence();
            for (int j = l; j < k; j += LANES) ss[j] = number((float)logits[ids[j]]);
            wave_fence();
        };
        auto total = [&]() {
            float z = 0.0f;
            for (int j = 0; j < k; ++j) z += ss[j];
            return z;
        };
        // (a softmax over the chosen: what the sum over all experts, or a sigmoid that underflows, would divide by cancels)
        auto relative = [&](auto log_of) {
            float m = -INFINITY;
            exchange(log_of);
            for (int j = 0; j < k; ++j) m = fmaxf(m, ss[j]);
            if (m == -INFINITY) m = 0.0f;
            exchange([&](float x) { return x == -INFINITY ? 0.0f : expf(log_of(x) - m); });
        };
        auto sigmoid = [](float x) { return 1.0f / (1.0f + expf(-x)); };
        float z = 1.0f;
        if (softmax && p.d.renormalise) {
            relative([](float x) { return x; });
            z = total();
        } else if (softmax) {
            exchange([&](float x) { return x == -INFINITY ? 0.0f : expf(x - top) / sum; });
        } else {
            exchange(sigmoid);
            if (p.d.renormalise) {
                z = total();
                if (z < 0x1p-100f) { // sigmoids that lose bits, or vanish: from their logarithms
                    relative(log_sigmoid);
                    z = total();
                }
            }
        }
        if (row0 + seg < p.d.T) {
            for (int j = l; j < k; j += LANES) {
                p.ids[row * k + j] = ids[j];
                p.weights[row * k + j] = p.d.scale * (ss[j] == 0.0f ? 0.0f : ss[j] / z);
            }
        }
        wave_fence();
    }
}

// Gradient of the logits, rows and lanes as in the forward pass.  Bound: HBM for many tokens (every entry is read and written), latency for
// few (5003 tokens over 150: 7.3 us; a wave a row 9.4).  With d_j = a_j - sum of w_i a_i / scale: renormalised, dl_j = w_j d_j (softmax), w_j (1 - s_j) d_j (sigmoid), nothing
// elsewhere; else dl_e = scale p_e ([chosen] a - sum of p_i a_i), scale s (1 - s) a.
template <rtp_dtype DT, rtp_dtype GT, int LANES, int EPL>
__global__ __launch_bounds__(64 * RW) void route_bwd_kernel(RouteArgs p)
{
    using L = typename Elem<DT>::t;
    constexpr int ROWS = 64 / LANES, SLOTS = ROWS * (LANES * EPL < RTP_ROUTE_MAX_TOP ? LANES * EPL : RTP_ROUTE_MAX_TOP);
    __shared__ int slot_id[RW][SLOTS];
    __shared__ float slot_a[RW][SLOTS], slot_x[RW][SLOTS]; // gradient of a slot's weight, its logit
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, seg = lane / LANES, l = lane % LANES;
    const int E = p.d.E, k = p.d.k;
    const bool softmax = p.d.score == RTP_SCORE_SOFTMAX, renorm = p.d.renormalise;
    int *const ids = slot_id[wave] + seg * k;
    float *const as = slot_a[wave] + seg * k, *const xs = slot_x[wave] + seg * k;
    const int left = E - l * EPL;
    for (int64_t row0 = ((int64_t)blockIdx.x * RW + wave) * ROWS; row0 < p.d.T; row0 += (int64_t)gridDim.x * RW * ROWS) {
        const int64_t row = min(row0 + seg, p.d.T - 1);
        const L *const logits = (const L *)p.logits + row * p.d.ld;
        wave_fence();
        for (int j = l; j < k; j += LANES) {
            const int e = p.ids_in[row * k + j];
            const bool there = (unsigned)e < (unsigned)E;
            const float x = there ? (float)logits[e] : -INFINITY;
            ids[j] = there ? e : -1;
            xs[j] = x;
            as[j] = x == -INFINITY ? 0.0f : p.dweights[row * k + j]; // (closed: whatever came back has no part)
        }
        float v[EPL];
#pragma unroll
        for (int i = 0; i < EPL; i += 8) {
            Eight<DT> x;
            if (left > i) x.load(logits + l * EPL + i, left - i);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[i + e] = i + e < left ? x.get(e) : -INFINITY;
        }
        wave_fence();
        // maximum and sum of the exponentials that the weights are quotients of (NaN: the maximum passes it over, the sum does not)
        auto lg = [&](float x) { return softmax ? x : log_sigmoid(x); };
        float m = -INFINITY, z = 0.0f, dot = 0.0f;
        if (renorm) {
            for (int j = 0; j < k; ++j) m = fmaxf(m, lg(xs[j]));
            if (m == -INFINITY) m = 0.0f;
            for (int j = 0; j < k; ++j) {
                const float x = xs[j] == -INFINITY ? 0.0f : expf(lg(xs[j]) - m);
                z += x;
                dot += x == 0.0f ? 0.0f : x * as[j];
            }
        } else if (softmax) {
#pragma unroll
            for (int e = 0; e < EPL; ++e) m = fmaxf(m, v[e]);
            m = over_fmax<LANES>(m);
            if (m == -INFINITY) m = 0.0f;
#pragma unroll
            for (int e = 0; e < EPL; ++e) z += expf(v[e] - m);
            z = over_sum<LANES>(z);
            for (int j = 0; j < k; ++j) dot += xs[j] == -INFINITY ? 0.0f : expf(xs[j] - m) * as[j];
        }
        if (z == 0.0f) z = 1.0f;
        dot /= z;
        // what the slots that name this lane's experts bring, and how many do
        float g[EPL], n[EPL];
#pragma unroll
        for (int e = 0; e < EPL; ++e) g[e] = n[e] = 0.0f;
        for (int j = 0; j < k; ++j) {
            const int at = ids[j] - l * EPL;
            const float a = as[j];
#pragma unroll
            for (int e = 0; e < EPL; ++e) {
                g[e] += e == at ? a : 0.0f;
                n[e] += e == at ? 1.0f : 0.0f;
            }
        }
        if (row0 + seg < p.d.T) {
            float o[EPL];
#pragma unroll
            for (int e = 0; e < EPL; ++e) {
                float d = 0.0f;
                const bool open = v[e] != -INFINITY;
                if (softmax && !renorm) {
                    d = open ? expf(v[e] - m) / z * (g[e] - dot) : 0.0f;
                } else if (open && n[e] > 0.0f) {
                    // (1 - s is the sigmoid of -l: of s itself nothing would be left of it from l = 17 on)
                    const float sig = 1.0f / (1.0f + expf(-v[e])), rest = 1.0f / (1.0f + expf(v[e]));
                    d = renorm ? expf(lg(v[e]) - m) / z * (g[e] - n[e] * dot) * (softmax ? 1.0f : rest) : sig * rest * g[e];
                }
                o[e] = p.d.scale * d;
            }
            using G = typename Elem<GT>::t;
#pragma unroll
            for (int i = 0; i < EPL; i += 8) {
                if (left <= i) continue;
                Eight<GT> x;
                float t[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) t[e] = o[i + e];
                x.set(t);
                x.store((G *)p.dlogits + row * p.d.ld_grad + l * EPL + i, left - i);
            }
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

static unsigned route_grid(int64_t T, int rows) { return (unsigned)std::min<int64_t>((T + RW * rows - 1) / (RW * rows), 1 << 20); }

// f.launch<LANES, EPL>(): eight experts a lane, sixteen where 64 lanes are not enough
template <class F>
static hipError_t by_experts(int E, F &f)
{
    if (E <= 8) return f.template launch<1, 8>();
    if (E <= 16) return f.template launch<2, 8>();
    if (E <= 32) return f.template launch<4, 8>();
    if (E <= 64) return f.template launch<8, 8>();
    if (E <= 128) return f.template launch<16, 8>();
    if (E <= 256) return f.template launch<32, 8>();
    if (E <= 512) return f.template launch<64, 8>();
    return f.template launch<64, 16>();
}

template <rtp_dtype DT> struct RouteFwdOf {
    const RouteArgs &p;
    hipStream_t s;
    template <int LANES, int EPL> hipError_t launch()
    {
        const unsigned grid = route_grid(p.d.T, 64 / LANES);
        if (p.bias || p.d.groups > 1) route_fwd_kernel<DT, LANES, EPL, true><<<grid, 64 * RW, 0, s>>>(p);
        else route_fwd_kernel<DT, LANES, EPL, false><<<grid, 64 * RW, 0, s>>>(p);
        return hipGetLastError();
    }
};
struct RouteFwd {
    const RouteArgs &p;
    hipStream_t s;
    template <rtp_dtype DT> hipError_t operator()()
    {
        RouteFwdOf<DT> f{p, s};
        return by_experts(p.d.E, f);
    }
};

hipError_t launch_route_fwd(const rtp_route_desc &d, const void *logits, const float *bias, int32_t *ids, float *weights, hipStream_t s)
{
    const RouteArgs p{d, logits, bias, ids, weights, nullptr, nullptr, nullptr};
    return by_type(d.dtype, RouteFwd{p, s});
}

template <rtp_dtype DT, rtp_dtype GT> struct RouteBwdOf {
    const RouteArgs &p;
    hipStream_t s;
    template <int LANES, int EPL> hipError_t launch()
    {
        route_bwd_kernel<DT, GT, LANES, EPL><<<route_grid(p.d.T, 64 / LANES), 64 * RW, 0, s>>>(p);
        return hipGetLastError();
    }
};
template <rtp_dtype DT> struct RouteBwdTo {
    const RouteArgs &p;
    hipStream_t s;
    template <rtp_dtype GT> hipError_t operator()()
    {
        RouteBwdOf<DT, GT> f{p, s};
        return by_experts(p.d.E, f);
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
