// Routing to experts (rtp_route_fwd, rtp_route_bwd).
#include "rtp_block_kernels.h"
#include "rtp_elem.h"
#include <algorithm>
#include <cmath>

namespace rtp {

constexpr int RW = 4; // waves of a workgroup, a row each

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

// What an expert is ranked by, as finite numbers: out of the choice (taken, of another group, not there) < closed < any choice < a NaN
// logit.  (Beside a NaN logit every softmax is NaN: such choices are alike.)
constexpr double KEY_NONE = -4e300, KEY_CLOSED = -1e300, KEY_NAN = 1e300;

__device__ __forceinline__ double rank_key(double logit, double choice)
{
    if (logit != logit) return KEY_NAN;
    if (choice != choice) return 0.0;
    return fmin(fmax(choice, KEY_CLOSED), 0.5 * KEY_NAN);
}

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

// log of a sigmoid, without the underflow of the sigmoid itself
__device__ __forceinline__ float log_sigmoid(float l) { return fminf(l, 0.0f) - log1pf(expf(-fabsf(l))); }

template <rtp_dtype DT>
__global__ __launch_bounds__(64 * RW) void route_fwd_wave_kernel(RouteArgs p)
{
    using L = typename Elem<DT>::t;
    __shared__ double keys[RW][RTP_ROUTE_MAX_EXPERTS];
    __shared__ double group[RW][RTP_ROUTE_MAX_GROUPS];
    __shared__ float slot_l[RW][RTP_ROUTE_MAX_TOP], slot_s[RW][RTP_ROUTE_MAX_TOP];
    __shared__ int slot_id[RW][RTP_ROUTE_MAX_TOP];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, E = p.d.E, k = p.d.k, G = p.d.groups, len = E / G;
    const bool softmax = p.d.score == RTP_SCORE_SOFTMAX, scored = p.bias || G > 1;
    double *key = keys[w];
    for (int64_t row0 = (int64_t)blockIdx.x * RW; row0 < p.d.T; row0 += (int64_t)gridDim.x * RW) {
        const int64_t row = row0 + w;
        const bool on = row < p.d.T;
        const L *l = (const L *)p.logits + (on ? row : 0) * p.d.ld;
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
        auto score = [&](double v) {
            return softmax ? (v == -INFINITY ? 0.0 : exp(v - top) / sum) : 1.0 / (1.0 + exp(-v));
        };
        for (int e = lane; e < E; e += 64) {
            const double v = (double)(float)l[e];
            key[e] = rank_key(v, !scored || v == -INFINITY ? v : score(v) + (p.bias ? (double)p.bias[e] : 0.0));
        }
        __syncthreads();
        if (G > 1) {
            if (lane < G) { // a group's score
                double a = KEY_NONE, b = KEY_NONE;
                for (int i = 0; i < len; ++i) {
                    const double v = key[lane * len + i];
                    b = fmax(b, fmin(a, v));
                    a = fmax(a, v);
                }
                group[w][lane] = p.d.group_top == 2 && b > KEY_CLOSED ? a + b : a;
            }
            __syncthreads();
            for (int g = 0; g < G; ++g) {
                int before = 0;
                for (int o = 0; o < G; ++o) before += group[w][o] > group[w][g] || (group[w][o] == group[w][g] && o < g);
                if (before >= p.d.kept_groups)
                    for (int i = lane; i < len; i += 64) key[g * len + i] = KEY_NONE;
            }
            __syncthreads();
        }
        for (int j = 0; j < k; ++j) {
            double best = KEY_NONE;
            int at = E;
            for (int e = lane; e < E; e += 64)
                if (key[e] > best) { best = key[e]; at = e; }
#pragma unroll
            for (int o = 32; o; o >>= 1) {
                const double b = __shfl_xor(best, o);
                const int a = __shfl_xor(at, o);
                if (b > best || (b == best && a < at)) { best = b; at = a; }
            }
            if (lane == 0) {
                const float v = (float)l[at];
                slot_id[w][j] = at;
                slot_l[w][j] = v;
                slot_s[w][j] = p.d.renormalise ? 0.0f : (float)score((double)v);
                key[at] = KEY_NONE;
            }
            __syncthreads();
        }
        if (on && lane < k) {
            const float v = slot_l[w][lane];
            float s;
            if (p.d.renormalise) {
                // softmax over the chosen logits, or over log sigmoid of them: what the sum over all experts or a tiny
                // sigmoid would divide by cancels
                float m = -INFINITY, z = 0.0f;
                for (int j = 0; j < k; ++j) {
                    const float o = softmax ? slot_l[w][j] : log_sigmoid(slot_l[w][j]);
                    m = fmaxf(m, o);
                }
                if (m == -INFINITY) m = 0.0f;
                for (int j = 0; j < k; ++j) {
                    const float o = softmax ? slot_l[w][j] : log_sigmoid(slot_l[w][j]);
                    z += slot_l[w][j] == -INFINITY ? 0.0f : expf(o - m);
                }
                s = v == -INFINITY ? 0.0f : expf((softmax ? v : log_sigmoid(v)) - m) / z;
            } else {
                s = v == -INFINITY ? 0.0f : slot_s[w][lane];
            }
            p.ids[row * k + lane] = slot_id[w][lane];
            p.weights[row * k + lane] = p.d.scale * s;
        }
        __syncthreads();
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

static unsigned route_grid(int64_t T) { return (unsigned)std::min<int64_t>((T + RW - 1) / RW, 1 << 20); }

struct RouteFwd {
    const RouteArgs &p;
    hipStream_t s;
    template <rtp_dtype DT> hipError_t operator()()
    {
        route_fwd_wave_kernel<DT><<<route_grid(p.d.T), 64 * RW, 0, s>>>(p);
        return hipGetLastError();
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
