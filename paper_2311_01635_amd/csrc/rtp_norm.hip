// Norms before and after a unit with its gate and residual (rtp_norm_fwd, rtp_norm_bwd).
#include "rtp_block_kernels.h"
#include "rtp_elem.h"
#include <algorithm>

namespace rtp {

constexpr int NT = 256;

// (a, b) summed over a group of `waves` waves that is the workgroup, or over a single wave; in every thread.  `lds` is free again
// when it returns.
template <int WAVES>
__device__ __forceinline__ float2 group_sum(float a, float b, float2 *lds)
{
    a = wave_sum(a);
    b = wave_sum(b);
    if (WAVES == 1) return make_float2(a, b);
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = make_float2(a, b);
    __syncthreads();
    float2 r = lds[0];
#pragma unroll
    for (int i = 1; i < WAVES; ++i) r = make_float2(r.x + lds[i].x, r.y + lds[i].y);
    __syncthreads();
    return r;
}

struct NormFwd {
    rtp_norm_desc d;
    rtp_norm_io io;
};

// ---- rows that are held in registers ------------------------------------------------------------------------
// Bound: HBM (a norm is 10 to 30 operations an element).  THREADS threads share a row, NV times eight elements each, which are
// read once and stay in registers over the sums; a wave alone needs no barrier.  A workgroup goes on to other rows so that the
// parameters, which would otherwise come out of L2 as often as the rows out of HBM, are fetched once, and sends for the next
// row before it adds up the present one.  4096 rows of 4096 (fp32 stream, bf16 unit): 39 us, 5.2 TB/s.  A workgroup a row: 53 us; without
// the next row on its way 46; loads past the caches 50; stores through them 43; 512, 1024, 1536 threads a compute unit instead of
// 768: 39.7, 40.9, 38.9.  Rows of 12288 and 16384: 4.9 and 5.0 TB/s.  Two rows: 4.4 us, latency.  A length just over one that fills
// its threads leaves half of them without work, and a row's last few elements go one by one: 8192 rows (bf16) of 1024 12 us, of 1032
// 25, of 1030 34; backward 30, 51, 85.

template <int THREADS> constexpr int norm_block() { return THREADS < 256 ? 256 : THREADS; }

__device__ __forceinline__ void load_params(float (&v)[8], const float *p, int64_t i, int64_t n, float missing)
{
    Eight<RTP_F32> e;
    if (p) e.load(p + i, n);
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = p ? e.get(k) : missing;
}

template <rtp_dtype SD, rtp_dtype BD, int THREADS, int NV, bool BIAS>
__global__ __launch_bounds__(norm_block<THREADS>()) void norm_fwd_kernel(NormFwd p)
{
    using S = typename Elem<SD>::t;
    using B = typename Elem<BD>::t;
    constexpr int WAVES = THREADS / 64, ROWS = norm_block<THREADS>() / THREADS;
    // 1024 threads have 128 registers each: no room for parameters and another row beside the present one
    constexpr bool KEEP = THREADS < 1024;
    __shared__ float2 lds[WAVES];
    const int tid = threadIdx.x % THREADS;
    const int64_t D = p.d.D;
    const bool layer = p.d.kind == RTP_NORM_LAYER, join = p.d.parts & RTP_NORM_JOIN, post = p.d.parts & RTP_NORM_POST, pre = p.d.parts & RTP_NORM_PRE;
    const bool elem = p.d.gate == RTP_GATE_ELEMENT;
    const float inv = 1.0f / (float)D;
    // r = res_scale x + (n a + c) g with a = out_scale gate w_post, c = out_scale gate b_post
    int64_t at[NV], left[NV];
    float a[NV][8], c[NV][8], w[NV][8], b[NV][8];
    auto post_params = [&](int j) {
        float g[8];
        load_params(a[j], p.d.w_post_dev, at[j], left[j], 1.0f);
        load_params(g, p.d.gate == RTP_GATE_CHANNEL ? (const float *)p.d.gate_dev : nullptr, at[j], left[j], 1.0f);
        if (BIAS) load_params(c[j], p.d.b_post_dev, at[j], left[j], 0.0f);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            g[k] *= p.d.out_scale;
            a[j][k] *= g[k];
            if (BIAS) c[j][k] *= g[k];
        }
    };
    auto pre_params = [&](int j) {
        load_params(w[j], p.d.w_pre_dev, at[j], left[j], 1.0f);
        if (BIAS) load_params(b[j], p.d.b_pre_dev, at[j], left[j], 0.0f);
    };
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        at[j] = (tid + j * THREADS) * 8;
        left[j] = D - at[j];
        if (KEEP) {
            post_params(j);
            pre_params(j);
        }
    }
    // mean and 1 / deviation of a row in registers
    auto moments = [&](const float (&v)[NV][8], float &mu, float &rs) {
        mu = 0.0f;
        if (layer) {
            float s = 0.0f;
#pragma unroll
            for (int j = 0; j < NV; ++j)
#pragma unroll
                for (int k = 0; k < 8; ++k) s += v[j][k];
            mu = group_sum<WAVES>(s, 0.0f, lds).x * inv;
        }
        float q = 0.0f;
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const float x = k < left[j] ? v[j][k] - mu : 0.0f;
                q += x * x;
            }
        rs = 1.0f / sqrtf(group_sum<WAVES>(q, 0.0f, lds).x * inv + p.d.eps);
    };
    const int64_t stride = (int64_t)gridDim.x * ROWS;
    int64_t row = (int64_t)blockIdx.x * ROWS + threadIdx.x / THREADS;
    Eight<SD> x[NV], next_x[NV];
    Eight<BD> y[NV], g[NV], next_y[NV], next_g[NV];
    auto fetch = [&](int64_t r) {
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            if (left[j] <= 0) continue;
            next_x[j].load((const S *)p.io.x_dev + r * p.io.ld_x + at[j], left[j]);
            if (join) next_y[j].load((const B *)p.io.y_dev + r * p.io.ld_y + at[j], left[j]);
            if (elem) next_g[j].load((const B *)p.d.gate_dev + r * p.d.ld_gate + at[j], left[j]);
        }
    };
    if (row < p.d.T) fetch(row);
    for (; row < p.d.T; row += stride) {
#pragma unroll
        for (int j = 0; j < NV; ++j) { x[j] = next_x[j]; y[j] = next_y[j]; g[j] = next_g[j]; }
        if (KEEP && row + stride < p.d.T) fetch(row + stride); // under this row's sums
        float v[NV][8];
        float mu = 0.0f, rs = 1.0f;
        if (join) {
#pragma unroll
            for (int j = 0; j < NV; ++j)
#pragma unroll
                for (int k = 0; k < 8; ++k) v[j][k] = left[j] > 0 ? y[j].get(k) : 0.0f;
            if (post) {
                moments(v, mu, rs);
                if (tid == 0) { p.io.stats_dev[row * 4] = mu; p.io.stats_dev[row * 4 + 1] = rs; }
            }
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                if (left[j] <= 0) continue;
                if (!KEEP) post_params(j);
                float o[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    o[k] = (v[j][k] - mu) * rs * a[j][k];
                    if (BIAS) o[k] += c[j][k];
                    if (elem) o[k] *= g[j].get(k);
                    o[k] = p.d.res_scale * x[j].get(k) + o[k];
                }
                x[j].set(o);
                x[j].store((S *)p.io.r_dev + row * p.io.ld_r + at[j], left[j]);
            }
        }
        if (pre) { // (of the stream as it is stored)
#pragma unroll
            for (int j = 0; j < NV; ++j)
#pragma unroll
                for (int k = 0; k < 8; ++k) v[j][k] = k < left[j] ? x[j].get(k) : 0.0f;
            moments(v, mu, rs);
            if (tid == 0) { p.io.stats_dev[row * 4 + 2] = mu; p.io.stats_dev[row * 4 + 3] = rs; }
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                if (left[j] <= 0) continue;
                if (!KEEP) pre_params(j);
                float o[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    o[k] = (v[j][k] - mu) * rs * w[j][k];
                    if (BIAS) o[k] += b[j][k];
                }
                Eight<BD> h;
                h.set(o);
                h.store((B *)p.io.h_dev + row * p.io.ld_h + at[j], left[j]);
            }
        }
        if (!KEEP && row + stride < p.d.T) fetch(row + stride);
    }
}

// ---- rows of any length -------------------------------------------------------------------------------------
// One workgroup a row, the row read once for each sum over it (rows of more than NORM_REG_D; 20000: 0.9 to 1.1 TB/s).
template <rtp_dtype SD, rtp_dtype BD>
__global__ __launch_bounds__(NT) void norm_fwd_row_kernel(NormFwd p)
{
    using S = typename Elem<SD>::t;
    using B = typename Elem<BD>::t;
    __shared__ float2 lds[NT / 64];
    const int64_t D = p.d.D;
    const bool layer = p.d.kind == RTP_NORM_LAYER, join = p.d.parts & RTP_NORM_JOIN, post = p.d.parts & RTP_NORM_POST;
    const float inv = 1.0f / (float)D;
    for (int64_t row = blockIdx.x; row < p.d.T; row += gridDim.x) {
        const S *x = (const S *)p.io.x_dev + row * p.io.ld_x;
        const B *y = (const B *)p.io.y_dev + row * p.io.ld_y;
        const S *v = x; // what the second norm is of
        float mu = 0.0f, rs = 1.0f;
        if (post) {
            if (layer) {
                float a = 0.0f;
                for (int64_t i = threadIdx.x; i < D; i += NT) a += (float)y[i];
                mu = group_sum<NT / 64>(a, 0.0f, lds).x * inv;
            }
            float q = 0.0f;
            for (int64_t i = threadIdx.x; i < D; i += NT) { const float c = (float)y[i] - mu; q += c * c; }
            rs = 1.0f / sqrtf(group_sum<NT / 64>(q, 0.0f, lds).x * inv + p.d.eps);
            if (threadIdx.x == 0) { p.io.stats_dev[row * 4] = mu; p.io.stats_dev[row * 4 + 1] = rs; }
        }
        if (join) {
            S *r = (S *)p.io.r_dev + row * p.io.ld_r;
            for (int64_t i = threadIdx.x; i < D; i += NT) {
                float o = (float)y[i];
                if (post) {
                    o = (o - mu) * rs;
                    if (p.d.w_post_dev) o *= p.d.w_post_dev[i];
                    if (p.d.b_post_dev) o += p.d.b_post_dev[i];
                }
                if (p.d.gate == RTP_GATE_CHANNEL) o *= ((const float *)p.d.gate_dev)[i];
                if (p.d.gate == RTP_GATE_ELEMENT) o *= (float)((const B *)p.d.gate_dev)[row * p.d.ld_gate + i];
                r[i] = (S)(p.d.res_scale * (float)x[i] + p.d.out_scale * o);
            }
            v = r; // (every thread reads back what it wrote itself)
        }
        if (p.d.parts & RTP_NORM_PRE) {
            B *h = (B *)p.io.h_dev + row * p.io.ld_h;
            mu = 0.0f;
            if (layer) {
                float a = 0.0f;
                for (int64_t i = threadIdx.x; i < D; i += NT) a += (float)v[i];
                mu = group_sum<NT / 64>(a, 0.0f, lds).x * inv;
            }
            float q = 0.0f;
            for (int64_t i = threadIdx.x; i < D; i += NT) { const float c = (float)v[i] - mu; q += c * c; }
            rs = 1.0f / sqrtf(group_sum<NT / 64>(q, 0.0f, lds).x * inv + p.d.eps);
            if (threadIdx.x == 0) { p.io.stats_dev[row * 4 + 2] = mu; p.io.stats_dev[row * 4 + 3] = rs; }
            for (int64_t i = threadIdx.x; i < D; i += NT) {
                float o = ((float)v[i] - mu) * rs;
                if (p.d.w_pre_dev) o *= p.d.w_pre_dev[i];
                if (p.d.b_pre_dev) o += p.d.b_pre_dev[i];
                h[i] = (B)o;
            }
        }
    }
}

struct NormBwd {
    rtp_norm_desc d;
    rtp_norm_grads g;
    unsigned sums;
    int nsums;
};

// Rows in registers.  Bound: HBM.  8192 rows of 8192 (bf16): 150 us, 8 of them the sums, 5.4 TB/s; without the next row on its way 190.  1990
// rows of 768 with every part: 14 and 5 us, latency (two rows a wave, one after the other).  Rows of more than 8192 do not
// fit 128 registers a thread and spill: 1.2 to 1.9 TB/s.  Of 4097 to 8192 an fp32 stream spills a little with fp32 units (8192 rows of
// 8192 3.8 TB/s, with biases 4.5) and with bf16 units and biases (4.4; without, 5.1).  The sums over rows stay in registers too, a thread's columns over all rows of its workgroup, so
// that they cost one write a workgroup (and one read by norm_sums_kernel, which adds the workgroups up in a fixed order).
// With k = out_scale gate w_post and q = dR k g (g: an element gate): dy = rs (q - mean q - n mean(q n)).
template <rtp_dtype SD, rtp_dtype BD, int THREADS, int NV, bool BIAS>
__global__ __launch_bounds__(norm_block<THREADS>()) void norm_bwd_kernel(NormBwd p)
{
    using S = typename Elem<SD>::t;
    using B = typename Elem<BD>::t;
    constexpr int WAVES = THREADS / 64, ROWS = norm_block<THREADS>() / THREADS;
    // the next row is fetched under the present one's sums where 256 registers hold both (nearly: see above for fp32 on both sides)
    constexpr bool AHEAD = THREADS < 512 || (THREADS == 512 && !BIAS);
    __shared__ float2 lds[WAVES];
    const int tid = threadIdx.x % THREADS;
    const int64_t D = p.d.D;
    const bool layer = p.d.kind == RTP_NORM_LAYER, join = p.d.parts & RTP_NORM_JOIN, post = p.d.parts & RTP_NORM_POST, pre = p.d.parts & RTP_NORM_PRE;
    const bool elem = p.d.gate == RTP_GATE_ELEMENT, has_y = post || p.d.gate != RTP_GATE_NONE;
    const float inv = 1.0f / (float)D, out_scale = join ? p.d.out_scale : 0.0f, res_scale = join ? p.d.res_scale : 1.0f;
    const int64_t stride = (int64_t)gridDim.x * ROWS;
    int64_t row = (int64_t)blockIdx.x * ROWS + threadIdx.x / THREADS;
    int64_t at[NV], left[NV];
    Eight<SD> next_r[NV], next_dr[NV];
    Eight<BD> next_y[NV], next_dh[NV], next_g[NV];
    float4 next_st = {0.0f, 1.0f, 0.0f, 1.0f};
    auto fetch = [&](int64_t i) {
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            if (left[j] <= 0) continue;
            if (pre) {
                next_r[j].template load<true>((const S *)p.g.r_dev + i * p.g.ld_r + at[j], left[j]);
                next_dh[j].template load<true>((const B *)p.g.dh_dev + i * p.g.ld_dh + at[j], left[j]);
            }
            if (p.g.dr_dev) next_dr[j].template load<true>((const S *)p.g.dr_dev + i * p.g.ld_dr + at[j], left[j]);
            if (has_y) next_y[j].template load<true>((const B *)p.g.y_dev + i * p.g.ld_y + at[j], left[j]);
            if (elem) next_g[j].template load<true>((const B *)p.d.gate_dev + i * p.d.ld_gate + at[j], left[j]);
        }
        if (post) { next_st.x = p.g.stats_dev[i * 4]; next_st.y = p.g.stats_dev[i * 4 + 1]; }
        if (pre) { next_st.z = p.g.stats_dev[i * 4 + 2]; next_st.w = p.g.stats_dev[i * 4 + 3]; }
    };
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        at[j] = (tid + j * THREADS) * 8;
        left[j] = D - at[j];
    }
    if (AHEAD && row < p.d.T) fetch(row);
    float w[NV][8], k2[NV][8];
    float s1[NV][8], s2[NV][8], q1[NV][8], q2[NV][8]; // sums over rows: dh n, f n, dh, f, with f = out_scale dR (times an element gate)
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        float g[8];
        load_params(w[j], p.d.w_pre_dev, at[j], left[j], 1.0f);
        load_params(k2[j], p.d.w_post_dev, at[j], left[j], 1.0f);
        load_params(g, p.d.gate == RTP_GATE_CHANNEL ? (const float *)p.d.gate_dev : nullptr, at[j], left[j], 1.0f);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            k2[j][k] *= out_scale * g[k];
            s1[j][k] = s2[j][k] = q1[j][k] = q2[j][k] = 0.0f;
        }
    }
    for (; row < p.d.T; row += stride) {
        if (!AHEAD) fetch(row);
        Eight<SD> r[NV], dr[NV];
        Eight<BD> y[NV], dh[NV], g[NV];
#pragma unroll
        for (int j = 0; j < NV; ++j) { r[j] = next_r[j]; dr[j] = next_dr[j]; y[j] = next_y[j]; dh[j] = next_dh[j]; g[j] = next_g[j]; }
        const float4 st = next_st;
        if (AHEAD && row + stride < p.d.T) fetch(row + stride);
        float v[NV][8]; // dR
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int k = 0; k < 8; ++k) v[j][k] = left[j] > 0 && p.g.dr_dev ? dr[j].get(k) : 0.0f;
        if (pre) {
            float a = 0.0f, b = 0.0f;
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                if (left[j] <= 0) continue;
#pragma unroll
                for (int k = 0; k < 8; ++k) { // (behind the row's end dh is zero)
                    const float d = dh[j].get(k), n = (r[j].get(k) - st.z) * st.w, dn = d * w[j][k];
                    a += dn;
                    b += dn * n;
                    s1[j][k] += d * n;
                    if (BIAS) q1[j][k] += d;
                }
            }
            float2 m = group_sum<WAVES>(a, b, lds);
            m = {layer ? m.x * inv : 0.0f, m.y * inv};
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                if (left[j] <= 0) continue;
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const float n = (r[j].get(k) - st.z) * st.w;
                    v[j][k] += st.w * (dh[j].get(k) * w[j][k] - m.x - n * m.y);
                }
            }
        }
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            if (left[j] <= 0) continue;
            float o[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) o[k] = res_scale * v[j][k];
            Eight<SD> dx;
            dx.set(o);
            dx.store((S *)p.g.dx_dev + row * p.g.ld_dx + at[j], left[j]);
        }
        if (!join) continue;
        if (elem && p.g.dgate_dev) {
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                if (left[j] <= 0) continue;
                float o[8], c[8];
                load_params(c, p.d.b_post_dev, at[j], left[j], 0.0f);
#pragma unroll
                for (int k = 0; k < 8; ++k) o[k] = v[j][k] * ((y[j].get(k) - st.x) * st.y * k2[j][k] + out_scale * c[k]);
                Eight<BD> dg;
                dg.set(o);
                dg.store((B *)p.g.dgate_dev + row * p.g.ld_dgate + at[j], left[j]);
            }
        }
        float a = 0.0f, b = 0.0f;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            if (left[j] <= 0) continue;
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                if (elem) v[j][k] *= g[j].get(k); // (behind the row's end the gate is zero, but dR need not be)
                else if (k >= left[j]) v[j][k] = 0.0f;
                const float n = has_y ? (y[j].get(k) - st.x) * st.y : 0.0f, f = out_scale * v[j][k], q = v[j][k] * k2[j][k];
                s2[j][k] += f * n;
                if (BIAS) q2[j][k] += f;
                a += q;
                b += q * n;
            }
        }
        float2 m = {0.0f, 0.0f};
        if (post) {
            m = group_sum<WAVES>(a, b, lds);
            m = {layer ? m.x * inv : 0.0f, m.y * inv};
        }
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            if (left[j] <= 0) continue;
            float o[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const float n = has_y ? (y[j].get(k) - st.x) * st.y : 0.0f;
                o[k] = st.y * (v[j][k] * k2[j][k] - m.x - n * m.y);
            }
            Eight<BD> dy;
            dy.set(o);
            dy.store((B *)p.g.dy_dev + row * p.g.ld_dy + at[j], left[j]);
        }
    }
    float *ws = (float *)p.g.ws_dev + (int64_t)blockIdx.x * p.nsums * D;
    auto put = [&](const float (&v)[NV][8]) {
        if (ROWS > 1) { // the workgroup's rows are apart by whole waves: joined in LDS
            __shared__ float part[ROWS > 1 ? ROWS * THREADS * NV * 8 : 1];
            __syncthreads();
#pragma unroll
            for (int j = 0; j < NV; ++j)
#pragma unroll
                for (int k = 0; k < 8; ++k) part[((threadIdx.x / THREADS) * NV * 8 + j * 8 + k) * THREADS + tid] = v[j][k];
            __syncthreads();
            for (int i = threadIdx.x; i < NV * 8 * THREADS; i += ROWS * THREADS) {
                const int t = i % THREADS, k = i / THREADS % 8, j = i / THREADS / 8; // thread t's column at 8 (t + j THREADS) + k
                const int64_t col = (int64_t)(t + j * THREADS) * 8 + k;
                float x = 0.0f;
#pragma unroll
                for (int q = 0; q < ROWS; ++q) x += part[(q * NV * 8 + j * 8 + k) * THREADS + t];
                if (col < D) ws[col] = x;
            }
        } else {
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                if (left[j] <= 0) continue;
                Eight<RTP_F32> e;
                e.set(v[j]);
                e.store(ws + at[j], left[j]);
            }
        }
        ws += D;
    };
    if (p.sums & SUM_PRE_W) put(s1);
    if (BIAS && p.sums & SUM_PRE_B) put(q1);
    if (p.sums & SUM_POST_W) put(s2);
    if (BIAS && p.sums & SUM_POST_B) put(q2);
}

// Rows of any length: a workgroup takes every gridDim.x-th row and keeps its column sums in its own part of the workspace, where each
// column is one thread's (20000: 0.4 to 0.55 TB/s).
template <rtp_dtype SD, rtp_dtype BD>
__global__ __launch_bounds__(NT) void norm_bwd_row_kernel(NormBwd p)
{
    using S = typename Elem<SD>::t;
    using B = typename Elem<BD>::t;
    __shared__ float2 lds[NT / 64];
    const int64_t D = p.d.D;
    const bool layer = p.d.kind == RTP_NORM_LAYER, join = p.d.parts & RTP_NORM_JOIN, post = p.d.parts & RTP_NORM_POST, pre = p.d.parts & RTP_NORM_PRE;
    const float inv = 1.0f / (float)D;
    float *ws = (float *)p.g.ws_dev + (int64_t)blockIdx.x * p.nsums * D;
    for (int64_t i = threadIdx.x; i < p.nsums * D; i += NT) ws[i] = 0.0f;
    __syncthreads();
    for (int64_t row = blockIdx.x; row < p.d.T; row += gridDim.x) {
        const S *r = (const S *)p.g.r_dev + row * p.g.ld_r, *dr = p.g.dr_dev ? (const S *)p.g.dr_dev + row * p.g.ld_dr : nullptr;
        const B *y = (const B *)p.g.y_dev + row * p.g.ld_y, *dh = (const B *)p.g.dh_dev + row * p.g.ld_dh;
        const B *gate = (const B *)p.d.gate_dev + row * p.d.ld_gate;
        S *dx = (S *)p.g.dx_dev + row * p.g.ld_dx;
        B *dy = (B *)p.g.dy_dev + row * p.g.ld_dy;
        float4 st = {0.0f, 1.0f, 0.0f, 1.0f};
        if (post) { st.x = p.g.stats_dev[row * 4]; st.y = p.g.stats_dev[row * 4 + 1]; }
        if (pre) { st.z = p.g.stats_dev[row * 4 + 2]; st.w = p.g.stats_dev[row * 4 + 3]; }
        float2 m1 = {0.0f, 0.0f}, m2 = {0.0f, 0.0f};
        if (pre) {
            float a = 0.0f, b = 0.0f;
            for (int64_t i = threadIdx.x; i < D; i += NT) {
                const float dn = (float)dh[i] * (p.d.w_pre_dev ? p.d.w_pre_dev[i] : 1.0f);
                a += dn;
                b += dn * ((float)r[i] - st.z) * st.w;
            }
            m1 = group_sum<NT / 64>(a, b, lds);
            m1 = {layer ? m1.x * inv : 0.0f, m1.y * inv};
        }
        // gradient of the stream's row at i
        auto stream = [&](int64_t i) {
            float v = dr ? (float)dr[i] : 0.0f;
            if (pre) {
                const float dn = (float)dh[i] * (p.d.w_pre_dev ? p.d.w_pre_dev[i] : 1.0f);
                v += st.w * (dn - m1.x - ((float)r[i] - st.z) * st.w * m1.y);
            }
            return v;
        };
        // ... of gate . N(y), with the gate's factor
        auto branch = [&](int64_t i, float v) {
            v *= p.d.out_scale;
            if (p.d.gate == RTP_GATE_CHANNEL) v *= ((const float *)p.d.gate_dev)[i];
            if (p.d.gate == RTP_GATE_ELEMENT) v *= (float)gate[i];
            return v;
        };
        if (post) {
            float a = 0.0f, b = 0.0f;
            for (int64_t i = threadIdx.x; i < D; i += NT) {
                const float dn = branch(i, stream(i)) * (p.d.w_post_dev ? p.d.w_post_dev[i] : 1.0f);
                a += dn;
                b += dn * ((float)y[i] - st.x) * st.y;
            }
            m2 = group_sum<NT / 64>(a, b, lds);
            m2 = {layer ? m2.x * inv : 0.0f, m2.y * inv};
        }
        for (int64_t i = threadIdx.x; i < D; i += NT) {
            const float v = stream(i);
            float *w = ws + i;
            if (p.sums & SUM_PRE_W) { *w += (float)dh[i] * ((float)r[i] - st.z) * st.w; w += D; }
            if (p.sums & SUM_PRE_B) { *w += (float)dh[i]; w += D; }
            dx[i] = (S)((join ? p.d.res_scale : 1.0f) * v);   // (dx may be dr: its last reader has read it)
            if (!join) continue;
            const bool has_y = post || p.d.gate != RTP_GATE_NONE;
            const float n = has_y ? ((float)y[i] - st.x) * st.y : 0.0f, wp = post && p.d.w_post_dev ? p.d.w_post_dev[i] : 1.0f;
            const float e = branch(i, v), f = p.d.gate == RTP_GATE_CHANNEL ? p.d.out_scale * v : e;
            if (p.sums & SUM_POST_W) { *w += f * n; w += D; }
            if (p.sums & SUM_POST_B) *w += f;
            if (p.d.gate == RTP_GATE_ELEMENT && p.g.dgate_dev)
                ((B *)p.g.dgate_dev)[row * p.g.ld_dgate + i] =
                    (B)(p.d.out_scale * v * (n * wp + (post && p.d.b_post_dev ? p.d.b_post_dev[i] : 0.0f)));
            dy[i] = (B)(post ? st.y * (e * wp - m2.x - n * m2.y) : e);
        }
    }
}

struct NormSums {
    const float *ws;
    int parts, nsums;
    unsigned sums;
    int64_t D;
    float *dw_pre, *db_pre, *dw_post, *db_post, *dgate;
    const float *gate, *w_post, *b_post; // of a channel gate
    int accumulate;
};

// The parts' column sums, and the gradients that follow from them: with a channel gate the sums over rows leave it out, S = sum of
// b dR n and Q = sum of b dR, so that dw = gate S, db = gate Q, dgate = w S + b Q.  Bound: latency (a few MB out of the caches).  16
// columns a workgroup, 64 threads to each of them, so that a thread has few loads and all of them in flight; the
// order of the additions is fixed.
constexpr int SUM_COLS = 16, SUM_THREADS = 1024, SUM_GROUPS = SUM_THREADS / SUM_COLS;
__global__ __launch_bounds__(SUM_THREADS) void norm_sums_kernel(NormSums p)
{
    __shared__ float lds[4][SUM_THREADS / 64][SUM_COLS];
    const int col = threadIdx.x % SUM_COLS, group = threadIdx.x / SUM_COLS;
    const int64_t i = (int64_t)blockIdx.x * SUM_COLS + col;
    int at = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        if (!(p.sums >> k & 1)) continue;
        float v = 0.0f;
        if (i < p.D) {
#pragma unroll 4
            for (int b = group; b < p.parts; b += SUM_GROUPS) v += p.ws[((int64_t)b * p.nsums + at) * p.D + i];
        }
        ++at;
#pragma unroll
        for (int o = SUM_COLS; o < 64; o *= 2) v += __shfl_xor(v, o);
        if (threadIdx.x % 64 < SUM_COLS) lds[k][threadIdx.x / 64][col] = v;
    }
    __syncthreads();
    if (threadIdx.x >= SUM_COLS || i >= p.D) return;
    float v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int k = 0; k < 4; ++k)
        if (p.sums >> k & 1)
            for (int w = 0; w < SUM_THREADS / 64; ++w) v[k] += lds[k][w][col];
    auto put = [&](float *to, float x) {
        if (to) to[i] = p.accumulate ? to[i] + x : x;
    };
    put(p.dw_pre, v[0]);
    put(p.db_pre, v[1]);
    const float gate = p.gate ? p.gate[i] : 1.0f;
    put(p.dw_post, gate * v[2]);
    put(p.db_post, gate * v[3]);
    put(p.dgate, (p.w_post ? p.w_post[i] : 1.0f) * v[2] + (p.b_post ? p.b_post[i] * v[3] : 0.0f));
}

template <class F>
static hipError_t by_types(const rtp_norm_desc &d, F f)
{
    if (d.stream_dtype == RTP_F32) {
        if (d.dtype == RTP_F32) return f.template operator()<RTP_F32, RTP_F32>();
        if (d.dtype == RTP_BF16) return f.template operator()<RTP_F32, RTP_BF16>();
        return f.template operator()<RTP_F32, RTP_F16>();
    }
    if (d.dtype == RTP_BF16) return f.template operator()<RTP_BF16, RTP_BF16>();
    return f.template operator()<RTP_F16, RTP_F16>();
}

// Threads that share a row held in registers, and the eights a thread has of it.
template <class F>
static hipError_t by_length(int64_t D, F &&f)
{
    if (D <= 512) return f.template operator()<64, 1>();
    if (D <= 1024) return f.template operator()<64, 2>();
    if (D <= 2048) return f.template operator()<256, 1>();
    if (D <= 4096) return f.template operator()<256, 2>();
    if (D <= 8192) return f.template operator()<512, 2>();
    return f.template operator()<1024, 2>();
}
constexpr int64_t NORM_REG_D = 16384;

template <rtp_dtype SD, rtp_dtype BD> struct RunFwdRegs {
    const NormFwd &p;
    hipStream_t s;
    template <int THREADS, int NV> hipError_t operator()()
    {
        constexpr int BLOCK = norm_block<THREADS>(), ROWS = BLOCK / THREADS;
        const unsigned grid = (unsigned)std::min<int64_t>((p.d.T + ROWS - 1) / ROWS, std::max(256, 256 * 768 / BLOCK));
        if (p.d.b_post_dev || p.d.b_pre_dev) norm_fwd_kernel<SD, BD, THREADS, NV, true><<<grid, BLOCK, 0, s>>>(p);
        else norm_fwd_kernel<SD, BD, THREADS, NV, false><<<grid, BLOCK, 0, s>>>(p);
        return hipGetLastError();
    }
};

struct RunFwd {
    const NormFwd &p;
    hipStream_t s;
    template <rtp_dtype SD, rtp_dtype BD> hipError_t operator()()
    {
        if (p.d.D <= NORM_REG_D) return by_length(p.d.D, RunFwdRegs<SD, BD>{p, s});
        norm_fwd_row_kernel<SD, BD><<<(unsigned)std::min<int64_t>(p.d.T, 1 << 20), NT, 0, s>>>(p);
        return hipGetLastError();
    }
};

hipError_t launch_norm_fwd(const rtp_norm_desc &d, const rtp_norm_io &io, hipStream_t s)
{
    const NormFwd p{d, io};
    return by_types(d, RunFwd{p, s});
}

// Workgroups of the backward pass, each of which leaves its sums: one to a compute unit; two where they have eight turns and more
// and there is room for two (256 threads, a 16-bit stream).  Two for all: 1990 rows of 768 24.8 us instead of 20.4, 8192 of 4096 with an fp32
// stream 150 instead of 137; one for all: 8192 rows of 2048 80 us instead of 55, of 4096 101 instead of 84.
struct Parts {
    int64_t T;
    bool half; // a 16-bit stream
    template <int THREADS, int NV> hipError_t operator()()
    {
        constexpr int BLOCK = norm_block<THREADS>(), ROWS = BLOCK / THREADS;
        const int64_t turns = (T + ROWS - 1) / ROWS;
        T = std::min<int64_t>(turns, BLOCK == 256 && half && turns >= 4096 ? 512 : 256);
        return hipSuccess;
    }
};
int norm_bwd_parts(const rtp_norm_desc &d)
{
    if (d.D > NORM_REG_D) return (int)std::min<int64_t>(d.T, 512);
    Parts parts{d.T, d.stream_dtype != RTP_F32};
    (void)by_length(d.D, parts);
    return (int)parts.T;
}

template <rtp_dtype SD, rtp_dtype BD> struct RunBwdRegs {
    const NormBwd &p;
    hipStream_t s;
    template <int THREADS, int NV> hipError_t operator()()
    {
        constexpr int BLOCK = norm_block<THREADS>();
        const unsigned grid = (unsigned)norm_bwd_parts(p.d);
        if (p.sums & (SUM_PRE_B | SUM_POST_B)) norm_bwd_kernel<SD, BD, THREADS, NV, true><<<grid, BLOCK, 0, s>>>(p);
        else norm_bwd_kernel<SD, BD, THREADS, NV, false><<<grid, BLOCK, 0, s>>>(p);
        return hipGetLastError();
    }
};

struct RunBwd {
    const NormBwd &p;
    hipStream_t s;
    template <rtp_dtype SD, rtp_dtype BD> hipError_t operator()()
    {
        if (p.d.D <= NORM_REG_D) return by_length(p.d.D, RunBwdRegs<SD, BD>{p, s});
        norm_bwd_row_kernel<SD, BD><<<norm_bwd_parts(p.d), NT, 0, s>>>(p);
        return hipGetLastError();
    }
};

hipError_t launch_norm_bwd(const rtp_norm_desc &d, const rtp_norm_grads &g, unsigned sums, hipStream_t s)
{
    const NormBwd p{d, g, sums, __builtin_popcount(sums)};
    if (d.T > 0) {
        const hipError_t e = by_types(d, RunBwd{p, s});
        if (e != hipSuccess) return e;
    }
    if (!sums) return hipSuccess;
    NormSums q{};
    q.ws = (const float *)g.ws_dev;
    q.parts = norm_bwd_parts(d);
    q.nsums = p.nsums;
    q.sums = sums;
    q.D = d.D;
    q.dw_pre = g.dw_pre_dev;
    q.db_pre = g.db_pre_dev;
    q.dw_post = g.dw_post_dev;
    q.db_post = g.db_post_dev;
    if (d.gate == RTP_GATE_CHANNEL) {
        q.dgate = (float *)g.dgate_dev;
        q.gate = (const float *)d.gate_dev;
    }
    q.w_post = d.parts & RTP_NORM_POST ? d.w_post_dev : nullptr;
    q.b_post = d.parts & RTP_NORM_POST ? d.b_post_dev : nullptr;
    q.accumulate = g.accumulate;
    norm_sums_kernel<<<(unsigned)((d.D + SUM_COLS - 1) / SUM_COLS), SUM_THREADS, 0, s>>>(q);
    return hipGetLastError();
}

} // namespace rtp
