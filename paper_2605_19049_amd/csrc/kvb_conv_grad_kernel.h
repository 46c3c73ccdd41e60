// kvb_conv_backward.  With E, z, y and r = 1 / sqrt(sum y^2 + eps) as in kvb_conv (worked out once more) and s = 1 / (1 + exp(-z)),
//     dy = r (dn - r^2 y (y.dn)) for q and k, dn for v          dz = dy (s + y (1 - s))
//     dE_e = sum_i w_i dz_{e-i}                                 dw_i = sum_t dz_t E_{t+i},  dbias = sum_t dz_t
//     da = -exp(A_log) dg / (1 + exp(-(a + dt_bias))),  db = dbeta beta (1 - beta),  dA_log = sum dg g,  ddt_bias = sum da
// A wave walks forward over its tokens of 512 channels (fp32: 256) and W - 1 more (whose dz its last inputs need), the last W inputs and dz in registers.
// E's rows ahead of the first input are the state's: their gradient is dstate0; the last W - 1 rows get dstate1 as well.  Sums over tokens stay
// in registers, then the four waves of a workgroup add theirs in LDS and leave one part; kvb_sums_kernel adds the parts in order, so
// the same inputs give the same bits.
// Bounded by memory: 4 x 2048 tokens, 16 + 32 heads of 128, bf16, 408 MB (a copy: 80 us) take 97 us, 5 of them the sums and some 6 the launch and what stands ahead of a wave's first
// token.  The vector units are busy 64 of them (counters: 32.6 M instructions; without norms the call takes 96), with two waves a SIMD (200 registers, with a bias 216), so what counts is that all
// of those have as much to do: stretches as long as fill the card once (three rounds of shorter ones took 136), and the groups of q and k on one compute
// unit with those of v (group by group in the launch: 97, stretch by stretch: 106).  Calls of some hundred tokens: the chain of launch, start, slot, inputs, then half a
// microsecond a token.
#ifndef KVB_CONV_GRAD_KERNEL_H
#define KVB_CONV_GRAD_KERNEL_H

#include "kvb_layer_device.h"

namespace kvb_impl {

// Gradients of the gates of some tokens; the sums over them in the lanes of the first token
template <typename T>
__device__ __forceinline__ void gate_grads(const ConvGradArgs &g, int64_t t0, int n, int h, const GateLanes &l, float &dA, float &ddt)
{
    const ConvArgs &a = g.f;
    const float rate = -expf(a.A_log[h]), shift = a.dt_bias[h];
#pragma unroll 2
    for (int t = l.token; t < n; t += l.tokens) {
        const int64_t at = t0 + t;
        const float y = to_f32(static_cast<const T *>(a.a)[at * a.a_stride + h]) + shift, b = to_f32(static_cast<const T *>(a.b)[at * a.b_stride + h]);
        const float dg = g.dg[at * a.Hv + h], dbeta = g.dbeta[at * a.Hv + h];
        const float s = 1.0f / (1.0f + expf(-y)), beta = 1.0f / (1.0f + expf(-b)), other = 1.0f / (1.0f + expf(b));
        const float da = dg * rate * s;
        static_cast<T *>(g.da)[at * a.a_stride + h] = from_f32<T>(da);
        static_cast<T *>(g.db)[at * a.b_stride + h] = from_f32<T>(dbeta * beta * other);
        dA = fmaf(dg, rate * softplus(y), dA);
        ddt += da;
    }
}

template <typename T, int W, bool BIAS>
__global__ __launch_bounds__(256) void kvb_conv_grad_kernel(const ConvGradArgs g, int64_t length)
{
    constexpr int AHEAD = 2;   // tokens asked for ahead (4: 98.5 us instead of 97.0, for the registers)
    constexpr int V = GRAD_CHANNELS<T>, PLANE = 64 * V;
    __shared__ float sums[4][(W + BIAS) * PLANE];
    const ConvArgs &a = g.f;
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), groups = grad_groups(a.C, V);
    const int group = blockIdx.x / g.parts, part = blockIdx.x - group * g.parts;
    float *to = g.part + (int64_t)part * g.columns;
    const int64_t from = (part * 4 + wave) * length, behind = from + length;   // the wave's places

    if (group == groups) {
        const GateLanes l = gate_lanes(a.Hv, lane);
        for (int h0 = 0; h0 < a.Hv; h0 += l.heads) {
            const int h = h0 + l.head;
            float dA = 0.0f, ddt = 0.0f;
            for (Shares shares(a, from, behind, W - 1); shares.more();) {
                const Share p = shares.take();
                if (p.some && p.t0 < p.t1 && h < a.Hv)
                    gate_grads<T>(g, (int64_t)p.first + p.t0, p.t1 - p.t0, h, l, dA, ddt);
            }
            sums[wave][lane] = dA;
            sums[wave][64 + lane] = ddt;
            __syncthreads();
            if (threadIdx.x < 2 * l.heads) {
                const int which = threadIdx.x / l.heads, head = threadIdx.x % l.heads;
                float s = 0.0f;
                for (int v = 0; v < 4; ++v)
                    for (int t = 0; t < l.tokens; ++t)
                        s += sums[v][64 * which + t * l.heads + head];
                if (h0 + head < a.Hv)
                    to[(int64_t)(W + BIAS) * a.C + which * a.Hv + h0 + head] = s;
            }
            __syncthreads();
        }
        return;
    }

    const int own_ch = group * PLANE + lane * V;
    const bool active = own_ch < a.C;
    const int ch = active ? own_ch : 0, nq = a.Hk * a.d, lgh = (a.d == 128 ? 4 : a.d == 64 ? 3 : 2) + (V == 4);
    float w[W][V], bias[V] = {}, dw[W][V] = {}, dbias[V] = {};
    {
        const T *wp = static_cast<const T *>(a.weight) + (int64_t)ch * W;
#pragma unroll
        for (int i = 0; i < W; ++i) {
            float y[V];
            unpack(load_raw<V>(wp + V * i), y);
#pragma unroll
            for (int j = 0; j < V; ++j)
                w[(V * i + j) % W][(V * i + j) / W] = y[j];
        }
        if constexpr (BIAS)
            unpack(load_raw<V>(static_cast<const T *>(a.bias) + ch), bias);
    }
    const bool unit = a.unit && ch < 2 * nq, any_unit = a.unit && group * PLANE < 2 * nq;   // of the lane; of some lane of the wave
    const T *dn_first = ch < nq ? static_cast<const T *>(g.dq) + ch : ch < 2 * nq ? static_cast<const T *>(g.dk) + (ch - nq) : static_cast<const T *>(g.dv) + (ch - 2 * nq);
    const int64_t dn_stride = ch < nq ? a.q_stride : ch < 2 * nq ? a.k_stride : a.v_stride;

    for (Shares shares(a, from, behind, W - 1); shares.more();) {
        const Share p = shares.take();
        if (!p.some || !active)
            continue;
        const T *x = static_cast<const T *>(a.x) + (int64_t)p.first * a.x_stride + ch, *dn = dn_first + (int64_t)p.first * dn_stride;
        T *dx = static_cast<T *>(g.dx) + (int64_t)p.first * a.x_stride + ch;
        const int64_t state_at = (int64_t)p.row * (W - 1) * a.C + ch;
        const T *s0 = a.state0 ? static_cast<const T *>(a.state0) + state_at : nullptr, *ds1 = g.dstate1 ? static_cast<const T *>(g.dstate1) + state_at : nullptr;
        T *ds0 = g.dstate0 ? static_cast<T *>(g.dstate0) + state_at : nullptr;
        const int end = p.t1 + W - 1, known = min(end, p.len);   // dz behind the sequence's end is zero
        float e[4][V], dz[4][V] = {};   // row t + W - 1 of E, and dz_t, at t % 4
#pragma unroll
        for (int i = 0; i < W - 1; ++i) {
            const int at = p.t0 + i;   // of E: token at - (W - 1)
            decltype(load_raw<V>(x)) r{};
            if (at >= W - 1)
                r = load_raw<V>(x + (int64_t)(at - (W - 1)) * a.x_stride);
            else if (s0)
                r = load_raw<V>(s0 + (int64_t)at * a.C);
            unpack(r, e[(i + 4 - (W - 1)) % 4]);
        }
        decltype(load_raw<V>(x)) rx[AHEAD], rn[AHEAD];
        if (known > 0)
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) {
                const int64_t t = min(p.t0 + u, known - 1);
                rx[u] = load_raw<V>(x + t * a.x_stride);
                rn[u] = load_raw<V>(dn + t * dn_stride);
            }
        for (int t4 = p.t0; t4 < end; t4 += 4)
            static_for<4>([&](auto U) {
                constexpr int u = U();
                const int t = t4 + u;
                if (t >= end)
                    return;
                if (t < known) {
                    float d[V], z[V], s[V], sq = 0.0f, dot = 0.0f;
                    unpack(rx[u % AHEAD], e[u]);
                    unpack(rn[u % AHEAD], d);
                    {
                        const int64_t next = min(t + AHEAD, known - 1);
                        rx[u % AHEAD] = load_raw<V>(x + next * a.x_stride);
                        rn[u % AHEAD] = load_raw<V>(dn + next * dn_stride);
                    }
#pragma unroll
                    for (int j = 0; j < V; ++j) {
                        z[j] = bias[j];
#pragma unroll
                        for (int i = 0; i < W; ++i)
                            z[j] = fmaf(w[i][j], e[(u + 4 - (W - 1) + i) % 4][j], z[j]);
                        s[j] = sigmoid(z[j]);
                        z[j] *= s[j];   // y
                    }
                    if (any_unit) {
#pragma unroll
                        for (int j = 0; j < V; ++j) {
                            sq = fmaf(z[j], z[j], sq);
                            dot = fmaf(z[j], d[j], dot);
                        }
                        sq = V == 8 ? sum_to16(sq, lgh) : sum_to32(sq, lgh);
                        dot = V == 8 ? sum_to16(dot, lgh) : sum_to32(dot, lgh);
                        const float r = unit ? __builtin_amdgcn_rsqf(sq + a.eps) : 1.0f, c = unit ? r * dot * r * r : 0.0f;   // (r dot first: for a row of zeros it is 0)
#pragma unroll
                        for (int j = 0; j < V; ++j)
                            d[j] = fmaf(r, d[j], -c * z[j]);   // dy
                    }
#pragma unroll
                    for (int j = 0; j < V; ++j)
                        dz[u][j] = d[j] * fmaf(z[j], 1.0f - s[j], s[j]);
                    if (t < p.t1)
#pragma unroll
                        for (int j = 0; j < V; ++j) {
                            if constexpr (BIAS)
                                dbias[j] += dz[u][j];
#pragma unroll
                            for (int i = 0; i < W; ++i)
                                dw[i][j] = fmaf(dz[u][j], e[(u + 4 - (W - 1) + i) % 4][j], dw[i][j]);
                        }
                } else {
#pragma unroll
                    for (int j = 0; j < V; ++j)
                        dz[u][j] = 0.0f;
                }
                if (t >= p.t0 + W - 1 || p.t0 == 0) {   // row t of E
                    float de[V];
#pragma unroll
                    for (int j = 0; j < V; ++j) {
                        de[j] = w[0][j] * dz[u][j];
#pragma unroll
                        for (int i = 1; i < W; ++i)
                            de[j] = fmaf(w[i][j], dz[(u + 4 - i) % 4][j], de[j]);
                    }
                    if (t >= p.len && ds1) {
                        float more[V];
                        unpack(load_raw<V>(ds1 + (int64_t)(t - p.len) * a.C), more);
#pragma unroll
                        for (int j = 0; j < V; ++j)
                            de[j] += more[j];
                    }
                    if (t >= W - 1)
                        store_values(dx + (int64_t)(t - (W - 1)) * a.x_stride, de);
                    else if (ds0)
                        store_values(ds0 + (int64_t)t * a.C, de);
                }
            });
    }

#pragma unroll
    for (int i = 0; i < W; ++i)
#pragma unroll
        for (int j = 0; j < V; ++j)
            sums[wave][i * PLANE + lane * V + j] = dw[i][j];
    if constexpr (BIAS)
#pragma unroll
        for (int j = 0; j < V; ++j)
            sums[wave][W * PLANE + lane * V + j] = dbias[j];
    __syncthreads();
    const int first = group * PLANE;
    for (int i = threadIdx.x; i < (W + BIAS) * PLANE; i += 256) {
        const int plane = i / PLANE, c = first + i % PLANE;
        if (c < a.C)   // (weights lie channel by channel)
            to[plane < W ? (int64_t)c * W + plane : (int64_t)W * a.C + c] = sums[0][i] + sums[1][i] + sums[2][i] + sums[3][i];
    }
}

template <typename T>
void launch_conv_grad_typed(int width, const ConvGradArgs &g, int64_t length, float *dweight, float *dbias, float *dA_log, float *ddt_bias, hipStream_t stream)
{
    const int64_t blocks = (int64_t)g.parts * (grad_groups(g.f.C, GRAD_CHANNELS<T>) + g.f.gates);
    auto go = [&]<int W>() {
        if (g.f.bias)
            launch_part(kvb_conv_grad_kernel<T, W, true>, true, false, blocks, 256, stream, g, length);
        else
            launch_part(kvb_conv_grad_kernel<T, W, false>, true, false, blocks, 256, stream, g, length);
    };
    if (g.parts == 0) {
    } else if (width == 4)
        go.template operator()<4>();
    else if (width == 3)
        go.template operator()<3>();
    else
        go.template operator()<2>();
    const int64_t gates = (int64_t)(width + (dbias != nullptr)) * g.f.C;
    launch_sums(g.part, g.parts, g.columns, SumsTo{{dweight, dbias, dA_log, ddt_bias}, {0, (int64_t)width * g.f.C, gates, gates + g.f.Hv}}, stream);
}

}  // namespace kvb_impl
#endif  // KVB_CONV_GRAD_KERNEL_H
