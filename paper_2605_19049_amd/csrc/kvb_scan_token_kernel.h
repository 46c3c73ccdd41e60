// kvb_scan token by token, for calls of about one token a sequence: serving's single-token step.
//     y = S'k,  e = beta (v - a y),  o = scale (a S'q + (k.q) e),  S = a S + k e',   a = exp(g)
// Everything is fp32 and on the vector units.  A call reads and writes the states and little else (4 d^2 bytes each way for each
// v-head, against 6 d bytes of a bf16 token), so what counts is that all of a state is on its way before anything waits: a wave
// has 32 columns, 4 of them and d / 8 rows a lane, asks for them in d / 8 loads of 16 bytes (128 bytes in a row from 8 lanes) and
// needs no other wave.  Measured: 16 single tokens of 32 v-heads of 128, 67.6 MB, 14.1 us or 4.8 TB/s (a copy of 1 GiB: 5.2 TB/s); 1 token
// 3.9 us, which is launch and latency.  A token then costs one pass over the registers for y and S'q and three additions across 8 lanes.
#ifndef KVB_SCAN_TOKEN_KERNEL_H
#define KVB_SCAN_TOKEN_KERNEL_H

#include "kvb_scan_device.h"

namespace kvb_impl {

template <typename T>
struct alignas(4 * sizeof(T)) Four {
    T x[4];
};

// the sum over 8 lanes, for all of them
template <int CTRL>
__device__ __forceinline__ float plus_lane(float x)
{
    return x + __uint_as_float(__builtin_amdgcn_update_dpp(0u, __float_as_uint(x), CTRL, 0xF, 0xF, false));
}
__device__ __forceinline__ float sum_lanes8(float x) { return plus_lane<0x141>(plus_lane<0x4E>(plus_lane<0xB1>(x))); }

template <typename TIn, typename TOut, int D>
__global__ __launch_bounds__(64) void kvb_scan_token_kernel(const ScanArgs a)
{
    constexpr int R = D / 8, PARTS = D / 32;   // rows of a lane; waves of a state
    const int lane = threadIdx.x, rows = R * (lane % 8), unit = blockIdx.x / PARTS, col = 32 * (blockIdx.x % PARTS) + 4 * (lane / 8);
    const int b = unit / a.Hv, hv = unit - b * a.Hv, hk = hv / a.r;
    const int row = state_row(a.slot, a.n_slots, b);
    if (row < 0)
        return;
    const Span span = span_of(a.start, a.n_tokens, b);
    const size_t own = ((size_t)row * a.Hv + hv) * D * D + rows * D + col;
    f32x4_t S[R] = {};
    if (a.state0)
#pragma unroll
        for (int i = 0; i < R; ++i)
            S[i] = *reinterpret_cast<const f32x4_t *>(a.state0 + own + i * D);
    // a token's inputs, asked for a token ahead (the last one's once more)
    Four<TIn> k[R / 4], q[R / 4], v;
    float gate = 0.0f, beta = 0.0f;
    auto request = [&](int t) {
        const size_t at = span.first + t;
        const TIn *kp = static_cast<const TIn *>(a.k) + at * a.k_stride + hk * D + rows, *qp = static_cast<const TIn *>(a.q) + at * a.q_stride + hk * D + rows;
#pragma unroll
        for (int i = 0; i < R / 4; ++i) {
            k[i] = *reinterpret_cast<const Four<TIn> *>(kp + 4 * i);
            q[i] = *reinterpret_cast<const Four<TIn> *>(qp + 4 * i);
        }
        v = *reinterpret_cast<const Four<TIn> *>(static_cast<const TIn *>(a.v) + at * a.v_stride + hv * D + col);
        gate = a.g[at * a.Hv + hv];
        beta = a.beta[at * a.Hv + hv];
    };
    if (span.len > 0)
        request(0);
    for (int t = 0; t < span.len; ++t) {
        float kr[R], qr[R];
#pragma unroll
        for (int i = 0; i < R; ++i) {
            kr[i] = to_f32(k[i / 4].x[i % 4]);
            qr[i] = to_f32(q[i / 4].x[i % 4]);
        }
        f32x4_t e = {to_f32(v.x[0]), to_f32(v.x[1]), to_f32(v.x[2]), to_f32(v.x[3])};
        const float al = decay(log2_gate(gate)), be = beta;
        request(min(t + 1, span.len - 1));
        float kq = 0.0f;
        f32x4_t y = {}, z = {};
#pragma unroll
        for (int i = 0; i < R; ++i) {
            kq = fmaf(kr[i], qr[i], kq);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                y[j] = fmaf(kr[i], S[i][j], y[j]);
                z[j] = fmaf(qr[i], S[i][j], z[j]);
            }
        }
        kq = sum_lanes8(kq);
        Four<TOut> o;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            e[j] = be * fmaf(-al, sum_lanes8(y[j]), e[j]);
            o.x[j] = from_f32<TOut>(a.scale * fmaf(kq, e[j], al * sum_lanes8(z[j])));
        }
#pragma unroll
        for (int i = 0; i < R; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j)
                S[i][j] = fmaf(kr[i], e[j], al * S[i][j]);
        if (lane % 8 == 0)
            *reinterpret_cast<Four<TOut> *>(static_cast<TOut *>(a.out) + ((size_t)(span.first + t) * a.Hv + hv) * D + col) = o;
    }
    if (a.state1)
#pragma unroll
        for (int i = 0; i < R; ++i)
            *reinterpret_cast<f32x4_t *>(a.state1 + own + i * D) = S[i];
}

}  // namespace kvb_impl
#endif  // KVB_SCAN_TOKEN_KERNEL_H
