// kvb_norm_backward, and the sums of columns that end it and kvb_conv_backward.  With h = s r, r = 1 / sqrt(mean s^2 + eps), c = gate / (1 + exp(-gate)),
//     dh = dout c weight     ds = r (dh - h mean(dh h)) + dsum     dx = scale ds,  dres = ds
//     dgate = dout h weight c',  c' = (1 + gate (1 - t)) t,  t = 1 / (1 + exp(-gate))     dweight = sum over rows of dout c h
// Rows go to lanes as in kvb_norm; a workgroup takes rows in turn, its lanes keep their columns' sums of dweight in registers and leave
// one part in the end; kvb_sums_kernel adds the parts in order: the same inputs give the same bits.
#include "kvb_layer_device.h"

namespace kvb_impl {

namespace {

template <typename TX, typename T>
struct Grad8 {
    float s[8], dh[8];   // dh: dout c, times the weight where it says so
    Raw8<T> dout, gate;
    Raw8<TX> dsum;
};

// EARLY: dsum too is asked for with the others (where the lane has the registers)
template <bool EARLY, typename TX, typename T>
__device__ __forceinline__ void load_grad(const NormGradArgs &g, int64_t token, int64_t row, int64_t in_token, int at, Grad8<TX, T> &p)
{
    const NormArgs &a = g.f;
    const Raw8<TX> x = load_raw8(static_cast<const TX *>(a.x) + token * a.x_stride + in_token + at);
    p.dout = load_raw8(static_cast<const T *>(g.dout) + row * a.width + at);
    if (a.gate)
        p.gate = load_raw8(static_cast<const T *>(a.gate) + token * a.gate_stride + in_token + at);
    if (EARLY && g.dsum)
        p.dsum = load_raw8(static_cast<const TX *>(g.dsum) + row * a.width + at);
    unpack8(x, p.s);
    unpack8(p.dout, p.dh);
    if (a.gate) {
        float z[8];
        unpack8(p.gate, z);
#pragma unroll
        for (int j = 0; j < 8; ++j)
            p.dh[j] *= z[j] * sigmoid(z[j]);
    }
}
// sums of s^2 and dh weight s
template <typename TX, typename T>
__device__ __forceinline__ void sums_of(const Grad8<TX, T> &p, const float (&w)[8], float &sq, float &dot)
{
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        sq = fmaf(p.s[j], p.s[j], sq);
        dot = fmaf(p.dh[j] * w[j], p.s[j], dot);
    }
}
template <bool EARLY, typename TX, typename T>
__device__ __forceinline__ void finish_grad(const NormGradArgs &g, int64_t token, int64_t row, int64_t in_token, int at, const Grad8<TX, T> &p, const float (&w)[8],
                                            float (&dw)[8], float r, float mean)
{
    const NormArgs &a = g.f;
    float ds[8], y[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const float h = p.s[j] * r;
        dw[j] = fmaf(p.dh[j], h, dw[j]);
        ds[j] = r * fmaf(-h, mean, p.dh[j] * w[j]);
    }
    if (a.gate) {
        float z[8], d[8];
        unpack8(p.gate, z);
        unpack8(p.dout, d);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float t = sigmoid(z[j]);
            y[j] = d[j] * (p.s[j] * r * w[j]) * (t * fmaf(z[j], 1.0f - t, 1.0f));
        }
        store8(static_cast<T *>(g.dgate) + token * a.gate_stride + in_token + at, y);
    }
    if (g.dsum) {
        unpack8(EARLY ? p.dsum : load_raw8(static_cast<const TX *>(g.dsum) + row * a.width + at), y);
#pragma unroll
        for (int j = 0; j < 8; ++j)
            ds[j] += y[j];
    }
    if (g.dres)
        store8(static_cast<TX *>(g.dres) + row * a.width + at, ds);
#pragma unroll
    for (int j = 0; j < 8; ++j)
        ds[j] *= g.dx_scale;
    store8(static_cast<TX *>(g.dx) + token * a.x_stride + in_token + at, ds);
}

}  // namespace

template <typename TX, typename T, int NV>
__global__ __launch_bounds__(256) void kvb_norm_grad_kernel(const NormGradArgs g, int lg)
{
    __shared__ float sums[4][64 * 8 * NV];
    const NormArgs &a = g.f;
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, lanes = 1 << lg, own = lane & (lanes - 1);
    const int64_t step = (int64_t)gridDim.x * 256 >> lg;
    float w[NV][8], dw[NV][8] = {};
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int at = 8 * (own + i * lanes);
        unpack8(load_raw8(static_cast<const T *>(a.weight) + (at < a.width ? at : 0)), w[i]);
    }
    for (int64_t first = (int64_t)blockIdx.x * 256 >> lg; first < a.rows; first += step) {
        const int64_t row = first + (threadIdx.x >> lg), token = a.heads == 1 ? row : row / a.heads, in_token = (row - token * a.heads) * a.width;
        Grad8<TX, T> p[NV];
        float sq = 0.0f, dot = 0.0f;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int at = 8 * (own + i * lanes);
            if (row < a.rows && at < a.width) {
                load_grad<(NV < 4)>(g, token, row, in_token, at, p[i]);
                sums_of(p[i], w[i], sq, dot);
            }
        }
        const float n = 1.0f / (float)a.width, r = __builtin_amdgcn_rsqf(sum_lanes(sq, lg) * n + a.eps), mean = sum_lanes(dot, lg) * r * n;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int at = 8 * (own + i * lanes);
            if (row < a.rows && at < a.width)
                finish_grad<(NV < 4)>(g, token, row, in_token, at, p[i], w[i], dw[i], r, mean);
        }
    }
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j)
            sums[wave][(i * 64 + lane) * 8 + j] = dw[i][j];
    __syncthreads();
    for (int c = threadIdx.x; c < a.width; c += 256) {   // column c: vector c / 8, of lane (c / 8) % lanes of each row's
        const int i = c / 8 / lanes, l = c / 8 % lanes;
        float s = 0.0f;
        for (int v = 0; v < 4; ++v)
            for (int k = l; k < 64; k += lanes)
                s += sums[v][(i * 64 + k) * 8 + c % 8];
        g.part[(int64_t)blockIdx.x * a.width + c] = s;
    }
}

template <typename TX, typename T, int NV, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void kvb_norm_grad_row_kernel(const NormGradArgs g)
{
    __shared__ float part[2][2 * WAVES];
    const NormArgs &a = g.f;
    const int wave = threadIdx.x / 64;
    float w[NV][8], dw[NV][8] = {};
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int at = 8 * (threadIdx.x + i * 64 * WAVES);
        unpack8(load_raw8(static_cast<const T *>(a.weight) + (at < a.width ? at : 0)), w[i]);
    }
    int turn = 0;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x, turn ^= 1) {
        const int64_t token = a.heads == 1 ? row : row / a.heads, in_token = (row - token * a.heads) * a.width;
        Grad8<TX, T> p[NV];
        float sq = 0.0f, dot = 0.0f;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int at = 8 * (threadIdx.x + i * 64 * WAVES);
            if (at < a.width) {
                load_grad<(NV < 4)>(g, token, row, in_token, at, p[i]);
                sums_of(p[i], w[i], sq, dot);
            }
        }
        sq = sum_lanes(sq, 6);
        dot = sum_lanes(dot, 6);
        if (threadIdx.x % 64 == 0) {   // (two sets in turn: a barrier a row)
            part[turn][wave] = sq;
            part[turn][WAVES + wave] = dot;
        }
        __syncthreads();
        const float *q = part[turn], n = 1.0f / (float)a.width;
        sq = q[0];
        dot = q[WAVES];
#pragma unroll
        for (int v = 1; v < WAVES; ++v) {
            sq += q[v];
            dot += q[WAVES + v];
        }
        const float r = __builtin_amdgcn_rsqf(sq * n + a.eps), mean = dot * r * n;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int at = 8 * (threadIdx.x + i * 64 * WAVES);
            if (at < a.width)
                finish_grad<(NV < 4)>(g, token, row, in_token, at, p[i], w[i], dw[i], r, mean);
        }
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int at = 8 * (threadIdx.x + i * 64 * WAVES);
        if (at < a.width)
            store8(g.part + (int64_t)blockIdx.x * a.width + at, dw[i]);
    }
}

// 64 columns a workgroup; wave v has the rows v, v + 16, ..
__global__ __launch_bounds__(1024) void kvb_sums_kernel(const float *part, int parts, int64_t columns, const SumsTo to)
{
    __shared__ float sums[16][64];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const int64_t c = (int64_t)blockIdx.x * 64 + lane;
    float s = 0.0f;
    if (c < columns)
#pragma unroll 16
        for (int p = wave; p < parts; p += 16)
            s += part[p * columns + c];
    sums[wave][lane] = s;
    __syncthreads();
    if (wave != 0 || c >= columns)
        return;
    for (int v = 1; v < 16; ++v)
        s += sums[v][lane];
    float *p = to.to[0];
    int64_t begin = to.begin[0];
#pragma unroll
    for (int i = 1; i < 4; ++i)
        if (to.to[i] && c >= to.begin[i]) {
            p = to.to[i];
            begin = to.begin[i];
        }
    p[c - begin] = s;
}

void launch_sums(const float *part, int parts, int64_t columns, const SumsTo &to, hipStream_t stream)
{
    launch_part(kvb_sums_kernel, parts == 0, true, (columns + 63) / 64, 1024, stream, part, parts, columns, to);
}

template <typename TX, typename T>
void launch_norm_grad_typed(const NormGradArgs &g, float *dweight, hipStream_t stream)
{
    const NormArgs &a = g.f;
    const int vectors = a.width / 8;
    if (g.parts == 0) {
    } else if (vectors > 256) {
        auto go = [&]<int NV, int WAVES>() { launch_part(kvb_norm_grad_row_kernel<TX, T, NV, WAVES>, true, false, g.parts, 64 * WAVES, stream, g); };
        if (vectors <= 512)
            go.template operator()<2, 4>();
        else if (vectors <= 1024)
            go.template operator()<4, 4>();
        else
            go.template operator()<4, 8>();
    } else {
        int lg = 2;
        while (lg < 6 && (1 << lg) < vectors)
            ++lg;
        auto go = [&]<int NV>() { launch_part(kvb_norm_grad_kernel<TX, T, NV>, true, false, g.parts, 256, stream, g, lg); };
        if (vectors <= 64)
            go.template operator()<1>();
        else if (vectors <= 128)
            go.template operator()<2>();
        else
            go.template operator()<4>();
    }
    launch_sums(g.part, g.parts, a.width, SumsTo{{dweight, nullptr, nullptr, nullptr}, {0, 0, 0, 0}}, stream);
}

template void launch_norm_grad_typed<float, float>(const NormGradArgs &, float *, hipStream_t);
template void launch_norm_grad_typed<bf16_t, bf16_t>(const NormGradArgs &, float *, hipStream_t);
template void launch_norm_grad_typed<f16_t, f16_t>(const NormGradArgs &, float *, hipStream_t);
template void launch_norm_grad_typed<float, bf16_t>(const NormGradArgs &, float *, hipStream_t);
template void launch_norm_grad_typed<float, f16_t>(const NormGradArgs &, float *, hipStream_t);

}  // namespace kvb_impl
