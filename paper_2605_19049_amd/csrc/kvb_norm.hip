// kvb_norm: with s = res + scale x as x's type holds it (x itself without a residual),
//     out = s / sqrt(mean s^2 + eps) weight gate / (1 + exp(-gate))
// The norm is of the rounded sum, so that kvb_norm_backward, which is given that, has the gradient of what was computed; out is rounded once.
// A lane has vectors of 8 elements.  Rows of up to 512 elements take 4 .. 64 lanes, several rows a wave; rows of up to 2048 a wave, or a
// workgroup where there are few of them; longer ones a workgroup.
// Bounded by memory: 8191 x 32 heads of 128 with their gate, bf16, 201 MB, 36.5 us or 5.5 TB/s; 8000 rows of 2048 with residual 131 MB, 28.1 us or 4.7 TB/s; 64 such
// rows 3.3 us, which is the launch.
#include "kvb_layer_device.h"

namespace kvb_impl {

namespace {

// 8 elements of a row, sum and norm apart
template <typename TX, typename T>
struct Part8 {
    float s[8];
    Raw8<T> gate;
};

template <bool STREAM, typename TX, typename T>
__device__ __forceinline__ void load_part(const NormArgs &a, int64_t token, int64_t row, int64_t in_token, int at, Part8<TX, T> &p)
{
    const Raw8<TX> x = load_raw8_if<STREAM>(static_cast<const TX *>(a.x) + token * a.x_stride + in_token + at);
    Raw8<TX> res{};
    if (a.res)
        res = load_raw8(static_cast<const TX *>(a.res) + row * a.width + at);
    if (a.gate)
        p.gate = load_raw8_if<STREAM>(static_cast<const T *>(a.gate) + token * a.gate_stride + in_token + at);
    unpack8(x, p.s);
    if (a.res) {
        float y[8];
        unpack8(res, y);
#pragma unroll
        for (int j = 0; j < 8; ++j)
            p.s[j] = rounded_to<TX>(fmaf(a.scale, p.s[j], y[j]));
    }
}
template <typename TX, typename T>
__device__ __forceinline__ void finish_part(const NormArgs &a, int64_t row, int at, const Part8<TX, T> &p, const float (&w)[8], float r)
{
    float y[8];
#pragma unroll
    for (int j = 0; j < 8; ++j)
        y[j] = p.s[j] * r * w[j];
    if (a.gate) {
        float z[8];
        unpack8(p.gate, z);
#pragma unroll
        for (int j = 0; j < 8; ++j)
            y[j] *= z[j] * sigmoid(z[j]);
    }
    if (a.sum)
        store8(static_cast<TX *>(a.sum) + row * a.width + at, p.s);
    store8(static_cast<T *>(a.out) + row * a.width + at, y);
}
__device__ __forceinline__ float squares(const float (&s)[8], float sum)
{
#pragma unroll
    for (int j = 0; j < 8; ++j)
        sum = fmaf(s[j], s[j], sum);
    return sum;
}

}  // namespace

// 2^lg lanes a row, NV vectors of 8 a lane
template <typename TX, typename T, int NV, bool STREAM>
__global__ __launch_bounds__(256) void kvb_norm_kernel(const NormArgs a, int lg)
{
    const int lane = threadIdx.x % 64, lanes = 1 << lg, own = lane & (lanes - 1);
    const int64_t step = (int64_t)gridDim.x * 256 >> lg;
    float w[NV][8];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int at = 8 * (own + i * lanes);
        unpack8(load_raw8(static_cast<const T *>(a.weight) + (at < a.width ? at : 0)), w[i]);
    }
    // (all lanes go round as often: sums go over all lanes of a row)
    for (int64_t first = (int64_t)blockIdx.x * 256 >> lg; first < a.rows; first += step) {
        const int64_t row = first + (threadIdx.x >> lg), token = token_of(a, row), in_token = (row - token * a.heads) * a.width;
        Part8<TX, T> p[NV];
        float sum = 0.0f;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int at = 8 * (own + i * lanes);
            if (row < a.rows && at < a.width) {
                load_part<STREAM>(a, token, row, in_token, at, p[i]);
                sum = squares(p[i].s, sum);
            }
        }
        const float r = __builtin_amdgcn_rsqf(sum_lanes(sum, lg) / (float)a.width + a.eps);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int at = 8 * (own + i * lanes);
            if (row < a.rows && at < a.width)
                finish_part(a, row, at, p[i], w[i], r);
        }
    }
}

// a workgroup a row
template <typename TX, typename T, int NV, int WAVES, bool STREAM>
__global__ __launch_bounds__(64 * WAVES) void kvb_norm_row_kernel(const NormArgs a)
{
    __shared__ float part[WAVES];
    const int64_t row = blockIdx.x, token = token_of(a, row), in_token = (row - token * a.heads) * a.width;
    Part8<TX, T> p[NV];
    Raw8<T> w[NV];
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int at = 8 * (threadIdx.x + i * 64 * WAVES);
        if (at < a.width) {
            w[i] = load_raw8(static_cast<const T *>(a.weight) + at);
            load_part<STREAM>(a, token, row, in_token, at, p[i]);
            sum = squares(p[i].s, sum);
        }
    }
    sum = sum_lanes(sum, 6);
    if (threadIdx.x % 64 == 0)
        part[threadIdx.x / 64] = sum;
    __syncthreads();
    float total = part[0];
#pragma unroll
    for (int v = 1; v < WAVES; ++v)
        total += part[v];
    const float r = __builtin_amdgcn_rsqf(total / (float)a.width + a.eps);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int at = 8 * (threadIdx.x + i * 64 * WAVES);
        if (at < a.width) {
            float y[8];
            unpack8(w[i], y);
            finish_part(a, row, at, p[i], y, r);
        }
    }
}

template <typename TX, typename T>
void launch_norm_typed(const NormArgs &a, hipStream_t stream)
{
    // x and the gate past the caches where they fill much of the last level: what reads the results next finds more of them there.  us, alone and with a matrix
    // product that reads out, plain / past them: gated, 4096 x 32 heads of 128 (64 MiB) 19.4 / 19.2 and 85.1 / 85.0, 8191 41.0 / 36.5 and 144.8 / 142.9; residual, 4096 rows
    // of 2048 12.7 / 15.2 and 68.5 / 70.8, 8191 (64 MiB) 25.6 / 25.0 and 138.4 / 138.1, 18000 57.9 / 57.2 and 345 / 340.  x in fp32, gated, alone: 8191 x 32 heads of 128 beside a
    // gate in bf16 53.8 / 47.6; 20000 x 32 all in fp32 183 / 199, so that calls all in fp32 with a gate lose 8 % by this rule, which looks at bytes alone.
    const int64_t read = a.rows * a.width * (int64_t)(sizeof(TX) + (a.gate ? sizeof(T) : 0) + (a.res ? sizeof(TX) : 0));
    const bool stream_x = read > 96 << 20;
    const int vectors = a.width / 8;
    if (vectors > 256 || (vectors > 64 && a.rows < 1024)) {
        auto go = [&]<int NV, int WAVES>() {
            if (stream_x)
                launch_part(kvb_norm_row_kernel<TX, T, NV, WAVES, true>, true, true, a.rows, 64 * WAVES, stream, a);
            else
                launch_part(kvb_norm_row_kernel<TX, T, NV, WAVES, false>, true, true, a.rows, 64 * WAVES, stream, a);
        };
        if (vectors <= 256)
            go.template operator()<1, 4>();
        else if (vectors <= 512)
            go.template operator()<2, 4>();
        else if (vectors <= 1024)
            go.template operator()<4, 4>();
        else
            go.template operator()<4, 8>();
        return;
    }
    int lg = 2;
    while (lg < 6 && (1 << lg) < vectors)
        ++lg;
    const int64_t rows_of_workgroup = 256 >> lg, n = (a.rows + rows_of_workgroup - 1) / rows_of_workgroup, blocks = n < 2048 ? n : 2048;
    auto go = [&]<int NV>() {
        if (stream_x)
            launch_part(kvb_norm_kernel<TX, T, NV, true>, true, true, blocks, 256, stream, a, lg);
        else
            launch_part(kvb_norm_kernel<TX, T, NV, false>, true, true, blocks, 256, stream, a, lg);
    };
    if (vectors <= 64)
        go.template operator()<1>();
    else if (vectors <= 128)
        go.template operator()<2>();
    else
        go.template operator()<4>();
}

template void launch_norm_typed<float, float>(const NormArgs &, hipStream_t);
template void launch_norm_typed<bf16_t, bf16_t>(const NormArgs &, hipStream_t);
template void launch_norm_typed<f16_t, f16_t>(const NormArgs &, hipStream_t);
template void launch_norm_typed<float, bf16_t>(const NormArgs &, hipStream_t);
template void launch_norm_typed<float, f16_t>(const NormArgs &, hipStream_t);

}  // namespace kvb_impl
