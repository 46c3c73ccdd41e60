// kvb_grad_norm, kvb_clip: the norm of many tensors together, and all of them cut down to a largest norm.
//     norm = sqrt(sum x^2)     to = from min(1, largest / (norm + 1e-6))
// A workgroup takes KVB_LIST_BLOCK elements of one tensor.  Squares are exact and summed in fp64: no range is left, and the norm does not
// depend on how the tensors are cut by more than its last bit.  Addresses need only an element's alignment: whole 16 bytes lie between a
// few elements at either end.
#include "kvb_layer_device.h"

namespace kvb_impl {

namespace {

struct BlockOf {
    int tensor;
    int64_t from;   // its first element
    int n;          // 0: nothing there
};
__device__ __forceinline__ BlockOf block_of(const ListArgs &a, int block)
{
    const int lane = threadIdx.x % 64;
    int before = 0;   // tensors that end at or before this block
    for (int i0 = 0; i0 < a.n; i0 += 64) {
        const int i = min(i0 + lane, a.n - 1);
        before += __popcll(__ballot(i0 + lane < a.n && a.first[i + 1] <= block));
    }
    const int i = __builtin_amdgcn_readfirstlane(min(before, a.n - 1));
    const int64_t from = (int64_t)(block - a.first[i]) * KVB_LIST_BLOCK, left = a.size[i] - from;
    return BlockOf{i, from, from < 0 || left <= 0 ? 0 : (int)min(left, (int64_t)KVB_LIST_BLOCK)};
}

__device__ __forceinline__ double squares(const float (&x)[8], double sum)
{
#pragma unroll
    for (int j = 0; j < 8; ++j)
        sum = fma((double)x[j], (double)x[j], sum);
    return sum;
}

// elements ahead of the first 16-byte address
template <typename T>
__device__ __forceinline__ int ahead_of(const T *p, int n)
{
    return min(n, (int)((-reinterpret_cast<uintptr_t>(p) & 15) / sizeof(T)));
}

template <typename T>
__device__ __forceinline__ double squares_of(const T *p, int n)
{
    double sum = 0.0;
    const int ahead = ahead_of(p, n), vectors = (n - ahead) / 8, tail = ahead + 8 * vectors;
#pragma unroll 4
    for (int i = threadIdx.x; i < vectors; i += 256) {
        float x[8];
        unpack8(load_raw8(p + ahead + 8 * i), x);
        sum = squares(x, sum);
    }
    const int at = (int)threadIdx.x < ahead ? threadIdx.x : tail + (int)threadIdx.x - ahead;
    if (at < n) {
        const double x = to_f32(p[at]);
        sum = fma(x, x, sum);
    }
    return sum;
}

__device__ __forceinline__ double sum_wave(double x)
{
#pragma unroll
    for (int s = 32; s > 0; s /= 2)
        x += __shfl_xor(x, s);
    return x;
}

template <typename T>
__device__ __forceinline__ void scale_of(const T *p, T *to, int n, float c)
{
    if (c == 1.0f && p == to)
        return;
    const bool alike = ((reinterpret_cast<uintptr_t>(p) ^ reinterpret_cast<uintptr_t>(to)) & 15) == 0;
    const int ahead = alike ? ahead_of(p, n) : 0, vectors = alike ? (n - ahead) / 8 : 0, tail = ahead + 8 * vectors;
#pragma unroll 4
    for (int i = threadIdx.x; i < vectors; i += 256) {
        float x[8];
        unpack8(load_raw8(p + ahead + 8 * i), x);
#pragma unroll
        for (int j = 0; j < 8; ++j)
            x[j] *= c;
        store8(to + ahead + 8 * i, x);
    }
    if ((int)threadIdx.x < ahead)
        to[threadIdx.x] = from_f32<T>(to_f32(p[threadIdx.x]) * c);
    for (int i = tail + threadIdx.x; i < n; i += 256)
        to[i] = from_f32<T>(to_f32(p[i]) * c);
}

}  // namespace

__global__ __launch_bounds__(256) void kvb_squares_kernel(const ListArgs a, double *sums)
{
    __shared__ double part[4];
    const BlockOf b = block_of(a, blockIdx.x);
    double sum = 0.0;
    if (b.n > 0) {
        const int type = a.type[b.tensor];
        const void *p = a.data[b.tensor];
        if (type == KVB_F32)
            sum = squares_of(static_cast<const float *>(p) + b.from, b.n);
        else if (type == KVB_BF16)
            sum = squares_of(static_cast<const bf16_t *>(p) + b.from, b.n);
        else
            sum = squares_of(static_cast<const f16_t *>(p) + b.from, b.n);
    }
    sum = sum_wave(sum);
    if (threadIdx.x % 64 == 0)
        part[threadIdx.x / 64] = sum;
    __syncthreads();
    if (threadIdx.x == 0)
        sums[blockIdx.x] = part[0] + part[1] + part[2] + part[3];
}

__global__ __launch_bounds__(1024) void kvb_root_kernel(const double *sums, int n, float *norm)
{
    __shared__ double part[16];
    double sum = 0.0;
#pragma unroll 8
    for (int i = threadIdx.x; i < n; i += 1024)
        sum += sums[i];
    sum = sum_wave(sum);
    if (threadIdx.x % 64 == 0)
        part[threadIdx.x / 64] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int v = 1; v < 16; ++v)
            sum += part[v];
        *norm = (float)sqrt(sum);
    }
}

__global__ __launch_bounds__(256) void kvb_clip_kernel(const ListArgs a, const float *norm, float largest)
{
    const BlockOf b = block_of(a, blockIdx.x);
    if (b.n <= 0)
        return;
    // (not fminf, which drops a norm that is not a number)
    const float cut = largest / (*norm + 1e-6f), c = cut > 1.0f ? 1.0f : cut;
    const int type = a.type[b.tensor];
    const void *p = a.data[b.tensor];
    void *to = a.to[b.tensor];
    if (type == KVB_F32)
        scale_of(static_cast<const float *>(p) + b.from, static_cast<float *>(to) + b.from, b.n, c);
    else if (type == KVB_BF16)
        scale_of(static_cast<const bf16_t *>(p) + b.from, static_cast<bf16_t *>(to) + b.from, b.n, c);
    else
        scale_of(static_cast<const f16_t *>(p) + b.from, static_cast<f16_t *>(to) + b.from, b.n, c);
}

void launch_grad_norm(const ListArgs &a, float *norm, double *work, hipStream_t stream)
{
    if (a.blocks > 0)
        launch_part(kvb_squares_kernel, true, false, a.blocks, 256, stream, a, work);
    launch_part(kvb_root_kernel, a.blocks == 0, true, 1, 1024, stream, (const double *)work, a.blocks, norm);
}
void launch_clip(const ListArgs &a, const float *norm, float largest, hipStream_t stream)
{
    launch_part(kvb_clip_kernel, true, true, a.blocks, 256, stream, a, norm, largest);
}

}  // namespace kvb_impl
