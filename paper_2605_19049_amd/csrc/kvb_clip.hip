// kvb_grad_norm, kvb_clip: the norm of many tensors together, and all of them cut down to a largest norm.
//     norm = sqrt(sum x^2)     to = from min(1, largest / (norm + 1e-6))
// A workgroup takes KVB_LIST_BLOCK elements of one tensor.  Squares are exact and summed in fp64: no range is left, and the norm does not
// depend on how the tensors are cut by more than its last bit.  Addresses need only an element's alignment: whole 16 bytes lie between a
// few elements at either end.
// Bounded by memory: 43 M bf16 elements are read in 15.6 us (5.5 TB/s, eight loads of a thread on their way; four: 24.6), then read once more and written in 26.8; both with the
// norm between them 45 us.  Results go past the caches: what of the tensors the first pass left there is then still there (plain stores: 54 us; 134 M
// elements in place, read by an addition next: the same either way).  Eleven small tensors 9.1 us, three launches.
// A result that lies otherwise among 16 bytes than its source goes element by element: clipping into the next tensors 63 us instead of 27.  Each workgroup looks through the list of tensors, 64 a
// step, before its first load: those 43 M elements in 50 / 300 / 1000 / 3000 tensors 44 / 48 / 54 / 90 us.
#include "kvb_layer_device.h"

namespace kvb_impl {

namespace {

// A part of a block, as scalars
struct Item {
    const void *p;
    void *to;
    int type, n;    // n = 0: nothing there
    int64_t from;   // its first element
};
__device__ __forceinline__ int of_lane(int x, int i) { return __builtin_amdgcn_readlane(x, i); }
__device__ __forceinline__ int64_t of_lane(int64_t x, int i)
{
    return (int64_t)((uint64_t)(uint32_t)of_lane((int)(x >> 32), i) << 32 | (uint32_t)of_lane((int)x, i));
}
// Lane i asks for all that there is of tensor i, so that up to 64 tensors take one wait, not two.
__device__ __forceinline__ Item item_of(const ListArgs &a, int unit, int split)
{
    const int lane = threadIdx.x % 64, block = unit / split, part = unit - block * split;
    int i = 0;   // the last tensor that the lane looked at; tensors that end at or before this block
    int before = 0;
    for (int i0 = 0; i0 + 64 < a.n; i0 += 64)
        before += __popcll(__ballot(a.first[i0 + lane + 1] <= block));
    // (what is left of the last 64, or of those that the block is among)
    const int base = before / 64 * 64;
    i = min(base + lane, a.n - 1);
    const int begin = a.first[i], end = a.first[i + 1], type = a.type[i];
    const int64_t size = a.size[i], p = reinterpret_cast<int64_t>(a.data[i]), to = reinterpret_cast<int64_t>(a.to ? a.to[i] : nullptr);
    const int at = min(base + (int)__popcll(__ballot(base + lane < a.n && end <= block)), a.n - 1) - base;
    const int64_t from = (int64_t)(block - of_lane(begin, at)) * KVB_LIST_BLOCK + part * (KVB_LIST_BLOCK / split), left = of_lane(size, at) - from;
    const bool there = block >= of_lane(begin, at) && left > 0;
    return Item{reinterpret_cast<const void *>(of_lane(p, at)), reinterpret_cast<void *>(of_lane(to, at)), of_lane(type, at),
                there ? (int)min(left, (int64_t)(KVB_LIST_BLOCK / split)) : 0, from};
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
    int i = threadIdx.x;
    for (; i + 7 * 256 < vectors; i += 8 * 256) {   // (eight loads on their way at once)
        Raw8<T> raw[8];
#pragma unroll
        for (int k = 0; k < 8; ++k)
            raw[k] = load_raw8(p + ahead + 8 * (i + k * 256));
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            float x[8];
            unpack8(raw[k], x);
            sum = squares(x, sum);
        }
    }
#pragma unroll 2
    for (; i < vectors; i += 256) {
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
__device__ __forceinline__ void scale8(const Raw8<T> &raw, T *to, float c)
{
    float x[8];
    unpack8(raw, x);
#pragma unroll
    for (int j = 0; j < 8; ++j)
        x[j] *= c;
    store8<true>(to, x);
}
template <typename T>
__device__ __forceinline__ void scale_of(const T *p, T *to, int n, float c)
{
    if (c == 1.0f && p == to)
        return;
    const bool alike = ((reinterpret_cast<uintptr_t>(p) ^ reinterpret_cast<uintptr_t>(to)) & 15) == 0;
    const int ahead = alike ? ahead_of(p, n) : 0, vectors = alike ? (n - ahead) / 8 : 0, tail = ahead + 8 * vectors;
    int i = threadIdx.x;
    for (; i + 7 * 256 < vectors; i += 8 * 256) {
        Raw8<T> raw[8];
#pragma unroll
        for (int k = 0; k < 8; ++k)
            raw[k] = load_raw8(p + ahead + 8 * (i + k * 256));
#pragma unroll
        for (int k = 0; k < 8; ++k)
            scale8(raw[k], to + ahead + 8 * (i + k * 256), c);
    }
#pragma unroll 2
    for (; i < vectors; i += 256)
        scale8(load_raw8(p + ahead + 8 * i), to + ahead + 8 * i, c);
    if ((int)threadIdx.x < ahead)
        to[threadIdx.x] = from_f32<T>(to_f32(p[threadIdx.x]) * c);
    for (i = tail + threadIdx.x; i < n; i += 256)
        to[i] = from_f32<T>(to_f32(p[i]) * c);
}

}  // namespace

__global__ __launch_bounds__(256) void kvb_squares_kernel(const ListArgs a, int split, double *sums)
{
    __shared__ double part[4];
    const Item b = item_of(a, blockIdx.x, split);
    double sum = 0.0;
    if (b.n > 0) {
        if (b.type == KVB_F32)
            sum = squares_of(static_cast<const float *>(b.p) + b.from, b.n);
        else if (b.type == KVB_BF16)
            sum = squares_of(static_cast<const bf16_t *>(b.p) + b.from, b.n);
        else
            sum = squares_of(static_cast<const f16_t *>(b.p) + b.from, b.n);
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

__global__ __launch_bounds__(256) void kvb_clip_kernel(const ListArgs a, int split, const float *norm, float largest)
{
    const float total = *norm;
    const Item b = item_of(a, blockIdx.x, split);
    if (b.n <= 0)
        return;
    // (not fminf, which drops a norm that is not a number)
    const float cut = largest / (total + 1e-6f), c = cut > 1.0f ? 1.0f : cut;
    if (b.type == KVB_F32)
        scale_of(static_cast<const float *>(b.p) + b.from, static_cast<float *>(b.to) + b.from, b.n, c);
    else if (b.type == KVB_BF16)
        scale_of(static_cast<const bf16_t *>(b.p) + b.from, static_cast<bf16_t *>(b.to) + b.from, b.n, c);
    else
        scale_of(static_cast<const f16_t *>(b.p) + b.from, static_cast<f16_t *>(b.to) + b.from, b.n, c);
}

void launch_grad_norm(const ListArgs &a, float *norm, double *work, hipStream_t stream)
{
    const int split = list_split(a.blocks);
    if (a.blocks > 0)
        launch_part(kvb_squares_kernel, true, false, (int64_t)a.blocks * split, 256, stream, a, split, work);
    launch_part(kvb_root_kernel, a.blocks == 0, true, 1, 1024, stream, (const double *)work, a.blocks * split, norm);
}
void launch_clip(const ListArgs &a, const float *norm, float largest, hipStream_t stream)
{
    const int split = list_split(a.blocks);
    launch_part(kvb_clip_kernel, true, true, (int64_t)a.blocks * split, 256, stream, a, split, norm, largest);
}

}  // namespace kvb_impl
