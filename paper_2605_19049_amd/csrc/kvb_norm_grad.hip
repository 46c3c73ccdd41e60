// kvb_norm_backward, and the sums of columns that end it and kvb_conv_backward.  With h = s r, r = 1 / sqrt(mean s^2 + eps), c = gate / (1 + exp(-gate)),
//     dh = dout c weight     ds = r (dh - h mean(dh h)) + dsum     dx = scale ds,  dres = ds
//     dgate = dout h weight c',  c' = (1 + gate (1 - t)) t,  t = 1 / (1 + exp(-gate))     dweight = sum over rows of dout c h
// A workgroup takes rows in turn, its lanes keep their columns' sums of dweight in registers and leave
// one part in the end; kvb_sums_kernel adds the parts in order: the same inputs give the same bits.
// Bounded by memory: 8192 x 32 heads of 128 with gate, x in fp32, 470 MB, 92.5 us (4 of them the sums) or 5.1 TB/s; 8000 rows of 2048, bf16, with dsum and dres
// 164 MB, 37.5 us, one row a wave with four vectors a lane, whose registers left two waves a SIMD, 45.8; small calls by their launches: two from some tens of rows on, 7 us, one below.
#include "kvb_layer_device.h"

namespace kvb_impl {

namespace {

// What a row has of 8 columns, as it lies in memory
template <typename TX, typename T>
struct GradRaw {
    Raw8<TX> x, dsum;
    Raw8<T> dout, gate;
};
template <typename TX, typename T>
struct Grad8 {
    float s[8], dh[8];   // dh: dout c
};

template <typename TX, typename T>
__device__ __forceinline__ void request(const NormGradArgs &g, int64_t token, int64_t row, int64_t in_token, int at, GradRaw<TX, T> &p)
{
    const NormArgs &a = g.f;
    p.x = load_raw8(static_cast<const TX *>(a.x) + token * a.x_stride + in_token + at);
    p.dout = load_raw8(static_cast<const T *>(g.dout) + row * a.width + at);
    if (a.gate)
        p.gate = load_raw8(static_cast<const T *>(a.gate) + token * a.gate_stride + in_token + at);
    if (g.dsum)
        p.dsum = load_raw8(static_cast<const TX *>(g.dsum) + row * a.width + at);
}
template <typename TX, typename T>
__device__ __forceinline__ void take(const NormGradArgs &g, const GradRaw<TX, T> &r, Grad8<TX, T> &p)
{
    unpack8(r.x, p.s);
    unpack8(r.dout, p.dh);
    if (g.f.gate) {
        float z[8];
        unpack8(r.gate, z);
#pragma unroll
        for (int j = 0; j < 8; ++j)
            p.dh[j] *= z[j] * sigmoid(z[j]);
    }
}
// The same bits, anew: what is worked out from them is worked out again, and takes no register until then
template <typename V>
__device__ __forceinline__ void renew(V &x)
{
    static_assert(sizeof(V) % 16 == 0);
    typedef uint32_t v4 __attribute__((ext_vector_type(4)));
    struct Words { v4 w[sizeof(V) / 16]; } words = __builtin_bit_cast(Words, x);
#pragma unroll
    for (int i = 0; i < (int)(sizeof(V) / 16); ++i)
        asm volatile("" : "+v"(words.w[i]));
    x = __builtin_bit_cast(V, words);
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
template <typename TX, typename T>
__device__ __forceinline__ void finish_grad(const NormGradArgs &g, int64_t token, int64_t row, int64_t in_token, int at, const GradRaw<TX, T> &raw,
                                            const Grad8<TX, T> &p, const float (&w)[8], float (&dw)[8], float r, float mean)
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
        unpack8(raw.gate, z);
        unpack8(raw.dout, d);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float t = sigmoid(z[j]);
            y[j] = d[j] * (p.s[j] * r * w[j]) * (t * fmaf(z[j], 1.0f - t, 1.0f));
        }
        store8(static_cast<T *>(g.dgate) + token * a.gate_stride + in_token + at, y);
    }
    if (g.dsum) {
        unpack8(raw.dsum, y);
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

// Rows of up to 512 elements: 2^lg lanes a row
template <typename TX, typename T>
__global__ __launch_bounds__(256) void kvb_norm_grad_kernel(const NormGradArgs g, int lg)
{
    __shared__ float sums[4][64 * 8];
    const NormArgs &a = g.f;
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, lanes = 1 << lg, own = lane & (lanes - 1), at = 8 * own;
    const int64_t step = (int64_t)gridDim.x * 256 >> lg;
    const float n = 1.0f / (float)a.width;
    float w[8], dw[8] = {};
    unpack8(load_raw8(static_cast<const T *>(a.weight) + (at < a.width ? at : 0)), w);
    // (all lanes go round as often: sums go over all lanes of a row)
    for (int64_t first = (int64_t)blockIdx.x * 256 >> lg; first < a.rows; first += step) {
        const int64_t row = first + (threadIdx.x >> lg), token = token_of(a, row), in_token = (row - token * a.heads) * a.width;
        const bool there = row < a.rows && at < a.width;
        GradRaw<TX, T> raw;
        Grad8<TX, T> p;
        float sq = 0.0f, dot = 0.0f;
        if (there) {
            request(g, token, row, in_token, at, raw);
            take(g, raw, p);
            sums_of(p, w, sq, dot);
        }
        const float r = __builtin_amdgcn_rsqf(sum_lanes(sq, lg) * n + a.eps), mean = sum_lanes(dot, lg) * r * n;
        if (there)
            finish_grad(g, token, row, in_token, at, raw, p, w, dw, r, mean);
    }
#pragma unroll
    for (int j = 0; j < 8; ++j)
        sums[wave][lane * 8 + j] = dw[j];
    __syncthreads();
    for (int c = threadIdx.x; c < a.width; c += 256) {   // (column c: lane c / 8 of each row's)
        float s = 0.0f;
        for (int v = 0; v < 4; ++v)
            for (int l = 0; l < 64; l += lanes)
                s += sums[v][l * 8 + c];
        g.part[(int64_t)blockIdx.x * a.width + c] = s;
    }
}

// Longer rows: a row the waves that its vectors need with NV a lane (up to eight of 64 lanes), as many rows side by side as eight waves have.  The next
// rows are asked for ahead; with four vectors a lane has no registers for that, nor for the weights, and works out what it needs twice.
template <typename TX, typename T, int NV>
__global__ __launch_bounds__(512) void kvb_norm_grad_row_kernel(const NormGradArgs g, int threads)
{
    __shared__ float part[2][16], sums[NV == 1 ? 512 * 8 : 1];
    const NormArgs &a = g.f;
    const int team = __builtin_amdgcn_readfirstlane(threadIdx.x / threads), teams = blockDim.x / threads, own = threadIdx.x - team * threads;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), waves = threads / 64;
    float w[NV][8], dw[NV][8] = {};
    auto load_weight = [&] {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int at = 8 * (own + i * threads);
            unpack8(load_raw8(static_cast<const T *>(a.weight) + (at < a.width ? at : 0)), w[i]);
        }
    };
    if (NV < 4)
        load_weight();
    GradRaw<TX, T> raw[NV], next[NV];
    auto ask = [&](int64_t row, GradRaw<TX, T> (&r)[NV]) {
        const int64_t token = token_of(a, row), in_token = (row - token * a.heads) * a.width;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int at = 8 * (own + i * threads);
            if (at < a.width)
                request(g, token, row, in_token, at, r[i]);
        }
    };
    const int64_t first = (int64_t)blockIdx.x * teams, step = (int64_t)gridDim.x * teams;
    if (NV < 4 && first + team < a.rows)
        ask(first + team, next);
    int turn = 0;
    for (int64_t at_once = first; at_once < a.rows; at_once += step, turn ^= 1) {   // (the same for all waves)
        const int64_t row = at_once + team, token = token_of(a, row), in_token = (row - token * a.heads) * a.width;
        Grad8<TX, T> p[NV];
        float sq = 0.0f, dot = 0.0f;
        if (NV < 4) {
#pragma unroll
            for (int i = 0; i < NV; ++i)
                raw[i] = next[i];
            if (row + step < a.rows)
                ask(row + step, next);
        } else {
            ask(row, raw);
            load_weight();
        }
        if (row < a.rows)
#pragma unroll
            for (int i = 0; i < NV; ++i)
                if (8 * (own + i * threads) < a.width) {
                    take(g, raw[i], p[i]);
                    sums_of(p[i], w[i], sq, dot);
                }
        sq = sum_lanes(sq, 6);
        dot = sum_lanes(dot, 6);
        if (threadIdx.x % 64 == 0) {   // (two sets in turn: a barrier a row)
            part[turn][wave] = sq;
            part[turn][8 + wave] = dot;
        }
        lds_barrier();
        if (row < a.rows) {
            const float *q = part[turn] + team * waves, n = 1.0f / (float)a.width;
            sq = q[0];
            dot = q[8];
            for (int v = 1; v < waves; ++v) {
                sq += q[v];
                dot += q[8 + v];
            }
            const float r = __builtin_amdgcn_rsqf(sq * n + a.eps), mean = dot * r * n;
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int at = 8 * (own + i * threads);
                if (at < a.width) {
                    if (NV == 4) {
                        renew(raw[i].x);
                        renew(raw[i].dout);
                        if (a.gate)
                            renew(raw[i].gate);
                        take(g, raw[i], p[i]);
                    }
                    finish_grad(g, token, row, in_token, at, raw[i], p[i], w[i], dw[i], r, mean);
                }
            }
        }
    }
    float *to = g.part + (int64_t)blockIdx.x * a.width;
    if constexpr (NV == 1) {   // rows side by side
        if (teams > 1) {
            if (team > 0)
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    sums[(j * 512) + threadIdx.x] = dw[0][j];
            __syncthreads();
            if (team > 0)
                return;
            for (int v = 1; v < teams; ++v)
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    dw[0][j] += sums[j * 512 + v * threads + threadIdx.x];
        }
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int at = 8 * (own + i * threads);
        if (at < a.width)
            store8(to + at, dw[i]);
    }
}

// COLUMNS columns a workgroup of 1024; its rows of threads have the parts in turn
template <int COLUMNS>
__global__ __launch_bounds__(1024) void kvb_sums_kernel(const float *part, int parts, int64_t columns, const SumsTo to)
{
    constexpr int TURNS = 1024 / COLUMNS;
    __shared__ float sums[TURNS][COLUMNS];
    const int own = threadIdx.x % COLUMNS, turn = threadIdx.x / COLUMNS;
    const int64_t c = (int64_t)blockIdx.x * COLUMNS + own;
    float s = 0.0f;
    if (c < columns)
#pragma unroll 16
        for (int p = turn; p < parts; p += TURNS)
            s += part[p * columns + c];
    sums[turn][own] = s;
    __syncthreads();
    if (turn != 0 || c >= columns)
        return;
#pragma unroll
    for (int v = 1; v < TURNS; ++v)
        s += sums[v][own];
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
    if (parts > 64)
        launch_part(kvb_sums_kernel<16>, parts == 0, true, (columns + 15) / 16, 1024, stream, part, parts, columns, to);
    else
        launch_part(kvb_sums_kernel<128>, parts == 0, true, (columns + 127) / 128, 1024, stream, part, parts, columns, to);
}

template <typename TX, typename T>
void launch_norm_grad_typed(const NormGradArgs &with_work, float *dweight, hipStream_t stream)
{
    NormGradArgs g = with_work;
    const NormArgs &a = g.f;
    const int vectors = a.width / 8;
    const bool alone = g.parts == 1 && reinterpret_cast<uintptr_t>(dweight) % 16 == 0;   // its only part is the sum (parts are stored 16 bytes at a time)
    if (alone)
        g.part = dweight;
    if (g.parts > 0 && vectors <= 64) {
        int lg = 2;
        while (lg < 6 && (1 << lg) < vectors)
            ++lg;
        launch_part(kvb_norm_grad_kernel<TX, T>, true, alone, g.parts, 256, stream, g, lg);
    } else if (g.parts > 0) {
        const int nv = norm_vectors(a.width), threads = norm_threads(a.width), all = threads * norm_teams(a.width);
        auto go = [&]<int NV>() { launch_part(kvb_norm_grad_row_kernel<TX, T, NV>, true, alone, g.parts, all, stream, g, threads); };
        if (nv == 1)
            go.template operator()<1>();
        else if (nv == 2)
            go.template operator()<2>();
        else
            go.template operator()<4>();
    }
    if (!alone)
        launch_sums(g.part, g.parts, a.width, SumsTo{{dweight, nullptr, nullptr, nullptr}, {0, 0, 0, 0}}, stream);
}

template void launch_norm_grad_typed<float, float>(const NormGradArgs &, float *, hipStream_t);
template void launch_norm_grad_typed<bf16_t, bf16_t>(const NormGradArgs &, float *, hipStream_t);
template void launch_norm_grad_typed<f16_t, f16_t>(const NormGradArgs &, float *, hipStream_t);
template void launch_norm_grad_typed<float, bf16_t>(const NormGradArgs &, float *, hipStream_t);
template void launch_norm_grad_typed<float, f16_t>(const NormGradArgs &, float *, hipStream_t);

}  // namespace kvb_impl
