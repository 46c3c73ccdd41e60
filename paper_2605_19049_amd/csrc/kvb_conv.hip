// kvb_conv, kvb_conv_decode, kvb_conv_verify, kvb_conv_commit: what makes a layer's queries, keys, values and gates from the rows of its
// projection.  With E the state's rows followed by a sequence's inputs,
//     z_t = bias + sum_i w_i E_{t+i},  y = z / (1 + exp(-z)),  q, k = y / sqrt(sum y^2 + eps) over a head,  v = y
//     g = -exp(A_log) log(1 + exp(a + dt_bias)),  beta = 1 / (1 + exp(-b))
// A lane has 8 channels, so that loads and stores are 16 bytes (16-bit types), a head is 4, 8 or 16 neighbouring lanes and its sum of squares
// stays inside a row of 16.  A wave has 512 channels; the units behind the channels' are the gates'.  All arithmetic is fp32; what is rounded
// is the result, once, to its own type.
// Bounded by memory: 8191 tokens, 16 + 32 heads of 128, bf16, 272 MB in 59 us or 4.6 TB/s (a copy: 5.0 .. 5.2), of which the vector units are busy some 40: 130
// instructions for a token's 8 channels, two of them slow (exp2, rcp).  Small calls are bounded by the chain launch, start, slot, inputs: a prompt of 37 tokens 4.6 us, a
// single token 3.8, 64 of them 4.0, 512 11.6 (67 MB, 5.8 TB/s, some of it from the last level).
#include "kvb_layer_device.h"

namespace kvb_impl {

namespace {

// A lane's 8 channels: their weights, where their results go
template <typename T, int W>
struct Lane8 {
    float w[W][8], bias[8];
    T *to;               // the first token's
    int64_t to_stride;
    int lg;              // 2^lg lanes a head
    bool unit;           // q or k, to be of length one
    float eps;

    // (strides: elements from a token's q to the next one's, and of k and v)
    __device__ __forceinline__ Lane8(const ConvBase &a, int ch, int64_t q_stride, int64_t k_stride, int64_t v_stride) : lg(a.d == 128 ? 4 : a.d == 64 ? 3 : 2), eps(a.eps)
    {
        const T *wp = static_cast<const T *>(a.weight) + (int64_t)ch * W;
        Raw8<T> raw[W], rb{};
#pragma unroll
        for (int i = 0; i < W; ++i)
            raw[i] = load_raw8(wp + 8 * i);
        if (a.bias)
            rb = load_raw8(static_cast<const T *>(a.bias) + ch);
#pragma unroll
        for (int i = 0; i < W; ++i) {   // (8 channels of W taps each, one after the other)
            float y[8];
            unpack8(raw[i], y);
#pragma unroll
            for (int j = 0; j < 8; ++j)
                w[(8 * i + j) % W][(8 * i + j) / W] = y[j];
        }
        unpack8(rb, bias);
        const int nq = a.Hk * a.d;
        unit = a.unit && ch < 2 * nq;
        to = ch < nq ? static_cast<T *>(a.q) + ch : ch < 2 * nq ? static_cast<T *>(a.k) + (ch - nq) : static_cast<T *>(a.v) + (ch - 2 * nq);
        to_stride = ch < nq ? q_stride : ch < 2 * nq ? k_stride : v_stride;
    }
    __device__ __forceinline__ Lane8(const ConvBase &a, int ch) : Lane8(a, ch, a.Hk * a.d, a.Hk * a.d, a.Hv * a.d) {}   // packed
    // y from z, and of length one
    __device__ __forceinline__ void finish(float (&z)[8]) const
    {
        float sum = 0.0f;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            z[j] *= sigmoid(z[j]);
            sum = fmaf(z[j], z[j], sum);
        }
        sum = sum_to16(sum, lg);
        const float r = unit ? __builtin_amdgcn_rsqf(sum + eps) : 1.0f;
#pragma unroll
        for (int j = 0; j < 8; ++j)
            z[j] *= r;
    }
};

// Gates of the tokens t0 .. t1-1
template <typename T>
__device__ __forceinline__ void gates_of(const ConvBase &a, int64_t t0, int n, int lane)
{
    const GateLanes l = gate_lanes(a.Hv, lane);
    for (int h = l.head; h < a.Hv; h += l.heads) {
        const float rate = -expf(a.A_log[h]), shift = a.dt_bias[h];
#pragma unroll 4
        for (int t = l.token; t < n; t += l.tokens) {
            const float y = to_f32(static_cast<const T *>(a.a)[(t0 + t) * a.a_stride + h]) + shift;
            const float b = to_f32(static_cast<const T *>(a.b)[(t0 + t) * a.b_stride + h]);
            a.g[(t0 + t) * a.Hv + h] = rate * softplus(y);
            a.beta[(t0 + t) * a.Hv + h] = 1.0f / (1.0f + expf(-b));
        }
    }
}

}  // namespace

// Whole sequences: a wave takes the tokens of `length` places one after the other, with the taps' inputs in registers, and asks for four tokens ahead: one as one is taken (16
// bits, x from the caches); four as the four ahead of them are done; or (LARGE) before those are begun.  LARGE leaves a SIMD three waves for its registers (W = 2: four), the others
// four (fp32 with W = 4: three).  us, one / four / LARGE: 300 tokens 5.7 / 6.1 / 5.8, 1000 10.9 / 11.1 / 11.3, 2000 16.1 / 16.1 / 16.5; 24 sequences of up to 1500, 4 + 8 heads, past the caches
// 36.2 / 34.8 / 36.3, one of 8191 62.2 / 62.0 / 58.6; fp32, 5284 tokens, W = 3, 81 / 75 / 81.
template <typename T, int W, bool STREAM, bool LARGE>
__global__ __launch_bounds__(256, LARGE || sizeof(T) == 4 ? 3 : 4) void kvb_conv_kernel(const ConvArgs a, int units, int64_t length)
{
    constexpr bool ONE = sizeof(T) == 2 && !STREAM;
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), groups = conv_groups(a.C);
    const int unit = blockIdx.x * 4 + wave, each = groups + a.gates;
    if (unit >= units)
        return;
    const int w = unit / each, group = unit - w * each;
    const int64_t from = w * length;
    Shares shares(a, from, from + length, W - 1);
    if (group == groups) {
        while (shares.more()) {
            const Share p = shares.take();
            if (p.some)
                gates_of<T>(a, (int64_t)p.first + p.t0, p.t1 - p.t0, lane);
        }
        return;
    }
    const int ch = group * CONV_LANES + lane * 8;
    if (ch >= a.C)
        return;
    while (shares.more()) {
        const Share p = shares.take();
        if (!p.some)
            continue;
        const T *x = static_cast<const T *>(a.x) + (int64_t)p.first * a.x_stride + ch;
        const T *s0 = a.state0 ? static_cast<const T *>(a.state0) + (int64_t)p.row * (W - 1) * a.C + ch : nullptr;
        auto input_at = [&](int e) {   // row e of E
            if (e >= W - 1)
                return load_raw8(x + (int64_t)(e - (W - 1)) * a.x_stride);
            return s0 ? load_raw8(s0 + (int64_t)e * a.C) : Raw8<T>{};
        };
        if (p.t0 < p.t1) {
            Raw8<T> raw[4], next[4], before[W - 1];
#pragma unroll
            for (int i = 0; i < W - 1; ++i)
                before[i] = input_at(p.t0 + i);
            auto request = [&](int t, Raw8<T> (&to)[4]) {
                if (t < p.t1)
#pragma unroll
                    for (int u = 0; u < 4; ++u)
                        to[u] = load_raw8_if<STREAM>(x + (int64_t)min(t + u, p.t1 - 1) * a.x_stride);
            };
            request(p.t0, LARGE ? next : raw);
            const Lane8<T, W> l(a, ch, a.q_stride, a.k_stride, a.v_stride);
            T *out = l.to + ((int64_t)p.first + p.t0) * l.to_stride;
            float e[4][8];   // row t + W - 1 of E at (t - t0) % 4
#pragma unroll
            for (int i = 0; i < W - 1; ++i)
                unpack8(before[i], e[i + 4 - (W - 1)]);
            for (int t4 = p.t0; t4 < p.t1; t4 += 4) {
                if constexpr (LARGE) {
#pragma unroll
                    for (int u = 0; u < 4; ++u)
                        raw[u] = next[u];
                    request(t4 + 4, next);
                }
                static_for<4>([&](auto at) {
                    constexpr int u = at();
                    if (t4 + u >= p.t1)
                        return;
                    unpack8(raw[u], e[u]);
                    if constexpr (ONE)
                        if (t4 + u + 4 < p.t1)
                            raw[u] = load_raw8(x + (int64_t)(t4 + u + 4) * a.x_stride);
                    float z[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        z[j] = l.bias[j];
#pragma unroll
                        for (int i = 0; i < W; ++i)
                            z[j] = fmaf(l.w[i][j], e[(u + 4 - (W - 1) + i) % 4][j], z[j]);
                    }
                    l.finish(z);
                    store8(out, z);
                    out += l.to_stride;
                });
                if constexpr (!ONE && !LARGE)
                    request(t4 + 4, raw);
            }
        }
        // Who has the first token writes the last state: nobody else reads the first one's rows, which it may lie in.
        if (p.t0 == 0 && a.state1) {
            T *s1 = static_cast<T *>(a.state1) + (int64_t)p.row * (W - 1) * a.C + ch;
            Raw8<T> last[W - 1];
#pragma unroll
            for (int i = 0; i < W - 1; ++i)
                last[i] = input_at(p.len + i);
#pragma unroll
            for (int i = 0; i < W - 1; ++i)
                store_raw8<false, true>(s1 + (int64_t)i * a.C, last[i]);
        }
    }
}

// One token of each request: the state's rows and the token's are the taps' inputs, and moved on by one row the next state.
template <typename T, int W>
__global__ __launch_bounds__(256) void kvb_conv_token_kernel(const ConvTokenArgs a, int units)
{
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), groups = conv_groups(a.C);
    const int unit = blockIdx.x * 4 + wave, each = groups + a.gates;
    if (unit >= units)
        return;
    const int b = unit / each, group = unit - b * each;
    if (group == groups) {
        if (state_row(a.slot, a.n_slots, b) >= 0)
            gates_of<T>(a, b, 1, lane);
        return;
    }
    const int own_ch = group * CONV_LANES + lane * 8, ch = own_ch < a.C ? own_ch : 0;
    Raw8<T> raw[W] = {};
    raw[W - 1] = load_raw8(static_cast<const T *>(a.x) + (int64_t)b * a.x_stride + ch);
    const Lane8<T, W> l(a, ch);
    const int row = state_row(a.slot, a.n_slots, b);   // (behind the loads that do not need it)
    if (row < 0 || own_ch >= a.C)
        return;
    const int64_t at = (int64_t)row * (W - 1) * a.C + ch;
    if (a.state0)
#pragma unroll
        for (int i = 0; i < W - 1; ++i)
            raw[i] = load_raw8(static_cast<const T *>(a.state0) + at + (int64_t)i * a.C);
    float z[8];
#pragma unroll
    for (int j = 0; j < 8; ++j)
        z[j] = l.bias[j];
#pragma unroll
    for (int i = 0; i < W; ++i) {
        float e[8];
        unpack8(raw[i], e);
#pragma unroll
        for (int j = 0; j < 8; ++j)
            z[j] = fmaf(l.w[i][j], e[j], z[j]);
    }
    l.finish(z);
    store8(l.to + (int64_t)b * l.to_stride, z);
    if (a.state1) {
#pragma unroll
        for (int i = 0; i < W - 1; ++i)
            store_raw8<false, true>(static_cast<T *>(a.state1) + at + (int64_t)i * a.C, raw[i + 1]);
    }
}

// Drafts: a workgroup has all of a request's for 512 channels, a wave one of them.  A draft's taps reach back over its ancestors and then the state's rows;
// every row is read once and found by the others in LDS, where a lane needs nothing but its own channels.  us with the commit behind it, tree of 4 for
// 128 requests, bf16, 16 + 32 heads of 128: 12.5 (13.3 with launch arguments of 250 bytes instead of 180, and so
// were: each draft reading its rows by itself 14.2, a wave all drafts of a request 13.9, but 256 requests of 8 28.3, here 30.5).
template <typename T, int W>
__global__ __launch_bounds__(64 * KVB_MAX_DRAFTS) void kvb_conv_drafts_kernel(const ConvDraftArgs a)
{
    __shared__ Raw8<T> rows[W - 1 + KVB_MAX_DRAFTS][64];
    const int lane = threadIdx.x % 64, i0 = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int groups = conv_groups(a.C), each = groups + a.gates, b = blockIdx.x / each, group = blockIdx.x - b * each, token = b * a.T + i0;
    if (group == groups) {
        if (state_row(a.slot, a.n_slots, b) >= 0)
            gates_of<T>(a, token, 1, lane);
        return;
    }
    const int own_ch = group * CONV_LANES + lane * 8, ch = own_ch < a.C ? own_ch : 0;
    const Raw8<T> own = load_raw8(static_cast<const T *>(a.x) + (int64_t)token * a.x_stride + ch);
    const Lane8<T, W> l(a, ch);
    int up = lane - 1;   // lane i: draft i's parent
    if (a.parent) {
        const int i = min(lane, a.T - 1), p = a.parent[(int64_t)b * a.T + i];
        up = p < -1 || p >= i ? -1 : p;
    }
    const int row = state_row(a.slot, a.n_slots, b);   // (behind the loads that do not need it)
    if (row < 0)
        return;
    for (int i = i0; i < W - 1; i += a.T)
        rows[i][lane] = a.state0 ? load_raw8(static_cast<const T *>(a.state0) + ((int64_t)row * (W - 1) + i) * a.C + ch) : Raw8<T>{};
    rows[W - 1 + i0][lane] = own;
    __syncthreads();
    float z[8];
#pragma unroll
    for (int j = 0; j < 8; ++j)
        z[j] = l.bias[j];
    int place[W];   // a draft, or row W - 1 + place of the state
    place[W - 1] = i0;
#pragma unroll
    for (int k = W - 2; k >= 0; --k)
        place[k] = place[k + 1] >= 0 ? __builtin_amdgcn_readlane(up, place[k + 1]) : place[k + 1] - 1;
#pragma unroll
    for (int k = 0; k < W; ++k) {
        float e[8];
        unpack8(rows[W - 1 + place[k]][lane], e);
#pragma unroll
        for (int j = 0; j < 8; ++j)
            z[j] = fmaf(l.w[k][j], e[j], z[j]);
    }
    l.finish(z);
    if (own_ch < a.C)
        store8(l.to + (int64_t)token * l.to_stride, z);
}

// The state behind the accepted drafts: the last W - 1 rows of the state and theirs.
template <typename T, int W>
__global__ __launch_bounds__(256) void kvb_conv_commit_kernel(const ConvCommitArgs a, int units)
{
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), groups = conv_groups(a.C);
    const int unit = blockIdx.x * 4 + wave;
    if (unit >= units)
        return;
    const int b = unit / groups, group = unit - b * groups;
    const int row = state_row(a.slot, a.n_slots, b);
    if (row < 0)
        return;
    int n = __builtin_amdgcn_readfirstlane(a.accepted[b]);
    const int at = a.path ? a.path[(int64_t)b * a.T + min(lane, a.T - 1)] : lane, prev = __shfl_up(at, 1);
    const bool good = lane >= n || (at >= 0 && at < a.T && (lane == 0 || at > prev));
    n = n < 0 || n > a.T || !__all(good) ? 0 : n;
    const int ch = group * CONV_LANES + lane * 8;
    int from[W - 1];   // rows of E: the state's, then the accepted drafts'
#pragma unroll
    for (int i = 0; i < W - 1; ++i)
        from[i] = n + i < W - 1 ? -1 : __builtin_amdgcn_readlane(at, n + i - (W - 1));
    if (ch >= a.C)
        return;
    const T *x = static_cast<const T *>(a.x) + (int64_t)b * a.T * a.x_stride + ch;
    const T *s0 = a.state0 ? static_cast<const T *>(a.state0) + (int64_t)row * (W - 1) * a.C + ch : nullptr;
    T *s1 = static_cast<T *>(a.state1) + (int64_t)row * (W - 1) * a.C + ch;
    Raw8<T> raw[W - 1];
#pragma unroll
    for (int i = 0; i < W - 1; ++i) {
        if (from[i] >= 0)
            raw[i] = load_raw8(x + (int64_t)from[i] * a.x_stride);
        else
            raw[i] = s0 ? load_raw8(s0 + (int64_t)(n + i) * a.C) : Raw8<T>{};
    }
#pragma unroll
    for (int i = 0; i < W - 1; ++i)
        store_raw8<false, true>(s1 + (int64_t)i * a.C, raw[i]);
}

namespace {

template <typename F>
void with_width(int width, F &&f)
{
    if (width == 4)
        f.template operator()<4>();
    else if (width == 3)
        f.template operator()<3>();
    else
        f.template operator()<2>();
}
template <typename F>
void with_taps(int dtype, int width, F &&f)
{
    with_width(width, [&]<int W>() {
        if (dtype == KVB_F32)
            f.template operator()<float, W>();
        else if (dtype == KVB_BF16)
            f.template operator()<bf16_t, W>();
        else
            f.template operator()<f16_t, W>();
    });
}

}  // namespace

void launch_conv(int dtype, int width, const ConvArgs &a, hipStream_t stream)
{
    // x past the caches where it and what is made from it fill half of the last level: what reads the results next finds more of them there.  us with the
    // kvb_scan behind it, plain / past them: 300 tokens 38.2 / 38.9, 1024 84.7 / 85.2, 4096 (64 MiB) 286.3 / 286.0, 8191 576 / 571, 24 sequences of 750 562 / 558.  Not
    // in fp32, where a lane's 32 bytes are two loads that a line has to stay for: 3 x 2048 tokens 96.7 / 89.7 without.
    // Above 100 MiB (with the results more than the last level has) memory does less for more waves: LARGE in six rounds / the others in four: 3000 tokens
    // 25.6 / 23.4, 24 sequences of up to 1500, 4 + 8 heads (71 MiB) 36.0 / 34.7, 5500 (86 MiB) 39.1 / 37.9, 6200 45.3 / 44.9, 7000 (109 MiB) 51.0 / 53.8, 8191 58.8 / 62.3.
    const int each = conv_groups(a.C) + a.gates;
    const int64_t bytes = (int64_t)a.n_tokens * a.C * (dtype == KVB_F32 ? 4 : 2);
    const bool stream_x = bytes > 64 << 20, large = bytes > 100 << 20;
    const ConvDeal deal = conv_deal(a.n_tokens, a.B, each, dtype == KVB_F32, large);
    const int units = (int)(deal.stretches * each);
    with_taps(dtype, width, [&]<typename T, int W>() {
        if constexpr (sizeof(T) == 4)
            launch_part(kvb_conv_kernel<T, W, false, false>, true, true, (units + 3) / 4, 256, stream, a, units, deal.length);
        else if (large)
            launch_part(kvb_conv_kernel<T, W, true, true>, true, true, (units + 3) / 4, 256, stream, a, units, deal.length);
        else if (stream_x)
            launch_part(kvb_conv_kernel<T, W, true, false>, true, true, (units + 3) / 4, 256, stream, a, units, deal.length);
        else
            launch_part(kvb_conv_kernel<T, W, false, false>, true, true, (units + 3) / 4, 256, stream, a, units, deal.length);
    });
}

void launch_conv_token(int dtype, int width, const ConvTokenArgs &a, hipStream_t stream)
{
    const int units = a.B * (conv_groups(a.C) + a.gates);
    with_taps(dtype, width, [&]<typename T, int W>() { launch_part(kvb_conv_token_kernel<T, W>, true, true, (units + 3) / 4, 256, stream, a, units); });
}

void launch_conv_drafts(int dtype, int width, const ConvDraftArgs &a, hipStream_t stream)
{
    const int units = a.B * (conv_groups(a.C) + a.gates);
    with_taps(dtype, width, [&]<typename T, int W>() { launch_part(kvb_conv_drafts_kernel<T, W>, true, true, units, 64 * a.T, stream, a); });
}

void launch_conv_commit(int dtype, int width, const ConvCommitArgs &a, hipStream_t stream)
{
    const int units = a.B * conv_groups(a.C);
    with_taps(dtype, width, [&]<typename T, int W>() { launch_part(kvb_conv_commit_kernel<T, W>, true, true, (units + 3) / 4, 256, stream, a, units); });
}

}  // namespace kvb_impl
