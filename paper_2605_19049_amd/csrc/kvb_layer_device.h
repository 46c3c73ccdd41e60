// What the kernels around the recurrence share (kvb_conv.hip, kvb_conv_grad_*.hip, kvb_norm.hip, kvb_norm_grad.hip, kvb_clip.hip): their
// arguments, sums over neighbouring lanes, shares of ragged sequences, sums of columns.
#ifndef KVB_LAYER_DEVICE_H
#define KVB_LAYER_DEVICE_H

#include "kvb_scan_device.h"

namespace kvb_impl {

// ---------------------------------------------------------------------------
// arguments
// ---------------------------------------------------------------------------
// (A kernel's first loads are its arguments: each form of the convolution has no more than it needs.  128 x 4 drafts with their commit, 250 bytes / 180: 13.3 / 12.5 us.)
struct ConvBase {
    const void *x, *a, *b;            // rows of C, Hv and Hv elements
    const void *weight, *bias;        // [C][width], [C] or nullptr
    const float *A_log, *dt_bias;     // [Hv]
    const void *state0;               // [n_slots][width - 1][C] or nullptr: zero
    void *q, *k, *v;
    float *g, *beta;                  // [n_tokens][Hv]
    const int32_t *slot;              // [B], or nullptr for whole sequences: row b
    int64_t x_stride, a_stride, b_stride;
    int32_t B, n_slots, Hk, Hv, d, C;
    int16_t gates, unit;              // whether there are gates; whether q and k get length one
    float eps;
};
struct ConvTokenArgs : ConvBase {
    void *state1;                     // as state0, or nullptr: not wanted
};
struct ConvDraftArgs : ConvBase {
    const int32_t *parent;            // [B][T] or nullptr: a chain
    int32_t T;
};
struct ConvArgs : ConvTokenArgs {
    const int32_t *start;             // [B + 1]
    int64_t q_stride, k_stride, v_stride;
    int32_t n_tokens;
};
struct ConvCommitArgs {
    const void *x, *state0;
    void *state1;
    const int32_t *slot, *path, *accepted;   // path: [B][T] or nullptr: 0, 1, ..
    int64_t x_stride;
    int32_t B, T, n_slots, C;
};

struct ConvGradArgs {
    ConvArgs f;                       // (what it writes is not used)
    const void *dq, *dk, *dv;         // strides of q, k, v
    const float *dg, *dbeta;          // [n_tokens][Hv]
    const void *dstate1;              // or nullptr: zero
    void *dx, *da, *db;               // strides of x, a, b
    void *dstate0;                    // or nullptr: not wanted
    float *part;                      // [parts][columns]
    int32_t parts, columns;           // columns of a part: width and bias planes of C, then dA_log and ddt_bias
};

struct NormArgs {
    const void *x, *res, *gate, *weight;   // res, gate or nullptr
    void *sum, *out;                       // sum or nullptr
    int64_t x_stride, gate_stride;
    int64_t rows;                          // tokens * heads
    int32_t heads, width;
    float eps, scale;
};

struct NormGradArgs {
    NormArgs f;                        // x: what the norm was taken of
    const void *dout, *dsum;           // dsum or nullptr
    void *dx, *dres, *dgate;           // strides of x, packed, of gate; dres, dgate or nullptr
    float *part;                       // [parts][width]
    int32_t parts;
    float dx_scale;
};

struct ListArgs {
    void *const *data;       // [n]
    void *const *to;         // clip: [n]
    const int64_t *size;     // [n]
    const int32_t *type;     // [n]
    const int32_t *first;    // [n + 1]
    int32_t n, blocks;
};

// ---------------------------------------------------------------------------
// device helpers
// ---------------------------------------------------------------------------
// Sums over groups of 2^lg neighbouring lanes (lg a scalar), for all of them.  Up to 16 lanes it goes by the permutations that an addition can
// read through: neighbours, pairs, the mirror images in half a row and in a row of 16.
template <int CTRL>
__device__ __forceinline__ float add_lane(float x)
{
    return x + __uint_as_float(__builtin_amdgcn_update_dpp(0u, __float_as_uint(x), CTRL, 0xF, 0xF, false));
}
__device__ __forceinline__ float sum_to16(float x, int lg)   // lg 2..4
{
    x = add_lane<0x4E>(add_lane<0xB1>(x));
    const float y = add_lane<0x141>(x);
    x = lg > 2 ? y : x;
    const float z = add_lane<0x140>(x);
    return lg > 3 ? z : x;
}
__device__ __forceinline__ float sum_to32(float x, int lg)   // lg 3..5
{
    x = sum_to16(x, lg < 4 ? lg : 4);
    const auto rows = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);   // rows 0, 0, 2, 2 and 1, 1, 3, 3
    const float y = __uint_as_float(rows[0]) + __uint_as_float(rows[1]);
    return lg > 4 ? y : x;
}
__device__ __forceinline__ float sum_lanes(float x, int lg)   // lg 2..6
{
    x = sum_to16(x, lg);
    if (lg > 4)
        x += __shfl_xor(x, 16);
    if (lg > 5)
        x += __shfl_xor(x, 32);
    return x;
}

// (rows are at most 2^31 - 1: a division in 32 bits)
__device__ __forceinline__ int64_t token_of(const NormArgs &a, int64_t row) { return a.heads == 1 ? row : (int64_t)((uint32_t)row / (uint32_t)a.heads); }

// 1 / (1 + exp(-z))
__device__ __forceinline__ float sigmoid(float z) { return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-1.442695041f * z)); }

template <typename T>
__device__ __forceinline__ Raw8<T> pack8(const float (&x)[8])
{
    if constexpr (sizeof(T) == 4)
        return Raw8<T>{make_float4(x[0], x[1], x[2], x[3]), make_float4(x[4], x[5], x[6], x[7])};
    else
        return Raw8<T>{make_uint4(pack_pair<T>(x[0], x[1]), pack_pair<T>(x[2], x[3]), pack_pair<T>(x[4], x[5]), pack_pair<T>(x[6], x[7]))};
}
// V elements (8 or 4), raw and converted
template <int V, typename T>
__device__ __forceinline__ auto load_raw(const T *p)
{
    if constexpr (V == 8)
        return load_raw8(p);
    else
        return load_raw4(p);
}
template <typename T>
__device__ __forceinline__ void unpack(const Raw8<T> &r, float (&o)[8]) { unpack8(r, o); }
template <typename T>
__device__ __forceinline__ void unpack(const Raw4<T> &r, float (&o)[4])
{
    const float4 x = unpack4(r);
    o[0] = x.x, o[1] = x.y, o[2] = x.z, o[3] = x.w;
}

// 8 elements that are not read again: past the caches
__device__ __forceinline__ Raw8<float> load_raw8_nt(const float *p)
{
    typedef float v4 __attribute__((ext_vector_type(4)));
    const v4 a = __builtin_nontemporal_load(reinterpret_cast<const v4 *>(p)), b = __builtin_nontemporal_load(reinterpret_cast<const v4 *>(p + 4));
    return Raw8<float>{make_float4(a.x, a.y, a.z, a.w), make_float4(b.x, b.y, b.z, b.w)};
}
template <typename T>
__device__ __forceinline__ Raw8<T> load_raw8_nt(const T *p)
{
    typedef uint32_t v4 __attribute__((ext_vector_type(4)));
    const v4 a = __builtin_nontemporal_load(reinterpret_cast<const v4 *>(p));
    return Raw8<T>{make_uint4(a.x, a.y, a.z, a.w)};
}

template <bool STREAM, typename T>
__device__ __forceinline__ Raw8<T> load_raw8_if(const T *p)
{
    if constexpr (STREAM)
        return load_raw8_nt(p);
    else
        return load_raw8(p);
}
// Results are left in the caches by plain stores: what comes next reads them.  us, kvb_conv of 8191 tokens (bf16, 16 + 32 heads of 128) with plain
// stores / past the caches 59.7 / 55.3 alone, 576 / 585 with the kvb_scan that reads them; 24 sequences of 750 in all 562 / 572; kvb_norm, 18000 x 32 heads of 128,
// gated, 88 / 84 alone, 405 / 416 with the matrix product that reads it.  Through the L2 as they are made (put): 66.6; kvb_norm_backward 137 instead of 98.
// STREAM: past them all the same, for what would push out what is read again (kvb_clip).
template <bool STREAM = false, typename T>
__device__ __forceinline__ void store8(T *p, const float (&x)[8]) { store_raw8<STREAM, !STREAM>(p, pack8<T>(x)); }

template <typename T>
__device__ __forceinline__ void store_values(T *p, const float (&x)[8]) { store8(p, x); }
template <typename T>
__device__ __forceinline__ void store_values(T *p, const float (&x)[4]) { store4<false, true>(p, make_float4(x[0], x[1], x[2], x[3])); }

// A ragged batch laid out by what it costs: sequence b takes the places start[b] + SEQUENCE b up to start[b + 1] + SEQUENCE (b + 1), the first SEQUENCE of them
// for itself (its bounds, its row of the states and the inputs ahead of it, asked for one after the other), then one a token.  A stretch of
// these places is a part of one sequence, or whole ones and a part of one at either end; each wave has one.
// us, against pieces of one sequence each (numbered start[b] / length + b, so that some numbers were nobody's), 1000 sequences of up to 20 tokens, 4 + 8 heads, kvb_conv 34.8 / 31.2,
// kvb_conv_backward 72.6 / 58.2; 200 of up to 64, 8 + 16 heads, 32.0 / 31.0 and 102.7 / 54.6; 24 of up to 1500, 4 + 8 heads, 36.3 / 36.7; one of 8191, 16 + 32 heads, 58.9 / 58.6;
// 4 of 2048, backward, 97.2 / 97.4.  SEQUENCE 4 / 6 / 12: backward, 200 sequences 53.1 / 52.9 / 56.6, 4 of 2048 98.3 / 98.3 / 96.4; 24 of up to 1500 37.9 / 37.1.
constexpr int SEQUENCE = 8;
inline int64_t places_of(int64_t n_tokens, int64_t B) { return n_tokens + SEQUENCE * B; }
__device__ __forceinline__ int64_t place_of(const int32_t *start, int n_tokens, int b) { return min(max(start[b], 0), n_tokens) + (int64_t)SEQUENCE * b; }
// The sequence that has the place, or the one before it
__device__ __forceinline__ int sequence_at(const int32_t *start, int n_tokens, int B, int64_t place)   // every lane of the wave calls it
{
    // 64 candidates at a time, a 64th of what is left apart, then neighbours
    const int lane = threadIdx.x % 64;
    int b = 0, step = 1;
    while ((int64_t)step * 64 < B)
        step *= 64;
    for (; step > 0; step /= 64) {
        const int64_t at = b + (int64_t)lane * step;   // (lane 0's is known to begin, or is sequence 0)
        const bool yes = at < B && place_of(start, n_tokens, (int)at) <= place;
        b += max((int)__popcll(__ballot(yes)) - 1, 0) * step;
    }
    return __builtin_amdgcn_readfirstlane(b);
}
// What some places have of a sequence
struct Share {
    int first, len, row;   // its first token, its length, its row of the states
    int t0, t1;            // the tokens, counted from there; t0 = t1 in an empty sequence, which is where it begins
    bool some;             // false: nothing (no token, a skipped sequence)
};
// One after the other; as one is taken the bounds and the slot of the next are asked for.  Where two waves share a sequence the first one has `least` tokens of it or
// all: a state reaches no further than that, so that who has t0 = 0 alone reads and writes it.
struct Shares {
    const int32_t *start, *slot;
    int n_tokens, n_slots, B;
    int64_t from, to;
    int b, least, bound, next_bound, next_row;   // the next sequence; tokens of its first part at least; its bounds and its row
    // (every lane of the wave calls it)
    __device__ __forceinline__ Shares(const ConvArgs &a, int64_t from, int64_t to, int least)
        : start(a.start), slot(a.slot), n_tokens(a.n_tokens), n_slots(a.n_slots), B(a.B), from(from), to(to), b(sequence_at(a.start, a.n_tokens, a.B, from)), least(least)
    {
        bound = __builtin_amdgcn_readfirstlane(start[b]);
        ask();
    }
    __device__ __forceinline__ void ask()   // (b < B)
    {
        next_bound = __builtin_amdgcn_readfirstlane(start[b + 1]);
        next_row = __builtin_amdgcn_readfirstlane(slot ? slot[b] : b);
    }
    __device__ __forceinline__ bool more() const { return b < B && min(max(bound, 0), n_tokens) + (int64_t)SEQUENCE * b < to; }
    __device__ __forceinline__ Share take()
    {
        const int first = min(max(bound, 0), n_tokens), len = min(max(next_bound, first), n_tokens) - first, row = next_row;
        const int64_t begin = first + (int64_t)SEQUENCE * b, token = begin + SEQUENCE;
        auto cut = [&](int64_t t) { return t <= 0 ? 0 : (int)min(max(t, (int64_t)least), (int64_t)len); };
        const int t0 = cut(from - token), t1 = cut(to - token);
        const bool some = row >= 0 && row < n_slots && (t0 < t1 || (len == 0 && begin >= from));
        bound = next_bound;
        if (++b < B)
            ask();
        return Share{first, len, row, t0, t1, some};
    }
};

// The gates of some tokens and heads, dealt over a wave: lane -> (token, head), heads in the next power of two of lanes.
struct GateLanes {
    int heads, tokens;   // lanes that a token's heads take (at most 64), tokens side by side
    int head, token;     // the lane's
};
__device__ __forceinline__ GateLanes gate_lanes(int Hv, int lane)
{
    int heads = 1;
    while (heads < Hv && heads < 64)
        heads *= 2;
    return GateLanes{heads, 64 / heads, lane % heads, lane / heads};
}
__device__ __forceinline__ float softplus(float y) { return fmaxf(y, 0.0f) + log1pf(expf(-fabsf(y))); }

// ---------------------------------------------------------------------------
// launchers
// ---------------------------------------------------------------------------
constexpr int CONV_LANES = 512;   // channels of a wave: 8 a lane
__host__ __device__ constexpr int conv_groups(int C) { return (C + CONV_LANES - 1) / CONV_LANES; }

// kvb_conv_backward: 16 bytes a lane.  us, fp32, 4 / 8 channels a lane: 3 x 2048 tokens, 16 + 32 heads of 128, 135 / 138; 5 x up to 150, 2 + 4 heads of 64, 9.1 / 10.7; 700 tokens,
// 4 + 8 heads of 128, 12.9 / 14.6; 2 x 6000, 8 + 16 heads, W = 2, 127 / 132 (2 x 5000, 8 + 8 heads, 92 / 86).  bf16: 4 x 2048 tokens 100 / 97, 4 x 4096 185 / 181, 200 x up to 64 88 / 102.
template <typename T>
constexpr int GRAD_CHANNELS = 16 / (int)sizeof(T);
__host__ __device__ constexpr int grad_groups(int C, int channels) { return (C + 64 * channels - 1) / (64 * channels); }

// Sums of columns over `parts` rows, in a fixed order.  Columns from begin[i] on go to to[i], whose last one may be followed by more ranges.
struct SumsTo {
    float *to[4];
    int64_t begin[4];
};
void launch_sums(const float *part, int parts, int64_t columns, const SumsTo &to, hipStream_t stream);   // kvb_norm_grad.hip; ends a call, parts = 0: is it

// (in_dtype and width are checked by the caller)
void launch_conv(int in_dtype, int width, const ConvArgs &a, hipStream_t stream);          // kvb_conv.hip
void launch_conv_token(int in_dtype, int width, const ConvTokenArgs &a, hipStream_t stream);
void launch_conv_drafts(int in_dtype, int width, const ConvDraftArgs &a, hipStream_t stream);
void launch_conv_commit(int in_dtype, int width, const ConvCommitArgs &a, hipStream_t stream);
template <typename T>
void launch_conv_grad_typed(int width, const ConvGradArgs &a, int64_t length, float *dweight, float *dbias, float *dA_log, float *ddt_bias,
                            hipStream_t stream);                                            // kvb_conv_grad_*.hip
template <typename TX, typename T>
void launch_norm_typed(const NormArgs &a, hipStream_t stream);                              // kvb_norm.hip
template <typename TX, typename T>
void launch_norm_grad_typed(const NormGradArgs &a, float *dweight, hipStream_t stream);     // kvb_norm_grad.hip
void launch_grad_norm(const ListArgs &a, float *norm, double *work, hipStream_t stream);    // kvb_clip.hip
void launch_clip(const ListArgs &a, const float *norm, float largest, hipStream_t stream);

// Places of a wave: as many as make the workgroups of four waves come out as `rounds` for each compute unit at most, the fewest with which they are no more than 16:
// what starts behind others runs alone, and few tokens pay for their weights and the inputs ahead of them.  units: waves of a stretch.
// us, kvb_conv, 16 + 32 heads of 128, bf16, W = 4, enough 8 / 16: 1000 tokens 11.8 / 11.6, 2000 19.0 / 16.7; 8191 tokens in 4 rounds 66, 5 59.1, 6 59.2, 7 61.3,
// 9 60.1; 200 sequences of up to 64, 8 + 16 heads, in 3 29.9, 4 28.8, 5 32.1, 8 32.4; fp32, 5284 tokens, W = 3, in 3 80.8, 4 84.4, 6 83.9.  kvb_conv_backward, bf16: 4 x 2048 tokens in 1.75 rounds 115, 2 104, 4 112;
// fp32, 3 x 2048 tokens in 2 147, 3 135, 4 139.
constexpr int CONV_LEAST = 4;   // places of a wave at least
inline int64_t conv_length(int64_t places, int units, int rounds)
{
    int64_t length = INT64_MAX;
    for (int k = 1; k <= rounds && length > 16; ++k) {
        const int64_t most = 256 * k / units * 4, waves = most < 4 ? 4 : most;
        length = (places + waves - 1) / waves;
    }
    return length < CONV_LEAST ? CONV_LEAST : length;
}
struct ConvDeal {
    int64_t length, stretches;
};
inline ConvDeal conv_deal(int64_t n_tokens, int64_t B, int units, bool wide, bool large)
{
    const int64_t places = places_of(n_tokens, B), most = conv_length(places, units, wide ? 3 : large ? 6 : 4), length = most < 64 ? most : 64;
    return ConvDeal{length, (places + length - 1) / length};
}
struct ConvParts {
    int64_t length;
    int parts;   // a workgroup's four waves leave one
};
// kvb_conv_backward, by the figures above.  In 16 bits two is what the registers leave a SIMD (W = 2 without a bias: three); in fp32, with half as many channels a wave, they
// leave four (W = 4 with a bias: three), and three rounds are faster than four all the same.
constexpr int grad_rounds(bool wide) { return wide ? 3 : 2; }
inline int64_t conv_part_limit(int units, bool wide) { return 256 * grad_rounds(wide) / units < 1 ? 1 : 256 * grad_rounds(wide) / units; }
inline ConvParts conv_parts(int64_t n_tokens, int64_t B, int units, bool wide)
{
    if (B == 0)   // (tokens of nobody)
        return ConvParts{CONV_LEAST, 0};
    const int64_t places = places_of(n_tokens, B), length = conv_length(places, units, grad_rounds(wide));
    return ConvParts{length, (int)((places + 4 * length - 1) / (4 * length))};
}
// The most that a call of up to so many tokens and sequences needs
inline int64_t conv_most_parts(int64_t n_tokens, int64_t B, int units, bool wide)
{
    const int64_t n = (places_of(n_tokens, B) + 4 * CONV_LEAST - 1) / (4 * CONV_LEAST), limit = conv_part_limit(units, wide);
    return n < 1 ? 1 : n < limit ? n : limit;
}

// Workgroups of a block of a list: several where the blocks alone do not fill the card
constexpr int LIST_SPLIT = 4, LIST_FULL = 512;
inline int list_split(int blocks) { return blocks < LIST_FULL ? LIST_SPLIT : 1; }
// The most sums that a list of up to so many blocks leaves, one a workgroup: what the longest split list does, where that is more
inline int64_t list_most_sums(int64_t blocks)
{
    const int64_t split = LIST_SPLIT * (blocks < LIST_FULL ? blocks : LIST_FULL - 1);
    return blocks > split ? blocks : split;
}
static_assert(KVB_LIST_BLOCK % (LIST_SPLIT * 8) == 0);

// kvb_norm_backward, rows above 512 elements: vectors of 8 that a lane has of a row, threads of a row, rows of a workgroup at once
inline int norm_vectors(int width) { return width <= 4096 ? 1 : width <= 8192 ? 2 : 4; }
inline int norm_threads(int width) { return ((width / 8 + norm_vectors(width) - 1) / norm_vectors(width) + 63) / 64 * 64; }
inline int norm_teams(int width) { return 512 / norm_threads(width); }
// Turns that rows take if each is a workgroup's
inline int64_t norm_turns(int64_t rows, int width)
{
    int64_t at_once = norm_teams(width);
    if (width <= 512) {
        int lanes = 4;
        while (lanes < 64 && lanes * 8 < width)
            lanes *= 2;
        at_once = 256 / lanes;
    }
    return (rows + at_once - 1) / at_once;
}
// Up to so many, one workgroup takes them all and its sums are the gradient: a launch less (us, 18 rows of 128, fp32, 2 turns: 4.5 instead of 7.1; 8 rows of 2048, bf16, 4 turns:
// 7.0, 9 in two launches 7.3; 4 rows of 8192 in one 10.6).
inline int norm_few(int width) { return width <= 4096 ? 4 : 2; }
// Its workgroups, each of which leaves one part.  us with 1024 / 512, rows of up to 512 elements: 948 turns (bf16, 128 wide, gated) 13.6 / 11.9, 4000 20.7 / 24, 8000
// 39.6 / 40.9, 16384 (x in fp32) 95.6 / 91.4, 36000 153.0 / 151.8.  Longer rows: what more parts there are is as much as rows.
inline int norm_parts(int64_t rows, int width)
{
    const int64_t n = norm_turns(rows, width);
    if (n <= norm_few(width))
        return n < 1 ? 0 : 1;
    if (width > 512)
        return (int)(n < 512 ? n : 512);
    return (int)(n <= 256 ? n : n <= 1024 ? (n + 1) / 2 : n < 12288 ? 1024 : 512);
}
// The most that a call of up to so many rows needs
inline int64_t norm_most_parts(int64_t rows, int width)
{
    const int64_t n = norm_turns(rows, width), most = width > 512 ? 512 : 1024;
    return n < most ? n : most;
}

}  // namespace kvb_impl
#endif  // KVB_LAYER_DEVICE_H
