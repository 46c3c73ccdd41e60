// What the kernels around the recurrence share (kvb_conv.hip, kvb_conv_grad_*.hip, kvb_norm.hip, kvb_norm_grad.hip, kvb_clip.hip): their
// arguments, sums over neighbouring lanes, pieces of ragged sequences, sums of columns.
#ifndef KVB_LAYER_DEVICE_H
#define KVB_LAYER_DEVICE_H

#include "kvb_scan_device.h"

namespace kvb_impl {

// ---------------------------------------------------------------------------
// arguments
// ---------------------------------------------------------------------------
struct ConvArgs {
    const void *x, *a, *b;            // rows of C, Hv and Hv elements
    const void *weight, *bias;        // [C][width], [C] or nullptr
    const float *A_log, *dt_bias;     // [Hv]
    const void *state0;               // [n_slots][width - 1][C] or nullptr: zero
    void *state1;                     // the same, or nullptr: not wanted
    void *q, *k, *v;
    float *g, *beta;                  // [n_tokens][Hv]
    const int32_t *start, *slot;      // whole sequences: [B + 1]; [B] or nullptr
    const int32_t *parent;            // drafts: [B][T] or nullptr: a chain
    const int32_t *path, *accepted;   // commit: [B][T] or nullptr: 0, 1, ..; [B]
    int64_t x_stride, a_stride, b_stride, q_stride, k_stride, v_stride;
    int32_t B, T, n_slots, n_tokens, Hk, Hv, d, C;
    int32_t gates, unit;              // whether there are gates; whether q and k get length one
    float eps;
};

struct ConvGradArgs {
    ConvArgs f;                       // (what it writes is not used)
    const void *dq, *dk, *dv;         // strides of q, k, v
    const float *dg, *dbeta;          // [n_tokens][Hv]
    const void *dstate1;              // or nullptr: zero
    void *dx, *da, *db;               // strides of x, a, b
    void *dstate0;                    // or nullptr: not wanted
    float *part;                      // [parts][columns]
    int32_t parts, each, columns;     // chunks of a wave; columns of a part: width and bias planes of C, then dA_log and ddt_bias
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
__device__ __forceinline__ float sum_lanes(float x, int lg)   // lg 2..6
{
    x = sum_to16(x, lg);
    if (lg > 4)
        x += __shfl_xor(x, 16);
    if (lg > 5)
        x += __shfl_xor(x, 32);
    return x;
}

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
template <typename T>
__device__ __forceinline__ void store8(T *p, const float (&x)[8]) { store_raw8<false, true>(p, pack8<T>(x)); }

// A stretch of 2^lg tokens of a ragged batch, numbered as the chunks of a scan are: those of sequence b start at start[b] / 2^lg + b, so that
// every sequence has one, an empty one too.
struct Piece {
    int b, first, len;   // the sequence, its first token, its length
    int t0, t1;          // the tokens of the piece, counted from there; t0 = t1 in an empty sequence's only one
    bool some;           // false: there is no piece with this number
};
inline int64_t pieces_of(int64_t n_tokens, int64_t B, int lg) { return (n_tokens >> lg) + B; }
__device__ __forceinline__ Piece piece_at(const int32_t *start, int n_tokens, int B, int w, int lg)   // every lane of the wave calls it
{
    const int lane = threadIdx.x % 64;
    int before = 0;   // sequences that start at or before w
    for (int b0 = 0; b0 < B; b0 += 64) {
        const int b = min(b0 + lane, B - 1);
        const bool yes = b0 + lane < B && (min(max(start[b], 0), n_tokens) >> lg) + b <= w;
        before += __popcll(__ballot(yes));
    }
    const int b = __builtin_amdgcn_readfirstlane(max(before - 1, 0));
    const Span s = span_of(start, n_tokens, b);
    const int c = w - ((s.first >> lg) + b);
    const int64_t at = (int64_t)c << lg;
    if (c < 0 || (c > 0 && at >= s.len))
        return Piece{b, s.first, s.len, 0, 0, false};
    return Piece{b, s.first, s.len, (int)at, min(s.len, (int)at + (1 << lg)), true};
}

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

// Sums of columns over `parts` rows, in a fixed order.  Columns from begin[i] on go to to[i], whose last one may be followed by more ranges.
struct SumsTo {
    float *to[4];
    int64_t begin[4];
};
void launch_sums(const float *part, int parts, int64_t columns, const SumsTo &to, hipStream_t stream);   // kvb_norm_grad.hip; ends a call, parts = 0: is it

// (in_dtype and width are checked by the caller)
void launch_conv(int in_dtype, int width, const ConvArgs &a, hipStream_t stream);          // kvb_conv.hip
void launch_conv_tokens(int in_dtype, int width, const ConvArgs &a, hipStream_t stream);
void launch_conv_commit(int in_dtype, int width, const ConvArgs &a, hipStream_t stream);
template <typename T>
void launch_conv_grad_typed(int width, const ConvGradArgs &a, int lg, float *dweight, float *dbias, float *dA_log, float *ddt_bias,
                            hipStream_t stream);                                            // kvb_conv_grad_*.hip
template <typename TX, typename T>
void launch_norm_typed(const NormArgs &a, hipStream_t stream);                              // kvb_norm.hip
template <typename TX, typename T>
void launch_norm_grad_typed(const NormGradArgs &a, float *dweight, hipStream_t stream);     // kvb_norm_grad.hip
void launch_grad_norm(const ListArgs &a, float *norm, double *work, hipStream_t stream);    // kvb_clip.hip
void launch_clip(const ListArgs &a, const float *norm, float largest, hipStream_t stream);

// Chunks of the gradients of the convolution, 2^lg tokens each, and how many a wave takes: a workgroup's four waves leave one part, at most
// CONV_PARTS of them.
constexpr int CONV_PARTS = 256;
constexpr int CONV_LEAST_LG = 3;   // (more than the taps reach back)
struct ConvParts {
    int lg, parts, each;
};
inline ConvParts conv_parts(int64_t n_tokens, int64_t B, int)
{
    const int lg = 5;
    const int64_t pieces = pieces_of(n_tokens, B, lg), each = (pieces + 4 * CONV_PARTS - 1) / (4 * CONV_PARTS);
    const int64_t e = each < 1 ? 1 : each;
    return ConvParts{lg, (int)((pieces + 4 * e - 1) / (4 * e)), (int)e};
}

// The most that a call of up to so many tokens and sequences needs
inline int64_t conv_most_parts(int64_t n_tokens, int64_t B)
{
    const int64_t n = (pieces_of(n_tokens, B, CONV_LEAST_LG) + 3) / 4;
    return n < 1 ? 1 : n < CONV_PARTS ? n : CONV_PARTS;
}

// Workgroups of kvb_norm_backward, each of which leaves one part.
constexpr int NORM_PARTS = 1024;
inline int norm_parts(int64_t rows, int width)
{
    int64_t rows_of_workgroup = 1;   // at once
    if (width <= 2048) {
        int lanes = 4;
        while (lanes < 64 && lanes * 8 < width)
            lanes *= 2;
        rows_of_workgroup = 256 / lanes;
    }
    const int64_t n = (rows + rows_of_workgroup - 1) / rows_of_workgroup;
    return (int)(n < NORM_PARTS ? n : NORM_PARTS);
}
inline int64_t norm_most_parts(int64_t rows, int width) { return norm_parts(rows, width); }

}  // namespace kvb_impl
#endif  // KVB_LAYER_DEVICE_H
