// What the kernels of kvb_scan and kvb_scan_backward share: their arguments, products on bf16 pieces, the images in which a chunk's
// keys, queries and triangular matrices stand in LDS, and the bookkeeping of ragged sequences.
//
// A sequence is cut into chunks of 64 tokens.  With c the log decays summed from the chunk's start, G_ij = exp(c_i - c_j) k_i.k_j for
// i > j and P_ij = exp(c_i - c_j) q_i.k_j for i >= j, the recurrence over a chunk that starts from the state S0 is
//     E = (1 + G beta)^-1 Y,   Y = V - exp(c) K S0          (E: what a token's value has that the state did not predict)
//     O = scale (exp(c) Q S0 + P beta E)                    S1 = exp(c_last) S0 + (exp(c_last - c) K)' beta E
// (1 + G beta)^-1 = 1 + M beta with a strictly lower triangular M that does not depend on the state or on V, so
//   kvb_scan_prep_kernel   works out M and P of all chunks side by side,
//   kvb_scan_kernel        passes the state from chunk to chunk; the columns of the state do not mix, so
//                          a wave takes 16 or 32 of them and is on its own but for the keys, queries, M and P, which the
//                          waves of a workgroup share in LDS.
//
// Precision.  All products are taken on the bf16 matrix instruction with fp32 sums, at 16 times the rate of the fp32 one.  A fp32
// factor is cut into three bf16 pieces (8 bits each: the pieces' sum is the value), a bf16 input is one piece and exact, a
// fp16 input two pieces and exact; of the products of pieces those down to 2^-16 of the largest are taken, what is left out is
// below 2^-24 of a term, the rounding of fp32.  bf16 pieces have the range of fp32, which states and
// gradients need.  An infinity becomes NaN in its pieces.
#ifndef KVB_SCAN_DEVICE_H
#define KVB_SCAN_DEVICE_H

#include "kvb_device.h"

namespace kvb_impl {

constexpr int SC = 64;                      // tokens of a chunk
constexpr int SCAN_TILES = 6;               // 16 x 32 tiles with something in them of a triangular 64 x 64 matrix
constexpr int SCAN_UNITS = SCAN_TILES * 64; // of 8 floats each: what a lane holds of a tile as the matrix instruction's first operand
constexpr int SCAN_MAT = SCAN_UNITS * 8;    // floats of a matrix's image
constexpr int SCAN_GATES = 4 * SC;          // gamma = exp(c), rest = exp(c_last - c), beta, c; behind a chunk's end beta and rest are 0

// floats of workspace for each (chunk, v-head)
constexpr int SCAN_PREP = 2 * SCAN_MAT + SCAN_GATES;

struct ScanArgs {
    const void *q, *k, *v;
    const float *g, *beta;
    const float *state0;   // or nullptr: zero
    float *state1;         // or nullptr: not wanted
    void *out;
    const int32_t *start;  // [B + 1]
    const int32_t *slot;   // or nullptr: sequence b's state is row b
    float *prep;           // [chunks][Hv][SCAN_PREP]
    int64_t q_stride, k_stride, v_stride;   // elements from a token's row to the next
    int32_t B, n_slots, n_tokens, Hk, Hv, r;
    int32_t out_wide;      // fp32 outputs (otherwise the 16-bit input type)
    float scale;
};

// Chunks are numbered so that no sums over the lengths are needed: those of sequence b start at start[b] / 64 + b.  (The next
// sequence starts at least ceil(length / 64) further on.)  Bounds that are not ascending within 0 .. n_tokens are cut off, which keeps
// every access inside: start / 64 + b + chunks - 1 <= n_tokens / 64 + B - 1.
__host__ __device__ inline int64_t scan_chunks(int64_t n_tokens, int64_t B) { return n_tokens / SC + B; }

struct Span {
    int first, len;   // of a sequence
};
__device__ __forceinline__ Span span_of(const int32_t *start, int n_tokens, int b)
{
    const int s = min(max(start[b], 0), n_tokens), e = min(max(start[b + 1], s), n_tokens);
    return Span{s, e - s};
}
__device__ __forceinline__ int first_chunk(const Span &s, int b) { return s.first / SC + b; }

// The state row of sequence b, or -1 if there is none.
__device__ __forceinline__ int state_row(const int32_t *slot, int n_slots, int b)
{
    const int s = slot ? slot[b] : b;
    return s >= 0 && s < n_slots ? s : -1;
}

struct ChunkAt {
    int b, first, n;   // n = 0: nothing there
};
// The chunk with number w; every lane of the wave calls it.
__device__ __forceinline__ ChunkAt chunk_at(const int32_t *start, int n_tokens, int B, int w)
{
    const int lane = threadIdx.x % 64;
    int before = 0;   // sequences that start at or before w
    for (int b0 = 0; b0 < B; b0 += 64) {
        const int b = min(b0 + lane, B - 1);
        const bool yes = b0 + lane < B && min(max(start[b], 0), n_tokens) / SC + b <= w;
        before += __popcll(__ballot(yes));
    }
    const int b = __builtin_amdgcn_readfirstlane(max(before - 1, 0));
    const Span s = span_of(start, n_tokens, b);
    const int c = w - first_chunk(s, b), at = c * SC;
    if (c < 0 || at >= s.len)
        return ChunkAt{b, 0, 0};
    return ChunkAt{b, s.first + at, min(SC, s.len - at)};
}

// bf16 pieces of an input value, and the most that any fp32 value is cut into
template <typename T>
constexpr int PIECES = __is_same(T, bf16_t) ? 1 : __is_same(T, f16_t) ? 2 : 3;
constexpr int FULL = 3;

// Eight values in N pieces, to nearest: each piece has 8 bits of what the ones before left.
template <int N>
__device__ __forceinline__ void cut8(const float (&x)[8], uint4 (&p)[N])
{
    float rest[8];
#pragma unroll
    for (int j = 0; j < 8; ++j)
        rest[j] = x[j];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        uint32_t w[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            w[j] = pack_pair<bf16_t>(rest[2 * j], rest[2 * j + 1]);
            rest[2 * j] -= __uint_as_float(w[j] << 16);
            rest[2 * j + 1] -= __uint_as_float(w[j] & 0xFFFF0000u);
        }
        p[i] = make_uint4(w[0], w[1], w[2], w[3]);
    }
}
template <typename T>
__device__ __forceinline__ void cut_raw(const Raw8<T> &r, uint4 (&p)[PIECES<T>])
{
    if constexpr (__is_same(T, bf16_t)) {
        p[0] = r.w;
    } else {
        float x[8];
        unpack8(r, x);
        cut8(x, p);
    }
}

// c += a b on their pieces (the products that are left out are below 2^-24)
template <int NA, int NB>
__device__ __forceinline__ void mma(f32x4_t &c, const uint4 (&a)[NA], const uint4 (&b)[NB])
{
#pragma unroll
    for (int i = 0; i < NA; ++i)
#pragma unroll
        for (int j = 0; j < NB; ++j)
            if (i + j < FULL)
                c = mfma16x32<bf16_t>(a[i], b[j], c);
}

// Operand layouts of v_mfma_f32_16x16x32: lane l holds row (first operand) or column (second) l % 16 and of the 32 that are summed
// over the 8 that belong to l / 16; a sum has column l % 16 in lane l and rows 4 (l / 16) + 0..3 in its four registers.  The order of
// what is summed over is free as long as both operands share it.  So 32 rows of a sum, two tiles of it, become a second
// operand without a move between lanes: lane group g then holds rows 4g .. 4g+3 of the first tile and of the second, and the first
// operand has its columns in that order: 4g .. 4g+3 and 16 + 4g .. 16 + 4g + 3 for group g.  "Paired order" below.
__device__ __forceinline__ void pair8(const f32x4_t &a, const f32x4_t &b, float (&x)[8])
{
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        x[r] = a[r];
        x[4 + r] = b[r];
    }
}

// A chunk's 64 x D keys (or queries) in LDS: piece, 16-token tile, 32-column step, lane, 16 bytes, in paired order.
// loaded: by the workgroup's waves in turns of a (tile, step), 16 bytes (of a 16-bit type) a lane.
template <typename T, int D, int NWV>
struct TokenTile {
    static constexpr int STEPS = D / 32, N = 4 * STEPS / NWV, NP = PIECES<T>, WORDS = NP * 4 * STEPS * 64;
    static_assert(4 * STEPS % NWV == 0);
    Raw8<T> x[N];
    __device__ __forceinline__ void load(const T *rows, int64_t stride, int n, int wave, int lane)
    {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int u = wave + NWV * i, row = min(16 * (u / STEPS) + lane % 16, n - 1);
            x[i] = load_raw8(rows + row * stride + 32 * (u % STEPS) + 8 * (lane / 16));
        }
    }
    __device__ __forceinline__ void store(uint4 *img, int wave, int lane) const
    {
        // a lane's eight columns are two runs of four, which belong to neighbouring lane groups
        const int g = lane / 16, at = (2 * g % 4) * 16 + lane % 16, half = g / 2;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int u = wave + NWV * i;
            uint4 p[NP];
            cut_raw(x[i], p);
#pragma unroll
            for (int j = 0; j < NP; ++j) {
                uint2 *to = reinterpret_cast<uint2 *>(img + (j * 4 * STEPS + u) * 64 + at) + half;
                to[0] = make_uint2(p[j].x, p[j].y);
                to[32] = make_uint2(p[j].z, p[j].w);
            }
        }
    }
    // rows of tokens as the first operand: tile rt, columns 32 ks ..
    static __device__ __forceinline__ void rows(const uint4 *img, int rt, int ks, int lane, uint4 (&a)[NP])
    {
#pragma unroll
        for (int j = 0; j < NP; ++j)
            a[j] = img[((j * 4 + rt) * STEPS + ks) * 64 + lane];
    }
    // the transpose: rows are columns 16 mt .. of the tile, summed over tokens 32 s .. in paired order (ds_read_b64_tr_b16: each 16
    // lanes read four rows of 16 and get a column of four each)
    static __device__ __forceinline__ void columns(const uint4 *img, int mt, int s, int lane, uint4 (&a)[NP])
    {
        typedef short v4s __attribute__((ext_vector_type(4)));
        typedef __attribute__((address_space(3))) v4s *Lds;
        const int at = (lane % 4) * 16 + 4 * (lane / 16) + lane % 16 / 4;
#pragma unroll
        for (int j = 0; j < NP; ++j) {
            const uint4 *p = img + ((j * 4 + 2 * s) * STEPS + mt / 2) * 64 + at;
            const v4s lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)(reinterpret_cast<const uint2 *>(p) + mt % 2));
            const v4s hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)(reinterpret_cast<const uint2 *>(p + STEPS * 64) + mt % 2));
            const uint2 l = __builtin_bit_cast(uint2, lo), h = __builtin_bit_cast(uint2, hi);
            a[j] = make_uint4(l.x, l.y, h.x, h.y);
        }
    }
};

// Images of triangular matrices: tile (16 rows rt, 32 columns s) has number tile_of(rt, s); in LDS three pieces of it, 16 bytes a lane.
template <bool UPPER>
__host__ __device__ constexpr int tile_of(int rt, int s)
{
    return UPPER ? (rt < 2 ? 2 * rt + s : 2 + rt) : (rt < 2 ? rt : 2 * rt - 2 + s);
}
template <bool UPPER>
__host__ __device__ constexpr bool has_tile(int rt, int s) { return UPPER ? rt < 2 || s == 1 : rt >= 2 || s == 0; }

// N units of 8 floats from a workspace into pieces in LDS, by all NTH threads of the workgroup
template <int N, int NTH>
struct MatTile {
    static constexpr int EACH = (N + NTH - 1) / NTH;
    Raw8<float> x[EACH];
    __device__ __forceinline__ void load(const float *img, int tid)
    {
#pragma unroll
        for (int i = 0; i < EACH; ++i)
            if (N % NTH == 0 || tid + NTH * i < N)
                x[i] = load_raw8(img + (tid + NTH * i) * 8);
    }
    __device__ __forceinline__ void store(uint4 *to, int tid) const
    {
#pragma unroll
        for (int i = 0; i < EACH; ++i)
            if (N % NTH == 0 || tid + NTH * i < N) {
                float f[8];
                uint4 p[FULL];
                unpack8(x[i], f);
                cut8(f, p);
#pragma unroll
                for (int j = 0; j < FULL; ++j)
                    to[j * N + tid + NTH * i] = p[j];
            }
    }
    static __device__ __forceinline__ void tile(const uint4 *img, int t, int lane, uint4 (&a)[FULL])
    {
#pragma unroll
        for (int j = 0; j < FULL; ++j)
            a[j] = img[j * N + t * 64 + lane];
    }
};

// One kernel of a call that makes several; an armed timer spans them from the first one's start to the last one's end.
template <typename... Params, typename... Args>
void launch_part(void (*kernel)(Params...), bool first, bool last, int64_t blocks, int threads, hipStream_t stream, const Args &...a)
{
    static_assert(sizeof...(Params) == sizeof...(Args), "one argument per kernel parameter");
    if (g_launch_status != hipSuccess)
        return;
    std::tuple<std::remove_cv_t<Params>...> params{a...};
    void *argv[sizeof...(Params)];
    std::apply([&](auto &...p) { int i = 0; ((argv[i++] = &p), ...); }, params);
    kvb_timer *t = g_armed;
    if (t && (first || last))
        g_launch_status = hipExtLaunchKernel(reinterpret_cast<const void *>(kernel), dim3((uint32_t)blocks), dim3(threads), argv, 0, stream,
                                             first ? t->start : nullptr, last ? t->stop : nullptr, 0);
    else
        g_launch_status = hipLaunchKernel(reinterpret_cast<const void *>(kernel), dim3((uint32_t)blocks), dim3(threads), argv, 0, stream);
    if (last)
        g_armed = nullptr;
}

// one unit per input type (kvb_scan_*.hip)
template <typename TIn>
void launch_scan_typed(int d, const ScanArgs &a, hipStream_t stream);

}  // namespace kvb_impl
#endif  // KVB_SCAN_DEVICE_H
