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
//                          a wave takes 16 of them and is on its own but for the keys, queries, M and P, which the
//                          waves of a workgroup share in LDS,
//   kvb_scan_token_kernel  does without chunks where there are only a few tokens a sequence.
//
// Precision.  All products are taken on the bf16 matrix instruction with fp32 sums, at 16 times the rate of the fp32 one.  A fp32
// factor is cut into three bf16 pieces (8 bits each: the pieces' sum is the value), a bf16 input is one piece and exact, a
// fp16 input two pieces and exact; of the products of pieces those down to 2^-16 of the largest are taken, what is left out is
// below 2^-24 of a term, the rounding of fp32.  bf16 pieces have the range of fp32, which states and
// gradients need.  An infinity becomes NaN in its pieces.
#ifndef KVB_SCAN_DEVICE_H
#define KVB_SCAN_DEVICE_H

#include "kvb_device.h"

#include <utility>

namespace kvb_impl {

constexpr int SC = 64;                      // tokens of a chunk
constexpr int FULL = 3;                     // bf16 pieces of a fp32 value
constexpr int SCAN_TILES = 6;               // 16 x 32 tiles with something in them of a triangular 64 x 64 matrix
constexpr int SCAN_UNITS = SCAN_TILES * 64; // what a lane holds of a tile as the matrix instruction's first operand: 16 bytes of each piece
constexpr int SCAN_MAT = FULL * SCAN_UNITS; // 16-byte words of a matrix's image: piece, tile, lane
constexpr int SCAN_GATES = 4 * SC;          // gamma = exp(c), rest = exp(c_last - c), beta, for the gradients q.k; behind a chunk's end
                                            // beta, rest and q.k are 0

// floats of workspace for each (chunk, v-head): the gates, M and P; for the gradients the gates, M, M' and P'
constexpr int SCAN_PREP = SCAN_GATES + 2 * 4 * SCAN_MAT;
constexpr int GRAD_PREP = SCAN_GATES + 3 * 4 * SCAN_MAT;

struct ScanArgs {
    const void *q, *k, *v;
    const float *g, *beta;
    const float *state0;   // or nullptr: zero
    float *state1;         // or nullptr: not wanted
    void *out;
    const int32_t *start;  // [B + 1]
    const int32_t *slot;   // or nullptr: sequence b's state is row b
    float *prep;           // [chunks][Hv][SCAN_PREP or GRAD_PREP]
    float *s0, *z;         // for the gradients: the state ahead of each chunk [chunks][Hv][d][d], and E - V [chunks][Hv][64][d]
    int64_t q_stride, k_stride, v_stride;   // elements from a token's row to the next
    int32_t B, n_slots, n_tokens, Hk, Hv, r;
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
    // (scalars: addresses that are built on them are scalars too)
    const int first = __builtin_amdgcn_readfirstlane(start[b]), behind = __builtin_amdgcn_readfirstlane(start[b + 1]);
    const int s = min(max(first, 0), n_tokens), e = min(max(behind, s), n_tokens);
    return Span{s, e - s};
}
__device__ __forceinline__ int first_chunk(const Span &s, int b) { return s.first / SC + b; }

// The state row of sequence b, or -1 if there is none.
__device__ __forceinline__ int state_row(const int32_t *slot, int n_slots, int b)
{
    const int s = __builtin_amdgcn_readfirstlane(slot ? slot[b] : b);
    return s >= 0 && s < n_slots ? s : -1;
}

// Workgroup w of those that `parts` each of `units` need, which read the same keys and queries: consecutive workgroups go to the eight XCDs in
// turn, so the parts of a unit are dealt eight apart and meet in one L2.  The units behind the last whole eight are dealt as they come.
// us, against parts that follow each other, bf16, d = 128: kvb_scan_reverse_kernel, 4 sequences of 2048 tokens 234 / 241, kvb_scan_kernel, one of 8191 462 / 470
// (0.29 GB read through the fabric, 1.29).
struct Dealt {
    int unit, part;
};
__device__ __forceinline__ Dealt dealt(int w, int units, int parts)
{
    const int whole = units / 8 * 8, rest = w - whole * parts;
    if (rest >= 0)
        return Dealt{whole + rest / parts, rest % parts};
    const int eight = w / (8 * parts), in = w - eight * 8 * parts;
    return Dealt{8 * eight + in % 8, in / 8};
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

// f(0), .. f(N - 1), each number a compile-time one
template <int N, typename F>
__device__ __forceinline__ void static_for(F &&f)
{
    [&]<int... I>(std::integer_sequence<int, I...>) { (f(std::integral_constant<int, I>{}), ...); }(std::make_integer_sequence<int, N>{});
}

// Sums over the lanes up to one's own, in fp64 (steps of 1, 2, 4 and 8 within rows of 16 lanes, then the rows' last lanes).
template <int CTRL, int ROWS>
__device__ __forceinline__ double shifted(double x)
{
    const uint2 w = __builtin_bit_cast(uint2, x);
    const uint32_t lo = __builtin_amdgcn_update_dpp(0u, w.x, CTRL, ROWS, 0xF, false), hi = __builtin_amdgcn_update_dpp(0u, w.y, CTRL, ROWS, 0xF, false);
    return __builtin_bit_cast(double, make_uint2(lo, hi));
}
__device__ __forceinline__ double sum_below(double x)
{
    x += shifted<0x111, 0xF>(x);
    x += shifted<0x112, 0xF>(x);
    x += shifted<0x114, 0xF>(x);
    x += shifted<0x118, 0xF>(x);
    x += shifted<0x142, 0xA>(x);
    x += shifted<0x143, 0xC>(x);
    return x;
}
// The log decays of a chunk's token in units of log 2 (the matrix of decays needs powers of two), cut off where they are zero anyhow
__device__ __forceinline__ double log2_gate(float g) { return (double)(g < -1e5f ? -1e5f : g) * 1.4426950408889634; }
__device__ __forceinline__ float decay(double c) { return __builtin_amdgcn_exp2f((float)c); }

// Sums over the 16 lanes of a row, of 16 values at once: lane l % 16 = m gets that of x[m].  A lane keeps half of the values in each
// step and hands the others to its mirror image in the row, the half row, the pair of its quad.
template <int CTRL, int N>
__device__ __forceinline__ void halve(float (&x)[16], bool upper)
{
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const float keep = upper ? x[N + i] : x[i], give = upper ? x[i] : x[N + i];
        x[i] = keep + __uint_as_float(__builtin_amdgcn_update_dpp(0u, __float_as_uint(give), CTRL, 0xF, 0xF, false));
    }
}
__device__ __forceinline__ float sum_rows16(float (&x)[16], int m)
{
    halve<0x140, 8>(x, m & 8);
    halve<0x141, 4>(x, m & 4);
    halve<0x4E, 2>(x, m & 2);
    halve<0xB1, 1>(x, m & 1);
    return x[0];
}

// bf16 pieces of an input value
template <typename T>
constexpr int PIECES = __is_same(T, bf16_t) ? 1 : __is_same(T, f16_t) ? 2 : 3;

// (both at once: the conversion of a pair is one instruction)
__device__ __forceinline__ uint32_t pair_bf16(float lo, float hi)
{
    typedef float v2f __attribute__((ext_vector_type(2)));
    typedef __bf16 v2b __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(v2f{lo, hi}, v2b));
}

// Values in N pieces, to nearest: each piece has 8 bits of what the ones before left.  Two values are a word of each piece, eight an
// operand's 16 bytes.
template <int N>
__device__ __forceinline__ void cut2(float x, float y, uint32_t (&p)[N])
{
#pragma unroll
    for (int i = 0; i < N; ++i) {
        p[i] = pair_bf16(x, y);
        x -= __uint_as_float(p[i] << 16);
        y -= __uint_as_float(p[i] & 0xFFFF0000u);
    }
}
template <int N>
__device__ __forceinline__ void cut8(const float (&x)[8], uint4 (&p)[N])
{
    uint32_t w[4][N];
#pragma unroll
    for (int j = 0; j < 4; ++j)
        cut2(x[2 * j], x[2 * j + 1], w[j]);
#pragma unroll
    for (int i = 0; i < N; ++i)
        p[i] = make_uint4(w[0][i], w[1][i], w[2][i], w[3][i]);
}
// An operand's pieces put together word by word
template <int N>
struct Pieces {
    uint32_t w[4][N];
    // words 2 h, 2 h + 1 from the four rows of a sum's tile; or one of them
    __device__ __forceinline__ void half(int h, const f32x4_t &x)
    {
        cut2(x[0], x[1], w[2 * h]);
        cut2(x[2], x[3], w[2 * h + 1]);
    }
    __device__ __forceinline__ void word(int j, const f32x4_t &lo, const f32x4_t &hi)
    {
        const f32x4_t &x = j < 2 ? lo : hi;
        cut2(x[2 * (j % 2)], x[2 * (j % 2) + 1], w[j]);
    }
    __device__ __forceinline__ uint4 piece(int i) const { return make_uint4(w[0][i], w[1][i], w[2][i], w[3][i]); }
};
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
// two sums at a time, in turns: a product waits for the one before on the same sum
template <int NA, int NB>
__device__ __forceinline__ void mma2(f32x4_t &c, f32x4_t &d, const uint4 (&a)[NA], const uint4 (&a2)[NA], const Pieces<NB> &b)
{
#pragma unroll
    for (int i = 0; i < NA; ++i)
#pragma unroll
        for (int j = 0; j < NB; ++j)
            if (i + j < FULL) {
                c = mfma16x32<bf16_t>(a[i], b.piece(j), c);
                d = mfma16x32<bf16_t>(a2[i], b.piece(j), d);
            }
}

// Products and what else there is to do, in turns.  A wave issues in order: products in a row wait for each other, 16 cycles
// each, while three other instructions fit between two of them.  So the steps of a phase alternate, the rest of a phase being work
// for the next one, and stay as they are written.
template <int N, typename F, typename G>
__device__ __forceinline__ void weave(F &&products, G &&rest)
{
    static_for<N>([&](auto i) {
        products(i);
        rest(i);
        __builtin_amdgcn_sched_barrier(0);
    });
}
// items of M that belong to step I of N
template <int M, int N, int I, typename F>
__device__ __forceinline__ void share(F &&f)
{
    constexpr int LO = M * I / N, HI = M * (I + 1) / N;
    static_for<HI - LO>([&](auto j) { f(std::integral_constant<int, LO + j()>{}); });
}
__device__ __forceinline__ f32x4_t as_f32x4(const float4 &x) { return f32x4_t{x.x, x.y, x.z, x.w}; }

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

// The same for M x N sums, each product of pieces for all of them in turn.
// LIM: the pieces i and j with i + j < LIM; what is left out is below 2^-16 of a term with 2, which is for what nothing but a
// result of 16 bits depends on.
template <int LIM = FULL, int M, int N, int NA, int NB>
__device__ __forceinline__ void mma(f32x4_t (&c)[M][N], const uint4 (&a)[M][NA], const uint4 (&b)[N][NB])
{
#pragma unroll
    for (int i = 0; i < NA; ++i)
#pragma unroll
        for (int j = 0; j < NB; ++j)
            if (i + j < LIM)
#pragma unroll
                for (int m = 0; m < M; ++m)
#pragma unroll
                    for (int n = 0; n < N; ++n)
                        c[m][n] = mfma16x32<bf16_t>(a[m][i], b[n][j], c[m][n]);
}

// Operand layouts of v_mfma_f32_16x16x32: lane l holds row (first operand) or column (second) l % 16 and of the 32 that are summed
// over the 8 that belong to l / 16; a sum has column l % 16 in lane l and rows 4 (l / 16) + 0..3 in its four registers.  The order of
// what is summed over is free as long as both operands share it, so the registers of two tiles of a sum become a second
// operand without a move between lanes: lane group g has rows 4g .. 4g+3 of the first tile and of the second.
//   Tokens: the tiles are tokens 16 rt .., and the images of M and P have their columns in that order (4g .. 4g+3, 16+4g .. 16+4g+3).
//   Rows of the state: tile 2 ks + h has in its row 4g + r the state's row 32 ks + 8g + 4h + r (state_row_of), so that a
//   lane group's eight are neighbours and the keys stand in LDS as they come.
__device__ __forceinline__ int state_row_of(int tile, int g, int r) { return 32 * (tile / 2) + 8 * g + 4 * (tile % 2) + r; }
__device__ __forceinline__ void pair8(const f32x4_t &a, const f32x4_t &b, float (&x)[8])
{
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        x[r] = a[r];
        x[4 + r] = b[r];
    }
}

// A stretch of memory: loads behind its end give zeros and stores there do nothing, so that a chunk's missing tokens need no
// test and no branch.  Offsets in bytes, 32 bits, from a scalar address.
struct Buffer {
    typedef int Words __attribute__((ext_vector_type(4)));
    __amdgpu_buffer_rsrc_t r;
    Words words;   // the same, for what there is no builtin of that fits (to_lds)
    // (all scalars, said so: where the compiler is not sure it loops over the lanes)
    __device__ __forceinline__ Buffer(const void *p, uint32_t bytes)
        : r(__builtin_amdgcn_make_buffer_rsrc(scalar(p), 0, __builtin_amdgcn_readfirstlane(bytes), 0x00020000)),
          words{(int)(uint32_t) reinterpret_cast<uint64_t>(scalar(p)), (int)(reinterpret_cast<uint64_t>(scalar(p)) >> 32 & 0xFFFF),
                (int)__builtin_amdgcn_readfirstlane(bytes), 0x00020000}
    {
    }
    // 16 bytes for each lane of the wave straight to LDS, to `to` (lds_at; the same in all lanes) + 16 lane.  Written by hand: behind
    // the builtin the compiler makes any read of LDS wait for it, also of another buffer.  lds_loads_done() is the wait.  (No clobber
    // of memory either, for reads of the other buffer may pass: those of this one are behind a barrier on both sides.)
    __device__ __forceinline__ void to_lds(uint32_t to, uint32_t at) const
    {
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(to), "v"(at), "s"(words) : "m0");
    }
    static __device__ __forceinline__ void *scalar(const void *p)
    {
        const uint64_t x = reinterpret_cast<uint64_t>(p);
        const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)x), hi = __builtin_amdgcn_readfirstlane((uint32_t)(x >> 32));
        return reinterpret_cast<void *>((uint64_t)hi << 32 | lo);
    }
    __device__ __forceinline__ uint4 load16(uint32_t at) const { return __builtin_bit_cast(uint4, __builtin_amdgcn_raw_buffer_load_b128(r, at, 0, 0)); }
    __device__ __forceinline__ uint32_t load4(uint32_t at) const { return __builtin_amdgcn_raw_buffer_load_b32(r, at, 0, 0); }
    __device__ __forceinline__ void store8(uint32_t at, uint2 x) const
    {
        typedef uint32_t v2 __attribute__((ext_vector_type(2)));
        __builtin_amdgcn_raw_buffer_store_b64(__builtin_bit_cast(v2, x), r, at, 0, 0);
    }
    __device__ __forceinline__ void store4(uint32_t at, uint32_t x) const { __builtin_amdgcn_raw_buffer_store_b32(x, r, at, 0, 0); }
};
__device__ __forceinline__ uint32_t lds_at(const uint4 *p) { return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const uint4 *)p; }
// x, anew: what is worked out from it inside a loop stays there and takes no register around it
__device__ __forceinline__ uint32_t anew(uint32_t x)
{
    asm volatile("" : "+v"(x));
    return x;
}
__device__ __forceinline__ void lds_loads_done() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }
template <typename T>
__device__ __forceinline__ Raw8<T> load_raw8(const Buffer &b, uint32_t at)
{
    if constexpr (sizeof(T) == 4)
        return Raw8<T>{__builtin_bit_cast(float4, b.load16(at)), __builtin_bit_cast(float4, b.load16(at + 16))};
    else
        return Raw8<T>{b.load16(at)};
}
// the rows of one head in n tokens, 0 among them (the stride in elements, at most 2^26 bytes: 64 rows in 32 bits)
template <typename T, int D>
__device__ __forceinline__ Buffer head_rows(const T *p, int64_t stride, int n)
{
    return Buffer(p, n == 0 ? 0u : (uint32_t)(n - 1) * (uint32_t)(stride * sizeof(T)) + D * (uint32_t)sizeof(T));
}
// Here and no later: what the values come from has been waited for, and is not waited for behind the stores and loads that follow.
__device__ __forceinline__ void settled(f32x4_t (&x)[4])
{
#pragma unroll
    for (int rt = 0; rt < 4; ++rt)
        asm volatile("" : "+v"(x[rt]));
}

// A barrier of the workgroup that orders what it has in LDS and leaves loads and stores of memory in flight.
__device__ __forceinline__ void lds_barrier()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

// ds_read_b64_tr_b16: 16 lanes read four rows of 16 (8 bytes a lane, rows in turn) and get a column of four each
__device__ __forceinline__ uint2 transposed_four(const uint2 *p)
{
    typedef short v4s __attribute__((ext_vector_type(4)));
    typedef __attribute__((address_space(3))) v4s *Lds;
    return __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)p));
}

// A wave's 16 columns of a chunk's 64 rows of a 16-bit array on their way in or out, in 2 KB of LDS of its own: two requests bring
// them (16 bytes a lane), transposing reads hand them out as a sum's tiles stand.  With a load of two bytes a lane and row, or a store,
// the memory unit was what a chunk waited for (a request takes it 40 to 80 cycles whatever its size).
template <typename T>
struct Slab {
    static constexpr int WORDS = 128;
    static_assert(sizeof(T) == 2);
    uint4 *img;      // the wave's
    uint32_t first;  // the wave's first column, in bytes
    // (a clobber of memory, unlike Buffer::to_lds: what was read from here before has to have been read)
    __device__ __forceinline__ void request(const Buffer &b, uint32_t stride_bytes, int lane) const
    {
        const uint32_t to = __builtin_amdgcn_readfirstlane(lds_at(img)), at = (uint32_t)(lane / 2) * stride_bytes + first + lane % 2 * 16;
#pragma unroll
        for (int i = 0; i < 2; ++i)
            asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(to + i * 1024), "v"(at + i * 32 * stride_bytes), "s"(b.words)
                         : "memory", "m0");
    }
    __device__ __forceinline__ void read(f32x4_t (&x)[4], int lane) const
    {
#pragma unroll
        for (int rt = 0; rt < 4; ++rt) {
            const uint2 w = transposed_four(reinterpret_cast<const uint2 *>(img) + (16 * rt + 4 * (lane / 16) + lane % 16 / 4) * 4 + lane % 4);
            const float2 lo = unpack_pair<T>(w.x), hi = unpack_pair<T>(w.y);
            x[rt] = f32x4_t{lo.x, lo.y, hi.x, hi.y};
        }
    }
    __device__ __forceinline__ void put(const Buffer &b, uint32_t stride_bytes, float scale, const f32x4_t (&x)[4], int lane) const
    {
        const int m = lane % 16, g = lane / 16;
        uint2 *to = reinterpret_cast<uint2 *>(img);
#pragma unroll
        for (int rt = 0; rt < 4; ++rt) {   // column m, rows 4 g ..
            const f32x4_t y = scale * x[rt];
            to[rt * 64 + m * 4 + g] = make_uint2(pack_pair<T>(y[0], y[1]), pack_pair<T>(y[2], y[3]));
        }
        const uint32_t at = m * stride_bytes + first + 8 * g;
#pragma unroll
        for (int rt = 0; rt < 4; ++rt)     // row m, columns 4 g ..
            b.store8(at + 16 * rt * stride_bytes, transposed_four(to + rt * 64 + (4 * g + m / 4) * 4 + m % 4));
    }
};

// The wave's 16 columns of a chunk's 64 rows of a token array, as a sum's tiles stand: of 16-bit arrays through a slab, of fp32 ones by a
// load for each row 16 rt + 4 g + r, which is on its way a chunk ahead.
template <typename T>
struct Columns {
    static constexpr bool SLAB = sizeof(T) == 2;
    uint32_t x[SLAB ? 1 : 16];
    __device__ __forceinline__ void request(const Buffer &b, uint4 *slab, uint32_t first, uint32_t stride_bytes, int lane)
    {
        if constexpr (SLAB) {
            Slab<T>{slab, first}.request(b, stride_bytes, lane);
        } else {
            const uint32_t own = anew(4 * (lane / 16) * stride_bytes + first + lane % 16 * 4);
#pragma unroll
            for (int i = 0; i < 16; ++i)
                x[i] = b.load4(own + (16 * (i / 4) + i % 4) * stride_bytes);
        }
    }
    __device__ __forceinline__ void read(const uint4 *slab, f32x4_t (&y)[4], int lane) const
    {
        if constexpr (SLAB)
            Slab<T>{const_cast<uint4 *>(slab), 0}.read(y, lane);
        else
#pragma unroll
            for (int i = 0; i < 16; ++i)
                y[i / 4][i % 4] = __uint_as_float(x[i]);
    }
    static __device__ __forceinline__ void put(const Buffer &b, uint4 *slab, uint32_t first, uint32_t stride_bytes, float scale, const f32x4_t (&y)[4], int lane)
    {
        if constexpr (SLAB) {
            Slab<T>{slab, first}.put(b, stride_bytes, scale, y, lane);
        } else {
            const uint32_t own = anew(4 * (lane / 16) * stride_bytes + first + lane % 16 * 4);
#pragma unroll
            for (int i = 0; i < 16; ++i)
                b.store4(own + (16 * (i / 4) + i % 4) * stride_bytes, __float_as_uint(scale * y[i / 4][i % 4]));
        }
    }
};

// Four values down a column from each of two blocks; the lane's 8 bytes are the first or second half of the words at p and q
__device__ __forceinline__ uint4 transposed_pair(const uint4 *p, const uint4 *q, int half)
{
    const uint2 l = transposed_four(reinterpret_cast<const uint2 *>(p) + half), h = transposed_four(reinterpret_cast<const uint2 *>(q) + half);
    return make_uint4(l.x, l.y, h.x, h.y);
}
// A 64 x 64 matrix's piece in LDS, tile row it, 32-column step s, lane (row m; group g: columns 4g .. and 16+4g .. of the step): its
// columns 16 jt .. as a second operand, summed over rows 32 s ..
__device__ __forceinline__ uint4 transposed(const uint4 *img, int jt, int s, int lane)
{
    const uint4 *p = img + (4 * s + jt / 2) * 64 + (lane % 4) * 16 + 4 * (lane / 16) + lane % 16 / 4;
    return transposed_pair(p, p + 128, jt % 2);
}

// A chunk's 64 x D keys (or queries) in LDS: piece, 16-token tile, 32-column step, lane, 16 bytes.
// loaded: by the workgroup's waves in turns of a (tile, step), 16 bytes (of a 16-bit type) a lane.
template <typename T, int D, int NWV>
struct TokenTile {
    static constexpr int STEPS = D / 32, N = 4 * STEPS / NWV, NP = PIECES<T>, WORDS = NP * 4 * STEPS * 64;
    static_assert(4 * STEPS % NWV == 0);
    Raw8<T> x[N];
    __device__ __forceinline__ void load(const Buffer &b, uint32_t stride_bytes, int wave, int lane)
    {
        const uint32_t own = (lane % 16) * stride_bytes + 8 * (lane / 16) * (uint32_t)sizeof(T);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int u = wave + NWV * i;
            x[i] = load_raw8<T>(b, own + 16 * (u / STEPS) * stride_bytes + 32 * (u % STEPS) * (uint32_t)sizeof(T));
        }
    }
    __device__ __forceinline__ void store(uint4 *img, int wave, int lane) const
    {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int u = wave + NWV * i;
            uint4 p[NP];
            cut_raw(x[i], p);
#pragma unroll
            for (int j = 0; j < NP; ++j)
                img[(j * 4 * STEPS + u) * 64 + lane] = p[j];
        }
    }
    // the same without registers between, for what is one piece as it comes; part PART of OF
    template <int PART, int OF>
    static __device__ __forceinline__ void to_lds(const Buffer &b, uint32_t stride_bytes, uint32_t img, int wave, int lane)
    {
        static_assert(NP == 1);
        const uint32_t own = anew(lane % 16) * stride_bytes + 8 * (lane / 16) * (uint32_t)sizeof(T);
#pragma unroll
        for (int i = N * PART / OF; i < N * (PART + 1) / OF; ++i) {
            const int u = wave + NWV * i;
            b.to_lds(img + u * 1024, own + 16 * (u / STEPS) * stride_bytes + 32 * (u % STEPS) * (uint32_t)sizeof(T));
        }
    }
    // rows of tokens as the first operand: tile rt, columns 32 ks ..
    static __device__ __forceinline__ void rows(const uint4 *img, int rt, int ks, int lane, uint4 (&a)[NP])
    {
#pragma unroll
        for (int j = 0; j < NP; ++j)
            a[j] = img[((j * 4 + rt) * STEPS + ks) * 64 + lane];
    }
    // the transpose: rows are the state's rows of tile mt, summed over tokens 32 s ..
    static __device__ __forceinline__ void columns(const uint4 *img, int mt, int s, int lane, uint4 (&a)[NP])
    {
        const int at = (lane % 4) * 16 + 4 * (lane / 16) + lane % 16 / 4;
#pragma unroll
        for (int j = 0; j < NP; ++j) {
            const uint4 *p = img + ((j * 4 + 2 * s) * STEPS + mt / 2) * 64 + at;
            a[j] = transposed_pair(p, p + STEPS * 64, mt % 2);
        }
    }
};

// Images of triangular matrices: tile (16 rows rt, 32 columns s) has number tile_of(rt, s); in LDS three pieces of it, 16 bytes a lane.
template <bool UPPER>
__host__ __device__ constexpr int tile_of(int rt, int s)
{
    return UPPER ? (rt < 2 ? 2 * rt + s : 2 + rt) : (rt < 2 ? rt : 2 * rt - 2 + s);
}

// N 16-byte words (blocks of 64) from a workspace to LDS as they are, by the NWV waves of the workgroup: through registers, or without
template <int N, int NWV>
struct Words {
    static_assert(N % 64 == 0);
    static constexpr int BLOCKS = N / 64, EACH = (BLOCKS + NWV - 1) / NWV;
    uint4 x[EACH];
    static __device__ __forceinline__ bool has(int i, int wave) { return NWV * (i + 1) <= BLOCKS || wave + NWV * i < BLOCKS; }
    __device__ __forceinline__ void load(const Buffer &b, int wave, int lane)   // (of N words: zeros behind them)
    {
#pragma unroll
        for (int i = 0; i < EACH; ++i)
            x[i] = b.load16((wave + NWV * i) * 1024 + lane * 16);
    }
    __device__ __forceinline__ void store(uint4 *to, int wave, int lane) const
    {
#pragma unroll
        for (int i = 0; i < EACH; ++i)
            if (has(i, wave))
                to[(wave + NWV * i) * 64 + lane] = x[i];
    }
    template <int PART, int OF>
    static __device__ __forceinline__ void to_lds(const Buffer &b, uint32_t to, int wave, int lane)
    {
#pragma unroll
        for (int i = EACH * PART / OF; i < EACH * (PART + 1) / OF; ++i)
            if (has(i, wave))
                b.to_lds(to + (wave + NWV * i) * 1024, (wave + NWV * i) * 1024 + lane * 16);
    }
};
// The tiles of such an image in pairs of one step: pair i has the tiles of rows pair_row(i) and the next, step pair_step(i).
constexpr int SCAN_PAIRS = SCAN_TILES / 2;
template <bool UPPER>
__host__ __device__ constexpr int pair_row(int i) { return UPPER ? (i == 2 ? 2 : 0) : (i == 0 ? 0 : 2); }
template <bool UPPER>
__host__ __device__ constexpr int pair_step(int i) { return UPPER ? i > 0 : i > 1; }
template <bool UPPER>
__device__ __forceinline__ void load_pair(const uint4 *img, int i, int lane, uint4 (&a)[2][FULL])
{
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int j = 0; j < FULL; ++j)
            a[h][j] = img[j * SCAN_UNITS + tile_of<UPPER>(pair_row<UPPER>(i) + h, pair_step<UPPER>(i)) * 64 + lane];
}

// Threads that a kernel over the chunks is built for.  With DMA a wave needs less than 256 registers; built for 8 waves a workgroup, the
// compiler keeps to that, and does without moves to and from the accumulation registers.
template <typename TIn>
constexpr int scan_bound(int waves) { return PIECES<TIn> == 1 ? 512 : 64 * waves; }

constexpr int SCAN_CUS = 256;   // compute units of the card

// Up to how many tokens a sequence, on average, kvb_scan goes token by token: 0.3 to 0.8 us a token against a chunk's fixed work.
// us, token by token against chunks, bf16, 32 v-heads of 128: 16 sequences of 1 token 14 / 38, of 4 18 / 38, of 8 23 / 38, of 16 33 / 41; one
// sequence of 1 4 / 12, of 8 10 / 12, of 16 16 / 13.  4 and not 8, for the tokens may all be one sequence's, one after the other: the host knows
// the average alone.  A long sequence among many that are empty or short then takes about 1 us a token: 128 slots of which one has 512 tokens 505 us,
// with 513 of them, by chunks, 145 (the one alone 43; the empty ones' states are copied); 512 slots, one of 2048, 2034 (alone 134); 63 single tokens and one sequence of 190 197, of 194 141.
constexpr int TOKEN_MAX = 4;

// Whether a workgroup works out M and P of its chunks itself, in one launch instead of two: for about a chunk a sequence, and workgroups
// that each find a free compute unit (both halves of a head's columns do that work).  us, alone against two launches, bf16, d = 128: 1
// sequence of 37 tokens, 32 v-heads 13.9 / 16.4; 8 of 64, 8 v-heads 15.5 / 19.3; 1 of 128, 32 v-heads 25.8 / 21.6; 32 of 64 (2048 workgroups)
// 122 / 87; 4 of 60, 8 v-heads, fp32, d = 64 14.7 / 18.0.  This, too, goes by the average: 8 sequences of 8 v-heads with all tokens in one of 512 88 us,
// of 513 45.  fp32 at d = 128 has no room for it in LDS, d = 32 too few waves.
template <typename TIn, int D>
constexpr bool CAN_ALONE = D >= 64 && sizeof(TIn) * D < 512;
template <int D>
bool scan_alone(const ScanArgs &a)
{
    return a.n_tokens <= (int64_t)SC * a.B && (int64_t)a.B * a.Hv * (D / 64) <= SCAN_CUS;
}

// How a head's columns are split over workgroups, 16 a wave: f<waves of a workgroup>(workgroups).  LDS has room for one workgroup a
// compute unit, so while there are units for all, fewer waves are faster: they share LDS with fewer others.  Beyond that eight: a
// unit does more at a time, and M and P are read once a head.
// us, bf16, d = 128, 32 v-heads, two waves against four: 1 sequence of 8191 tokens 523 / 558, of 512 43.7 / 46.6, 4 of 512 (two
// rounds of workgroups) 93.6 / 67.1; eight against four: 2 of 512 66 / 53, 4 79 / 68, 6 95 / 113, 8 110 / 126, 16 215 / 240.
// More than one piece passes through registers, and more of them with fewer waves: two against four, fp16, 1 of 2000 234 / 230, fp32, 1
// of 500 86 / 81; eight waves' images and registers do not fit.
template <typename TIn, int D, typename F>
void scan_split(const ScanArgs &a, F &&f)
{
    const int64_t heads = (int64_t)a.B * a.Hv;
    if constexpr (D == 32) {
        f.template operator()<2>(heads);
    } else if constexpr (PIECES<TIn> > 1) {
        f.template operator()<4>(D / 64 * heads);
    } else {
        if (D / 32 * heads <= SCAN_CUS)
            f.template operator()<2>(D / 32 * heads);
        else if (D == 64 || D / 64 * heads <= SCAN_CUS)
            f.template operator()<4>(D / 64 * heads);
        else if constexpr (D == 128)
            f.template operator()<8>(heads);
    }
}

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

// What the gradients need beside the forward pass's arguments (whose out and state1 are not used)
struct GradArgs {
    ScanArgs f;
    const void *dout;
    const float *dstate1;          // or nullptr: zero
    void *dq, *dk, *dv;            // strides of q, k, v
    float *dg, *dbeta, *dstate0;   // dstate0 or nullptr: not wanted
    float *ds;                     // the state's gradient behind each chunk [chunks][Hv][d][d]
    float *dd;                     // D [chunks][Hv][64][d]
    float *part;                   // [chunks][Hv][GRAD_PARTS]
};
constexpr int GRAD_PARTS = 8 * 2 * SC;   // two sums a token of each of the (at most eight) waves that share a head's columns
// floats of workspace for each (chunk, v-head)
__host__ __device__ constexpr int64_t grad_floats(int d) { return GRAD_PREP + 2 * d * d + 2 * SC * d + GRAD_PARTS; }

// one unit per input type (kvb_scan_*.hip, kvb_scan_grad_*.hip)
template <typename TIn, typename TOut>
void launch_scan_typed(int d, const ScanArgs &a, hipStream_t stream);
template <typename TIn, typename TOut>
void launch_scan_grad_typed(int d, const GradArgs &a, hipStream_t stream);

}  // namespace kvb_impl
#endif  // KVB_SCAN_DEVICE_H
