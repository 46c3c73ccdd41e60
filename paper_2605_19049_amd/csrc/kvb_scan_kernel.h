// kvb_scan: the gated delta rule over whole sequences (the mathematics and the images: kvb_scan_device.h).
#ifndef KVB_SCAN_KERNEL_H
#define KVB_SCAN_KERNEL_H

#include "kvb_scan_token_kernel.h"

namespace kvb_impl {

// M and P of one chunk and v-head: a workgroup of four waves, of which wave w has rows 16 w .. of K K' and Q K', G and P.
// M = -(1 + G beta)^-1 G by 16 x 16 blocks: the diagonal blocks column by column in registers (each wave one), then wave J the
// blocks below its own,  M_IJ = -(1 + M_II beta) (G_IJ + sum_K G_IK beta M_KJ),  on the fp32 matrix instruction: the sums'
// registers are its second operand as they stand, if row 4 g + r is taken for what lane group g sums in its r-th step.
// GRAD: M, M' and P' without its diagonal, which goes to the gates, instead of M and P.
// Bounded by latency: some 30 dependent steps (products, the diagonal block's 15 columns, the blocks below) with four LDS round trips between, 8 us
// for a chunk alone, and by its 37 KB of output where there are many.  Three workgroups a compute unit cover each other: 4096 units
// (8191 tokens, 32 v-heads, d = 128) 82 us, 20 ns each.  Working M and P out once for all columns of a head, beside the chain over the
// chunks and not in it, is what the split is for: 64 x 64 triangles cost a wave as much as its share of a chunk.
// c is summed in fp64, so that differences of it are good to fp32 whatever its size; a decay below exp(-1e5) counts as that (zero).
struct PrepScratch {
    static constexpr int LD = SC + 4;
    float gs[SC * LD], ps[SC * LD], td[4 * 16 * 20], beta[SC];
    double cs[SC];
};
// (of the n tokens from `first` on, by 256 threads; what comes out goes to gates and mats, in LDS or in memory)
template <typename TIn, int D, bool GRAD>
__device__ __forceinline__ void prep_chunk(const ScanArgs &a, int first, int n, int hv, PrepScratch &lds, float *gates, uint4 *mats)
{
    constexpr int LD = PrepScratch::LD, MATS = GRAD ? 3 : 2;
    float *gs = lds.gs, *ps = lds.ps, *td = lds.td, *beta = lds.beta;
    double *cs = lds.cs;
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid / 64), lane = tid % 64, m = lane % 16, g = lane / 16, hk = hv / a.r;
    const size_t tok = (size_t)(first + min(lane, n - 1)) * a.Hv + hv;
    const float g1 = a.g[tok], b1 = a.beta[tok];
    const Buffer k = head_rows<TIn, D>(static_cast<const TIn *>(a.k) + first * a.k_stride + hk * D, a.k_stride, n);
    const Buffer q = head_rows<TIn, D>(static_cast<const TIn *>(a.q) + first * a.q_stride + hk * D, a.q_stride, n);
    const uint32_t kst = a.k_stride * sizeof(TIn), qst = a.q_stride * sizeof(TIn), col = 8 * g * sizeof(TIn);
    f32x4_t kk[4] = {}, qk[4] = {};
#pragma unroll
    for (int ks = 0; ks < D / 32; ++ks) {
        const uint32_t c = col + 32 * ks * sizeof(TIn);
        const Raw8<TIn> kr = load_raw8<TIn>(k, (16 * wave + m) * kst + c), qr = load_raw8<TIn>(q, (16 * wave + m) * qst + c);
        Raw8<TIn> br[4];
#pragma unroll
        for (int nt = 0; nt < 4; ++nt)
            br[nt] = load_raw8<TIn>(k, (16 * nt + m) * kst + c);
        uint4 ka[PIECES<TIn>], qa[PIECES<TIn>], b[PIECES<TIn>];
        cut_raw(kr, ka);
        cut_raw(qr, qa);
#pragma unroll
        for (int nt = 0; nt < 4; ++nt) {
            cut_raw(br[nt], b);
            mma(kk[nt], ka, b);
            mma(qk[nt], qa, b);
        }
    }
    const double c = sum_below(lane < n ? log2_gate(g1) : 0.0);
    if (wave == 0) {
        const double last = __shfl(c, 63);
        const float bt = lane < n ? b1 : 0.0f;
        gates[lane] = decay(c);
        gates[SC + lane] = lane < n ? decay(last - c) : 0.0f;
        gates[2 * SC + lane] = bt;
        if (!GRAD)
            gates[3 * SC + lane] = 0.0f;
        cs[lane] = c;
        beta[lane] = bt;
    }
    lds_barrier();
    float *gt = td + wave * 320;   // the transpose of the wave's diagonal block of G
#pragma unroll
    for (int nt = 0; nt < 4; ++nt) {
        const int j = 16 * nt + m;
        float gr[4] = {}, pr[4] = {};
        if (nt <= wave) {
            const double cj = cs[j];
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int i = 16 * wave + 4 * g + r;
                const float d = decay(cs[i] - cj);
                gr[r] = i > j ? d * kk[nt][r] : 0.0f;
                pr[r] = (GRAD ? i > j : i >= j) ? d * qk[nt][r] : 0.0f;
                if (GRAD && i == j)
                    gates[3 * SC + i] = qk[nt][r];
            }
            if (nt == wave)
                *reinterpret_cast<float4 *>(gt + m * 20 + 4 * g) = make_float4(gr[0], gr[1], gr[2], gr[3]);
        }
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            gs[(16 * wave + 4 * g + r) * LD + j] = gr[r];
            ps[(16 * wave + 4 * g + r) * LD + j] = pr[r];
        }
    }
    // the diagonal block: lane m has column m of it (in all four lane groups)
    f32x4_t diag;
    {
        float x[16];
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
            const float4 f = *reinterpret_cast<const float4 *>(gt + m * 20 + i);
            x[i] = -f.x;
            x[i + 1] = -f.y;
            x[i + 2] = -f.z;
            x[i + 3] = -f.w;
        }
#pragma unroll
        for (int l = 0; l < 15; ++l) {
            const float y = -beta[16 * wave + l] * x[l];
#pragma unroll
            for (int i4 = l / 4 * 4; i4 < 16; i4 += 4) {
                const float4 f = *reinterpret_cast<const float4 *>(gt + l * 20 + i4);
                x[i4] = i4 > l ? fmaf(f.x, y, x[i4]) : x[i4];
                x[i4 + 1] = i4 + 1 > l ? fmaf(f.y, y, x[i4 + 1]) : x[i4 + 1];
                x[i4 + 2] = i4 + 2 > l ? fmaf(f.z, y, x[i4 + 2]) : x[i4 + 2];
                x[i4 + 3] = fmaf(f.w, y, x[i4 + 3]);
            }
        }
        const float bm = beta[16 * wave + m];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            diag[r] = g == 0 ? x[r] : g == 1 ? x[4 + r] : g == 2 ? x[8 + r] : x[12 + r];
            gt[(4 * g + r) * 20 + m] = (4 * g + r == m ? 1.0f : 0.0f) + diag[r] * bm;
        }
    }
    lds_barrier();
    f32x4_t mm[4], ym[4];   // block column `wave` of M, and beta M
#pragma unroll
    for (int I = 0; I < 4; ++I) {
        f32x4_t below = {};
        if (I > 0) {
            f32x4_t s;
#pragma unroll
            for (int r = 0; r < 4; ++r)
                s[r] = gs[(16 * I + 4 * g + r) * LD + 16 * wave + m];
#pragma unroll
            for (int K = 0; K < I; ++K) {
                const float4 f = *reinterpret_cast<const float4 *>(gs + (16 * I + m) * LD + 16 * K + 4 * g);
                s = __builtin_amdgcn_mfma_f32_16x16x4f32(f.x, ym[K][0], s, 0, 0, 0);
                s = __builtin_amdgcn_mfma_f32_16x16x4f32(f.y, ym[K][1], s, 0, 0, 0);
                s = __builtin_amdgcn_mfma_f32_16x16x4f32(f.z, ym[K][2], s, 0, 0, 0);
                s = __builtin_amdgcn_mfma_f32_16x16x4f32(f.w, ym[K][3], s, 0, 0, 0);
            }
            const float4 f = *reinterpret_cast<const float4 *>(td + (16 * I + m) * 20 + 4 * g);
            below = __builtin_amdgcn_mfma_f32_16x16x4f32(f.x, s[0], below, 0, 0, 0);
            below = __builtin_amdgcn_mfma_f32_16x16x4f32(f.y, s[1], below, 0, 0, 0);
            below = __builtin_amdgcn_mfma_f32_16x16x4f32(f.z, s[2], below, 0, 0, 0);
            below = __builtin_amdgcn_mfma_f32_16x16x4f32(f.w, s[3], below, 0, 0, 0);
        }
        const float4 b4 = *reinterpret_cast<const float4 *>(beta + 16 * I + 4 * g);
        const float br[4] = {b4.x, b4.y, b4.z, b4.w};
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            mm[I][r] = I < wave ? 0.0f : I == wave ? diag[r] : -below[r];
            ym[I][r] = mm[I][r] * br[r];
        }
    }
    lds_barrier();
#pragma unroll
    for (int I = 0; I < 4; ++I)
#pragma unroll
        for (int r = 0; r < 4; ++r)
            gs[(16 * I + 4 * g + r) * LD + 16 * wave + m] = mm[I][r];
    lds_barrier();
    for (int u = tid; u < MATS * SCAN_UNITS; u += 256) {
        const int of = u / SCAN_UNITS, t = (u - of * SCAN_UNITS) / 64;
        const float *from = (of == MATS - 1 ? ps : gs);
        float x[8];
        if (GRAD && of > 0) {   // the transpose: tile t is tile_of<true>(rt, s)
            const int rt = t < 4 ? t / 2 : t - 2, s = t < 4 ? t % 2 : 1;
            from += (32 * s + 4 * g) * LD + 16 * rt + m;
#pragma unroll
            for (int j = 0; j < 8; ++j)
                x[j] = from[(16 * (j / 4) + j % 4) * LD];
        } else {                // tile_of<false>(rt, s)
            const int rt = t < 2 ? t : 1 + t / 2, s = t < 2 ? 0 : t % 2;
            from += (16 * rt + m) * LD + 32 * s + 4 * g;
            const float4 lo = *reinterpret_cast<const float4 *>(from), hi = *reinterpret_cast<const float4 *>(from + 16);
            pair8(f32x4_t{lo.x, lo.y, lo.z, lo.w}, f32x4_t{hi.x, hi.y, hi.z, hi.w}, x);
        }
        uint4 p[FULL];
        cut8(x, p);
        uint4 *to = mats + of * SCAN_MAT + u - of * SCAN_UNITS;
#pragma unroll
        for (int j = 0; j < FULL; ++j)
            to[j * SCAN_UNITS] = p[j];
    }
}

template <typename TIn, int D, bool GRAD>
__global__ __launch_bounds__(256, 3) void kvb_scan_prep_kernel(const ScanArgs a)
{
    __shared__ PrepScratch lds;
    const int w = blockIdx.x / a.Hv, hv = blockIdx.x - w * a.Hv;
    const ChunkAt at = chunk_at(a.start, a.n_tokens, a.B, w);
    if (at.n == 0)
        return;
    float *prep = a.prep + ((size_t)w * a.Hv + hv) * (GRAD ? GRAD_PREP : SCAN_PREP);
    prep_chunk<TIn, D, GRAD>(a, at.first, at.n, hv, lds, prep, reinterpret_cast<uint4 *>(prep + SCAN_GATES));
}

// The state from chunk to chunk: a workgroup has NWV waves of 16 columns each of one (sequence, v-head).
// A wave keeps its columns of the state in its sums' registers for the whole sequence; the chunk's
// K S and Q S, E and the state's update follow from each other within the wave, and the sums' registers are the next product's second operand
// as they stand.  What the next chunk needs from memory is requested a chunk ahead.
// Bounded by the chain of a chunk's products in a wave: 3.6 us a chunk, of which the matrix instructions are busy 1.5 (three pieces of the state
// against one of the keys), cutting into pieces takes 0.6, requests and stores 0.9, the rest are waits for LDS (37 % of the cycles it is in use go to
// bank conflicts) and for sums.  Few sequences
// leave most of the card idle: one of 8191 tokens, 32 v-heads, d = 128 455 us on 128 compute units, 128 chunks one after the other (55 Tflop/s
// of the recurrence); 24 ragged ones of 1500 340 us on all of them (166 Tflop/s, 1.6 TB/s).
// ALONE: M and P are not there yet, the workgroup works them out itself chunk by chunk: for few chunks, one launch instead of two.
// STATES: for the gradients, no outputs; the state ahead of each chunk and Z = E - V go to the workspace (E - V is no larger
// than the decays, which a difference of E and V would lose).
template <typename TIn, typename TOut, int D, int NWV, bool STATES, bool ALONE>
__global__ __launch_bounds__(ALONE ? 256 : scan_bound<TIn>(NWV)) void kvb_scan_kernel(const ScanArgs a)
{
    constexpr int KT = D / 16, KS = D / 32, SPLIT = D / (16 * NWV);
    using Tok = TokenTile<TIn, D, NWV>;
    constexpr int NP = Tok::NP;
    constexpr bool DMA = NP == 1;   // keys and queries are operands as they come: all images go to LDS without passing registers, into
    constexpr int BUF = DMA && !ALONE ? 2 : 1;   // one buffer while the other is in use
    static_assert(!ALONE || (NWV == 4 && !STATES));
    constexpr int WORDS = SCAN_GATES / 4 + (STATES ? 1 : 2) * SCAN_MAT, PREP = STATES ? GRAD_PREP : SCAN_PREP;
    using Prep = Words<WORDS, NWV>;
    __shared__ uint4 kimgs[BUF][Tok::WORDS], qimgs[BUF][STATES ? 1 : Tok::WORDS], preps[BUF][WORDS];
    __shared__ uint4 slabs[NWV][sizeof(TIn) == 2 || sizeof(TOut) == 2 ? 128 : 1];   // (values in, outputs out)
    struct Nothing {};
    __shared__ std::conditional_t<ALONE, PrepScratch, Nothing> scratch;
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid / 64), lane = tid % 64, m = lane % 16, g = lane / 16;
    const Dealt at = dealt(blockIdx.x, a.B * a.Hk, a.r * SPLIT);
    const int b = at.unit / a.Hk, hk = at.unit - b * a.Hk, hv = hk * a.r + at.part / SPLIT, part = at.part % SPLIT;
    const int row = state_row(a.slot, a.n_slots, b);
    if (row < 0)
        return;
    const Span span = span_of(a.start, a.n_tokens, b);
    const int chunks = (span.len + SC - 1) / SC, col = (part * NWV + wave) * 16 + m;
    const size_t own = ((size_t)row * a.Hv + hv) * D * D + col;

    f32x4_t S[KT] = {};
    if (a.state0)
#pragma unroll
        for (int t = 0; t < KT; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r)
                S[t][r] = a.state0[own + state_row_of(t, g, r) * D];

    const TIn *kp = static_cast<const TIn *>(a.k) + span.first * a.k_stride + hk * D;
    const TIn *qp = static_cast<const TIn *>(a.q) + span.first * a.q_stride + hk * D;
    const TIn *vp = static_cast<const TIn *>(a.v) + span.first * a.v_stride + hv * D;
    const float *prep = a.prep + ((size_t)first_chunk(span, b) * a.Hv + hv) * PREP;
    const size_t prep_step = (size_t)a.Hv * PREP;
    const uint32_t kst = a.k_stride * sizeof(TIn), qst = a.q_stride * sizeof(TIn), vst = a.v_stride * sizeof(TIn), ost = a.Hv * D * sizeof(TOut);
    const uint32_t first = 16 * (part * NWV + wave);   // the wave's column
    uint4 *slab = slabs[wave];

    const uint32_t kat = lds_at(kimgs[0]), qat = lds_at(qimgs[0]), pat = lds_at(preps[0]);
    Tok knext, qnext;   // (without DMA)
    Prep pnext;
    Columns<TIn> vnext;
    int next = min(SC, span.len);   // tokens of the chunk to be asked for, which kp .. prep point to
    // What that needs, asked for in KS parts, one for each step of the products with the state: at once, the requests would
    // wait for each other at the memory unit and the wave with them.
    auto request = [&](auto step, int buf) {
        constexpr int PART = step(), KS = ALONE ? 1 : D / 32;
        const Buffer kb = head_rows<TIn, D>(kp, a.k_stride, next), qb = head_rows<TIn, D>(qp, a.q_stride, next), image(prep, 16 * WORDS);
        if constexpr (DMA) {
            Tok::template to_lds<PART, KS>(kb, kst, kat + buf * 16 * Tok::WORDS, wave, lane);
            if constexpr (!STATES)
                Tok::template to_lds<PART, KS>(qb, qst, qat + buf * 16 * Tok::WORDS, wave, lane);
            if constexpr (!ALONE)
                Prep::template to_lds<PART, KS>(image, pat + buf * 16 * WORDS, wave, lane);
        } else if constexpr (PART == 0) {
            knext.load(kb, kst, wave, lane);
            if constexpr (!STATES)
                qnext.load(qb, qst, wave, lane);
            if constexpr (!ALONE)
                pnext.load(image, wave, lane);
        }
        if constexpr (PART == KS - 1)
            vnext.request(head_rows<TIn, D>(vp, a.v_stride, next), slab, first * sizeof(TIn), vst, lane);
    };
    Pieces<FULL> sp[KS];   // of the state
#pragma unroll
    for (int j = 0; j < 4; ++j)
        sp[0].word(j, S[0], S[1]);
    f32x4_t O[4] = {};
    const size_t own_chunk = (size_t)first_chunk(span, b) * a.Hv + hv;
    auto put = [&](int c) {   // (STATES: O holds Z)
        if constexpr (STATES) {
            Columns<float>::put(head_rows<float, D>(a.z + (own_chunk + (int64_t)c * a.Hv) * SC * D, D, c < 0 ? 0 : SC), nullptr, first * 4, 4 * D, 1.0f, O, lane);
            return;
        }
        TOut *p = static_cast<TOut *>(a.out) + ((int64_t)(span.first + c * SC) * a.Hv + hv) * D;
        Columns<TOut>::put(head_rows<TOut, D>(p, (int64_t)a.Hv * D, c < 0 ? 0 : min(SC, span.len - c * SC)), slab, first * sizeof(TOut), ost, a.scale, O, lane);
    };
    if (!ALONE && chunks > 0)
        static_for<KS>([&](auto step) { request(step, 0); });
    for (int c = 0; c < chunks; ++c) {
        const int buf = BUF == 2 ? c & 1 : 0;
        if constexpr (ALONE) {
            lds_barrier();   // (the chunk before has been read)
            request(std::integral_constant<int, 0>{}, 0);
            prep_chunk<TIn, D, false>(a, span.first + c * SC, next, hv, scratch, reinterpret_cast<float *>(preps[0]), preps[0] + SCAN_GATES / 4);
        }
        const uint4 *kimg = kimgs[buf], *qimg = qimgs[buf], *mats = preps[buf] + SCAN_GATES / 4;
        const float4 *gate = reinterpret_cast<const float4 *>(preps[buf]);
        if constexpr (DMA || Columns<TIn>::SLAB)
            lds_loads_done();
        if constexpr (!DMA) {
            knext.store(kimgs[0], wave, lane);
            if constexpr (!STATES)
                qnext.store(qimgs[0], wave, lane);
            if constexpr (!ALONE)
                pnext.store(preps[0], wave, lane);
        }
        f32x4_t E[4], y[4] = {};
        vnext.read(slab, E, lane);
        settled(E);
        lds_barrier();
        if (c + 1 < chunks) {   // (the last chunk is asked for once more behind it)
            kp += SC * a.k_stride;
            qp += SC * a.q_stride;
            vp += SC * a.v_stride;
            prep += prep_step;
            next = min(SC, span.len - (c + 1) * SC);
        }
        // The outputs of the chunk before leave here: what a wave waits for at the chunk's end is then not a store just made.  (Nothing
        // for the first, and the last chunk's inputs once more behind it: branches would make the waits wait for everything.)
        put(c - 1);
#pragma unroll
        for (int rt = 0; rt < 4; ++rt)
            O[rt] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
        if constexpr (STATES) {
            const Buffer to(a.s0 + (own_chunk + (size_t)c * a.Hv) * D * D, 4 * D * D);
#pragma unroll
            for (int t = 0; t < KT; ++t)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    to.store4((state_row_of(t, g, r) * D + col) * 4, __float_as_uint(S[t][r]));
        }
        // y = K S; the state's pieces
        Pieces<FULL> yp[2], up[2], ep[2];
        uint4 fr[2][4][NP], ft[2][2][NP], fm[2][2][FULL];
        f32x4_t gm[4], bt[4], re[4];
        auto columns = [&](auto i) {   // pair i of KT
#pragma unroll
            for (int h = 0; h < 2; ++h)
                Tok::columns(kimg, (2 * i() + h) % KT, 2 * i() / KT, lane, ft[i() % 2][h]);
        };
        auto rows = [&](const uint4 *img, int ks, uint4 (&f)[4][NP]) {
#pragma unroll
            for (int rt = 0; rt < 4; ++rt)
                Tok::rows(img, rt, ks, lane, f[rt]);
        };
        rows(kimg, 0, fr[0]);
        weave<2 * KS>([&](auto i) { constexpr int rt = 2 * (i() % 2); mma2(y[rt], y[rt + 1], fr[i() / 2 % 2][rt], fr[i() / 2 % 2][rt + 1], sp[i() / 2]); },
                      [&](auto i) {
                          constexpr int ks = i() / 2, rt = 2 * (i() % 2);
                          if constexpr (ks + 1 < KS) {
                              sp[ks + 1].word(rt, S[2 * ks + 2], S[2 * ks + 3]);
                              sp[ks + 1].word(rt + 1, S[2 * ks + 2], S[2 * ks + 3]);
                              if constexpr (rt == 0)
                                  rows(kimg, ks + 1, fr[(ks + 1) % 2]);
                          } else {
                              if constexpr (rt == 0 && !STATES)
                                  rows(qimg, 0, fr[KS % 2]);
#pragma unroll
                              for (int h = rt; h < rt + 2; ++h) {
                                  gm[h] = as_f32x4(gate[4 * h + g]);
                                  bt[h] = as_f32x4(gate[32 + 4 * h + g]);
                              }
                          }
                          if constexpr (rt == 2 && !ALONE)
                              request(std::integral_constant<int, ks>{}, buf ^ 1);
                      });
        // O = Q S; Y = V - gamma y, the pieces of beta Y
        auto residual = [&](auto i) {
            constexpr int rt = i() / 3;
            if constexpr (i() % 3 == 0) {
                if constexpr (STATES) {
                    O[rt] = -gm[rt] * y[rt];
                    y[rt] = bt[rt] * (E[rt] + O[rt]);
                } else {
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        E[rt][r] = fmaf(-gm[rt][r], y[rt][r], E[rt][r]);
                    y[rt] = bt[rt] * E[rt];
                }
            } else {
                yp[rt / 2].word(2 * (rt % 2) + i() % 3 - 1, y[rt], y[rt]);
            }
        };
        if constexpr (STATES)
            static_for<12>(residual);
        else
            weave<2 * KS>([&](auto i) { constexpr int rt = 2 * (i() % 2); mma2(O[rt], O[rt + 1], fr[(KS + i() / 2) % 2][rt], fr[(KS + i() / 2) % 2][rt + 1], sp[i() / 2]); },
                          [&](auto i) {
                              if constexpr (i() % 2 == 0 && i() / 2 + 1 < KS)
                                  rows(qimg, i() / 2 + 1, fr[(KS + i() / 2 + 1) % 2]);
                              share<12, 2 * KS, i()>(residual);
                          });
        // E = Y + M beta Y (STATES: Z); the state and O decay, and the pieces of beta E and rest beta E of the first 32 tokens
        const float last = reinterpret_cast<const float *>(gate)[SC - 1];
        f32x4_t(&sum)[4] = STATES ? O : E;
        // item i of two tiles' ten: beta E, its words, rest beta E, its words
        auto weigh = [&](auto s, auto i) {
            constexpr int lo = 2 * s(), hi = lo + 1;
            if constexpr (i() == 0) {
                if constexpr (STATES) {
                    E[lo] += O[lo];
                    E[hi] += O[hi];
                }
                y[lo] = bt[lo] * E[lo];
                y[hi] = bt[hi] * E[hi];
            } else if constexpr (i() < 5) {
                if constexpr (!STATES)
                    up[s()].word(i() - 1, y[lo], y[hi]);
            } else if constexpr (i() == 5) {
                y[lo] *= re[lo];
                y[hi] *= re[hi];
            } else {
                ep[s()].word(i() - 6, y[lo], y[hi]);
            }
        };
        load_pair<false>(mats, 0, lane, fm[0]);
        weave<SCAN_PAIRS>([&](auto i) { constexpr int rt = pair_row<false>(i()); mma2(sum[rt], sum[rt + 1], fm[i() % 2][0], fm[i() % 2][1], yp[pair_step<false>(i())]); },
                          [&](auto i) {
                              if constexpr (i() + 1 < SCAN_PAIRS)
                                  load_pair<false>(mats, i() + 1, lane, fm[(i() + 1) % 2]);
                              else
                                  columns(std::integral_constant<int, 0>{});
                              if constexpr (i() == 0) {
#pragma unroll
                                  for (int rt = 0; rt < 4; ++rt) {
                                      re[rt] = as_f32x4(gate[16 + 4 * rt + g]);
                                      if constexpr (!STATES)
                                          O[rt] *= gm[rt];
                                  }
                              } else if constexpr (i() == 1) {
                                  static_for<10>([&](auto j) { weigh(std::integral_constant<int, 0>{}, j); });
                              } else {
#pragma unroll
                                  for (int t = 0; t < KT; ++t)
                                      S[t] *= last;
                              }
                          });
        // S += K' rest beta E, O += P beta E: the state from the first 32 tokens, while the others' pieces are made, O, the state from the others
        auto update = [&](auto i) { constexpr int t = 2 * i() % KT; mma2(S[t], S[t + 1], ft[i() % 2][0], ft[i() % 2][1], ep[2 * i() / KT]); };
        weave<KT / 2>(update, [&](auto i) {
            columns(std::integral_constant<int, i() + 1>{});
            if constexpr (!STATES && i() + 1 == KT / 2)
                load_pair<false>(mats + SCAN_MAT, 0, lane, fm[0]);
            share<10, KT / 2, i()>([&](auto j) { weigh(std::integral_constant<int, 1>{}, j); });
        });
        if constexpr (!STATES)
            weave<SCAN_PAIRS>([&](auto i) { constexpr int rt = pair_row<false>(i()); mma2(O[rt], O[rt + 1], fm[i() % 2][0], fm[i() % 2][1], up[pair_step<false>(i())]); },
                              [&](auto i) {
                                  if constexpr (i() + 1 < SCAN_PAIRS)
                                      load_pair<false>(mats + SCAN_MAT, i() + 1, lane, fm[(i() + 1) % 2]);
                              });
        weave<KT / 2>([&](auto i) { update(std::integral_constant<int, KT / 2 + i()>{}); },
                      [&](auto i) {
                          if constexpr (i() + 1 < KT / 2)
                              columns(std::integral_constant<int, KT / 2 + i() + 1>{});
                          // the first pieces of the next chunk's state
                          if constexpr (i() > 0)
                              share<4, KT / 2 - 1, i() - 1>([&](auto j) { sp[0].word(j(), S[0], S[1]); });
                      });
        if constexpr (KT == 2)
            static_for<4>([&](auto j) { sp[0].word(j(), S[0], S[1]); });
        if constexpr (!DMA && !ALONE)
            lds_barrier();
    }
    lds_loads_done();   // (what was asked for once more: it must not land in the slab below, or in a later workgroup's LDS)
    if (chunks > 0)
        put(chunks - 1);
    if (a.state1)
#pragma unroll
        for (int t = 0; t < KT; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r)
                a.state1[own + state_row_of(t, g, r) * D] = S[t][r];
}

template <typename TIn, typename TOut, int D>
void launch_scan_sized(const ScanArgs &a, hipStream_t stream)
{
    if (a.n_tokens <= TOKEN_MAX * (int64_t)a.B) {
        launch_part(kvb_scan_token_kernel<TIn, TOut, D>, true, true, (int64_t)a.B * a.Hv * (D / 32), 64, stream, a);
        return;
    }
    if constexpr (CAN_ALONE<TIn, D>) {
        if (scan_alone<D>(a)) {
            launch_part(kvb_scan_kernel<TIn, TOut, D, 4, false, true>, true, true, (int64_t)a.B * a.Hv * (D / 64), 256, stream, a);
            return;
        }
    }
    launch_part(kvb_scan_prep_kernel<TIn, D, false>, true, false, scan_chunks(a.n_tokens, a.B) * a.Hv, 256, stream, a);
    scan_split<TIn, D>(a, [&]<int NWV>(int64_t blocks) {
        launch_part(kvb_scan_kernel<TIn, TOut, D, NWV, false, false>, false, true, blocks, 64 * NWV, stream, a);
    });
}
template <typename TIn, typename TOut>
void launch_scan_typed(int d, const ScanArgs &a, hipStream_t stream)
{
    if (d == 32)
        launch_scan_sized<TIn, TOut, 32>(a, stream);
    else if (d == 64)
        launch_scan_sized<TIn, TOut, 64>(a, stream);
    else
        launch_scan_sized<TIn, TOut, 128>(a, stream);
}

}  // namespace kvb_impl
#endif  // KVB_SCAN_KERNEL_H
