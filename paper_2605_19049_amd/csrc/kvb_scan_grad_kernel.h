// kvb_scan_backward: the gradients of kvb_scan (images, layouts and precision: kvb_scan_device.h).
//
// With dO' = scale dO, the chunk's first state S0, the gradient dS1 of the state behind it, and E, G, M, P of the forward pass:
//     X   = P' dO' + rest K dS1                      D   = X + M' beta X              dV = beta D
//     dS0 = exp(c_last) dS1 + Q' (gamma dO') - K' (gamma dV)
//     dQ  = gamma dO' S0' + W1 K                     W1_ij = exp(c_i - c_j) beta_j dO'_i.E_j   i >= j
//     dK  = rest beta E dS1' - gamma dV S0' + W1' Q - W2 K - W2' K      W2_ij = exp(c_i - c_j) beta_j dV_i.E_j   i > j
//     dbeta_i = D_i.E_i
// (gamma = exp(c), rest = exp(c_last - c).)  A token's log decay scales what was there before it for all tokens from it on:
//     dg_t = sum_{i >= t} (Q_i.dQ'_i + Z_i.dV_i - beta_i E_i.D'_i) + sum_{i < t} beta_i E_i.(rest K dS1)_i + exp(c_last) <dS1, S0>
// over the chunk, with Z = E - V, and dQ' and D' without what has no decay in it (W1's diagonal; rest K dS1 and P's diagonal).
// So every term is as small as its decays are, and nothing large cancels; W1's and P's diagonals are kept apart throughout.
//   kvb_scan_prep_kernel<GRAD>, kvb_scan_kernel<STATES>   M, M', P' of all chunks; S0 and Z, from chunk to chunk
//   kvb_scan_reverse_kernel                               dS, D and dV from the last chunk to the first, split like the forward pass
//   kvb_scan_grad_kernel                                  dQ, dK, dbeta, dg of all chunks side by side; a workgroup has a qk-head and
//                                                         adds up its v-heads in their order: the same bits every time
#ifndef KVB_SCAN_GRAD_KERNEL_H
#define KVB_SCAN_GRAD_KERNEL_H

#include "kvb_scan_kernel.h"

namespace kvb_impl {

// From the last chunk to the first: dS in the sums' registers, as the state in kvb_scan_kernel.  Bounded by the chain of a chunk's products, like that,
// and by what it leaves for the next kernel (dS and D, 96 KB a chunk and head at d = 128): 4 sequences of 2048 tokens, 32 v-heads, bf16 234 us, 7.3 us a
// chunk, 0.54 GB read and 0.49 written, 4.4 TB/s.  States ahead of and gradients behind each chunk are stored because the chunks' other gradients are then
// independent; working them out again would put two more chains in front of kvb_scan_grad_kernel.
template <typename TIn, typename TOut, int D, int NWV>
__global__ __launch_bounds__(scan_bound<TIn>(NWV)) void kvb_scan_reverse_kernel(const GradArgs ga)
{
    constexpr int KT = D / 16, KS = D / 32, SPLIT = D / (16 * NWV);
    using Tok = TokenTile<TIn, D, NWV>;
    constexpr int NP = Tok::NP;
    constexpr bool DMA = NP == 1;   // (as in kvb_scan_kernel)
    constexpr int BUF = DMA ? 2 : 1;
    using Gates = Words<SCAN_GATES / 4, NWV>;
    using Mats = Words<2 * SCAN_MAT, NWV>;
    __shared__ uint4 kimgs[BUF][Tok::WORDS], qimgs[BUF][Tok::WORDS], matss[BUF][2 * SCAN_MAT], gatess[BUF][SCAN_GATES / 4];
    __shared__ uint4 slabs[NWV][sizeof(TIn) == 2 ? 128 : 1], oslabs[NWV][sizeof(TOut) == 2 ? 128 : 1];   // (values in, their gradients out; the outputs' in)
    const ScanArgs &a = ga.f;
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid / 64), lane = tid % 64, m = lane % 16, g = lane / 16;
    const Dealt at = dealt(blockIdx.x, a.B * a.Hk, a.r * SPLIT);
    const int b = at.unit / a.Hk, hk = at.unit - b * a.Hk, hv = hk * a.r + at.part / SPLIT, part = at.part % SPLIT;
    const int row = state_row(a.slot, a.n_slots, b);
    if (row < 0)
        return;
    const Span span = span_of(a.start, a.n_tokens, b);
    const int chunks = (span.len + SC - 1) / SC, col = (part * NWV + wave) * 16 + m;
    const size_t own = ((size_t)row * a.Hv + hv) * D * D;
    const size_t own_chunk = (size_t)first_chunk(span, b) * a.Hv + hv;

    f32x4_t S[KT] = {};   // the gradient of the state
    auto state_at = [&](int t, int r) { return (uint32_t)(state_row_of(t, g, r) * D + col) * 4; };
    auto store_state = [&](float *p) {
        const Buffer to(p, 4 * D * D);
#pragma unroll
        for (int t = 0; t < KT; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r)
                to.store4(state_at(t, r), __float_as_uint(S[t][r]));
    };
    if (ga.dstate1) {
        const Buffer from(ga.dstate1 + own, 4 * D * D);
#pragma unroll
        for (int t = 0; t < KT; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r)
                S[t][r] = __uint_as_float(from.load4(state_at(t, r)));
    }

    const TIn *kp = static_cast<const TIn *>(a.k) + span.first * a.k_stride + hk * D;
    const TIn *qp = static_cast<const TIn *>(a.q) + span.first * a.q_stride + hk * D;
    const TOut *op = static_cast<const TOut *>(ga.dout) + ((size_t)span.first * a.Hv + hv) * D;
    const TIn *vp = static_cast<const TIn *>(a.v) + span.first * a.v_stride + hv * D;
    TIn *dvp = static_cast<TIn *>(ga.dv) + span.first * a.v_stride + hv * D;
    const uint32_t kst = a.k_stride * sizeof(TIn), qst = a.q_stride * sizeof(TIn), vst = a.v_stride * sizeof(TIn), ost = a.Hv * D * sizeof(TOut);
    const uint32_t first = 16 * (part * NWV + wave);   // the wave's column
    uint4 *slab = slabs[wave], *oslab = oslabs[wave];

    const uint32_t kat = lds_at(kimgs[0]), qat = lds_at(qimgs[0]), mat = lds_at(matss[0]), gat = lds_at(gatess[0]);
    Tok knext, qnext;   // (without DMA)
    Mats mnext;
    Gates gnext;
    Columns<TOut> onext;
    Columns<float> znext;
    Columns<TIn> vnext;
    auto request = [&](auto step, int c, int buf) {   // (in parts: kvb_scan_kernel)
        constexpr int PART = step();
        const int n = min(SC, span.len - c * SC);
        const Buffer kb = head_rows<TIn, D>(kp + (int64_t)c * SC * a.k_stride, a.k_stride, n);
        const Buffer qb = head_rows<TIn, D>(qp + (int64_t)c * SC * a.q_stride, a.q_stride, n);
        const float *prep = a.prep + (own_chunk + (size_t)c * a.Hv) * GRAD_PREP;
        const Buffer gates(prep, 4 * SCAN_GATES), images(prep + SCAN_GATES + 4 * SCAN_MAT, 2 * 16 * SCAN_MAT);
        if constexpr (DMA) {
            Tok::template to_lds<PART, KS>(kb, kst, kat + buf * 16 * Tok::WORDS, wave, lane);
            Tok::template to_lds<PART, KS>(qb, qst, qat + buf * 16 * Tok::WORDS, wave, lane);
            Mats::template to_lds<PART, KS>(images, mat + buf * 32 * SCAN_MAT, wave, lane);
            Gates::template to_lds<PART, KS>(gates, gat + buf * 4 * SCAN_GATES, wave, lane);
        } else if constexpr (PART == 0) {
            knext.load(kb, kst, wave, lane);
            qnext.load(qb, qst, wave, lane);
            mnext.load(images, wave, lane);
            gnext.load(gates, wave, lane);
        }
    };
    auto request_rows = [&](int c) {
        const int n = min(SC, span.len - c * SC);
        onext.request(head_rows<TOut, D>(op + (int64_t)c * SC * a.Hv * D, (int64_t)a.Hv * D, n), oslab, first * sizeof(TOut), ost, lane);
        znext.request(head_rows<float, D>(a.z + (own_chunk + (size_t)c * a.Hv) * SC * D, D, SC), nullptr, first * 4, 4 * D, lane);
        vnext.request(head_rows<TIn, D>(vp + (int64_t)c * SC * a.v_stride, a.v_stride, n), slab, first * sizeof(TIn), vst, lane);
    };
    if (chunks > 0) {
        static_for<KS>([&](auto step) { request(step, chunks - 1, 0); });
        request_rows(chunks - 1);
    }
    f32x4_t X[4] = {}, dn[4] = {};   // from a chunk's end on dV and D
    auto put = [&](int c) {
        const bool none = c >= chunks;
        Columns<TIn>::put(head_rows<TIn, D>(dvp + (int64_t)c * SC * a.v_stride, a.v_stride, none ? 0 : min(SC, span.len - c * SC)), slab, first * sizeof(TIn), vst,
                          1.0f, X, lane);
        Columns<float>::put(head_rows<float, D>(ga.dd + (own_chunk + (int64_t)c * a.Hv) * SC * D, D, none ? 0 : SC), nullptr, first * 4, 4 * D, 1.0f, dn, lane);
    };
    for (int c = chunks - 1, buf = 0; c >= 0; --c, buf = DMA ? buf ^ 1 : 0) {
        const uint4 *kimg = kimgs[buf], *qimg = qimgs[buf], *mats = matss[buf];
        const float4 *gate = reinterpret_cast<const float4 *>(gatess[buf]);
        if constexpr (DMA || Columns<TIn>::SLAB)
            lds_loads_done();
        if constexpr (!DMA) {
            knext.store(kimgs[0], wave, lane);
            qnext.store(qimgs[0], wave, lane);
            mnext.store(matss[0], wave, lane);
            gnext.store(gatess[0], wave, lane);
        }
        f32x4_t dO[4], E[4], Z[4], kd[4] = {};
        onext.read(oslab, dO, lane);
        vnext.read(slab, E, lane);
        znext.read(nullptr, Z, lane);
#pragma unroll
        for (int rt = 0; rt < 4; ++rt)
            E[rt] += Z[rt];
        settled(dO);
        settled(E);
        lds_barrier();
        put(c + 1);   // (here for the reasons of kvb_scan_kernel)
        store_state(ga.ds + (own_chunk + (size_t)c * a.Hv) * D * D);
#pragma unroll
        for (int rt = 0; rt < 4; ++rt)
            X[rt] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
        // kd = K dS; the pieces of dS
        Pieces<FULL> sp[KS], oq[2], xp[2], zp[2];
        Pieces<PIECES<TOut>> od[2];
        uint4 fr[2][4][NP], ft[2][2][NP], fm[2][2][FULL];
        auto columns = [&](const uint4 *img, auto i) {   // pair i of KT
#pragma unroll
            for (int h = 0; h < 2; ++h)
                Tok::columns(img, (2 * i() + h) % KT, 2 * i() / KT, lane, ft[i() % 2][h]);
        };
        auto update = [&](auto i, const Pieces<FULL> (&p)[2]) { constexpr int t = 2 * i() % KT; mma2(S[t], S[t + 1], ft[i() % 2][0], ft[i() % 2][1], p[2 * i() / KT]); };
        auto gate_at = [&](int which, int rt) { return as_f32x4(gate[16 * which + 4 * rt + g]); };
        auto rows = [&](int ks) {
#pragma unroll
            for (int rt = 0; rt < 4; ++rt)
                Tok::rows(kimg, rt, ks, lane, fr[ks % 2][rt]);
        };
        rows(0);
#pragma unroll
        for (int j = 0; j < 4; ++j)
            sp[0].word(j, S[0], S[1]);
        weave<2 * KS>([&](auto i) { constexpr int rt = 2 * (i() % 2); mma2(kd[rt], kd[rt + 1], fr[i() / 2 % 2][rt], fr[i() / 2 % 2][rt + 1], sp[i() / 2]); },
                      [&](auto i) {
                          constexpr int ks = i() / 2, rt = 2 * (i() % 2);
                          if constexpr (ks + 1 < KS) {
                              sp[ks + 1].word(rt, S[2 * ks + 2], S[2 * ks + 3]);
                              sp[ks + 1].word(rt + 1, S[2 * ks + 2], S[2 * ks + 3]);
                              if constexpr (rt == 0)
                                  rows(ks + 1);
                          } else {
                              od[rt / 2].half(0, dO[rt]);
                              od[rt / 2].half(1, dO[rt + 1]);
                              if constexpr (rt == 2)
                                  load_pair<true>(mats + SCAN_MAT, 0, lane, fm[0]);
                          }
                          if constexpr (rt == 2)
                              request(std::integral_constant<int, ks>{}, max(c - 1, 0), buf ^ 1);
                      });
        // X = P' dO (without P's diagonal); dS decays, the pieces of scale gamma dO
        const float last = reinterpret_cast<const float *>(gate)[SC - 1];
        weave<SCAN_PAIRS>([&](auto i) { constexpr int rt = pair_row<true>(i()); mma2(X[rt], X[rt + 1], fm[i() % 2][0], fm[i() % 2][1], od[pair_step<true>(i())]); },
                          [&](auto i) {
                              if constexpr (i() + 1 < SCAN_PAIRS)
                                  load_pair<true>(mats + SCAN_MAT, i() + 1, lane, fm[(i() + 1) % 2]);
                              else
                                  columns(qimg, std::integral_constant<int, 0>{});
                              if constexpr (i() < 2) {
                                  oq[i()].half(0, a.scale * gate_at(0, 2 * i()) * dO[2 * i()]);
                                  oq[i()].half(1, a.scale * gate_at(0, 2 * i() + 1) * dO[2 * i() + 1]);
                              } else {
#pragma unroll
                                  for (int t = 0; t < KT; ++t)
                                      S[t] *= last;
                              }
                          });
        // dS += Q' scale gamma dO; kd = rest kd + scale q.k dO, dn = scale P' dO, the pieces of beta X, X = dn + kd; E rest kd
        float inner[16], outer[16];
        auto join = [&](auto i) {
            constexpr int rt = i() / 3;
            if constexpr (i() % 3 == 0) {
                const f32x4_t back = gate_at(1, rt) * kd[rt], own_share = a.scale * gate_at(3, rt);
                kd[rt] = own_share * dO[rt] + back;
                dn[rt] = a.scale * X[rt];
                X[rt] = gate_at(2, rt) * (dn[rt] + kd[rt]);
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    outer[4 * rt + r] = E[rt][r] * back[r];
            } else {
                xp[rt / 2].word(2 * (rt % 2) + i() % 3 - 1, X[rt], X[rt]);
            }
        };
        weave<KT>([&](auto i) { update(i, oq); },
                  [&](auto i) {
                      if constexpr (i() + 1 < KT)
                          columns(qimg, std::integral_constant<int, i() + 1>{});
                      else
                          load_pair<true>(mats, 0, lane, fm[0]);
                      share<12, KT, i()>(join);
                  });
        // dn += M' beta X: what D has that decays.  Then the tokens' sums of E dn and E rest kd over the wave's columns, D = dn + kd,
        // dV = beta D, and the pieces of -gamma dV
        request_rows(max(c - 1, 0));
        float *sums = ga.part + (own_chunk + (size_t)c * a.Hv) * GRAD_PARTS + (part * NWV + wave) * 2 * SC + 16 * (m / 4) + 4 * g + m % 4;
        auto end = [&](auto s, auto i) {
            constexpr int lo = 2 * s();
            if constexpr (i() == 0) {
#pragma unroll
                for (int rt = lo; rt < lo + 2; ++rt) {
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        inner[4 * rt + r] = E[rt][r] * dn[rt][r];
                    dn[rt] += kd[rt];
                    X[rt] = gate_at(2, rt) * dn[rt];
                    kd[rt] = -gate_at(0, rt) * X[rt];
                }
            } else {
                zp[s()].word(i() - 1, kd[lo], kd[lo + 1]);
            }
        };
        weave<SCAN_PAIRS>([&](auto i) { constexpr int rt = pair_row<true>(i()); mma2(dn[rt], dn[rt + 1], fm[i() % 2][0], fm[i() % 2][1], xp[pair_step<true>(i())]); },
                          [&](auto i) {
                              if constexpr (i() + 1 < SCAN_PAIRS)
                                  load_pair<true>(mats, i() + 1, lane, fm[(i() + 1) % 2]);
                              else
                                  columns(kimg, std::integral_constant<int, 0>{});
                              if constexpr (i() == 0)
                                  sums[SC] = sum_rows16(outer, m);
                              if constexpr (i() == 2)
                                  static_for<5>([&](auto j) { end(std::integral_constant<int, 0>{}, j); });
                          });
        // dS -= K' gamma dV
        weave<KT>([&](auto i) { update(i, zp); },
                  [&](auto i) {
                      if constexpr (i() + 1 < KT)
                          columns(kimg, std::integral_constant<int, i() + 1>{});
                      if constexpr (i() < KT / 2)
                          share<5, KT / 2, i()>([&](auto j) { end(std::integral_constant<int, 1>{}, j); });
                      else if constexpr (i() == KT / 2)
                          sums[0] = sum_rows16(inner, m);
                  });
        if constexpr (!DMA)
            lds_barrier();
    }
    lds_loads_done();   // (what was asked for once more: it must not land in the slab below, or in a later workgroup's LDS)
    if (chunks > 0)
        put(0);
    if (ga.dstate0)
        store_state(ga.dstate0 + own);
}

// dQ, dK, dbeta and dg of one chunk and qk-head.  D / 32 waves; wave w has columns 32 w .. of dQ and dK for all 64 tokens, as their
// transposes: dQ' = S0 dO' and so on have the state's rows as first operand, which each wave reads from memory once, and
// the tokens' rows (dO, E, dV) as second, from LDS.  The two 64 x 64 matrices are worked out a tile column a
// wave, transposed; their sums' registers, two tiles together, are a second operand for W K, and read back transposed one for W' Q.
// Bounded by memory and its latency, one workgroup of four waves a compute unit (some 500 registers a wave: all of dQ, dK and the products in flight;
// 39 % of a wave's life is waiting for loads): the example above 358 us, 1.24 GB read, 3.7 TB/s (keys and queries asked for anew for each
// v-head 376 us, 1.35 GB).  A qk-head a workgroup, not a v-head, makes dQ and dK sums in a fixed order
// without atomics or another pass.
// Products that only dK depends on keep 2^-16 of a term for 16-bit dK; dQ is needed to fp32 for dg.  That leaves dK within 3e-5 of its RMS, also where
// tokens repeat a key with beta = 1 and no decay and terms cancel; fp16's own rounding is 2e-4 of it on average.
// d < 128: a tile column's matrices (x1, x2) are indexed at run time and stand in private memory, 272 bytes a lane at d = 64, 528 at 32, so
// all their products pass through it: 50 us of the 86 that 2 sequences of up to 150 tokens take, fp32, d = 64.
template <typename TIn, typename TOut, int D>
__global__ __launch_bounds__(2 * D, 1) void kvb_scan_grad_kernel(const GradArgs ga)
{
    constexpr int NWV = D / 32, KS = D / 32, NP = PIECES<TIn>, NO = PIECES<TOut>, LK = sizeof(TIn) == 2 ? 2 : FULL, ITS = 4 / NWV;
    constexpr int ROWS = 4 * KS * 64;   // 16-byte words of a piece of 64 rows of D
    constexpr int ONE = (NO + FULL + LK) * ROWS, W = 512, TWO = (FULL + LK) * W + 2 * NP * ROWS;
    using Tok = TokenTile<TIn, D, NWV>;
    // (d < 128: the matrices beside the rows, for the few waves have several tile columns to get rid of)
    constexpr bool APART = D < 128;
    constexpr int BESIDE = ONE > 2 * NP * ROWS ? ONE : 2 * NP * ROWS;
    constexpr int UNROLL = NP == FULL ? 1 : KS;   // (registers)
    constexpr int SHARED = APART ? BESIDE + (FULL + LK) * W : ONE > TWO ? ONE : TWO;
    // bf16: what the next v-head's start needs from memory is asked for while this one's products with matrices run, its states a step
    // ahead (with more pieces there are no registers for it), and keys and queries stay in LDS for all v-heads (nor room for that).
    constexpr bool AHEAD = NP == 1 && NO == 1;
    __shared__ uint4 lds[SHARED + (AHEAD ? 2 * ROWS : 0)];
    __shared__ float sums[5][4][SC], square[4];   // the tokens' dO'.E, Z.dV and Q.dQ', E.D' and E.(rest K dS1), and <dS1, S0>, by waves
    __shared__ double cs[SC];
    uint4 *oimg = lds, *eimg = oimg + NO * ROWS, *vimg = eimg + FULL * ROWS;
    uint4 *w1 = lds + (APART ? BESIDE : 0), *w2 = w1 + FULL * W, *kimg = AHEAD ? lds + SHARED : APART ? lds : w2 + LK * W, *qimg = kimg + NP * ROWS;
    const ScanArgs &a = ga.f;
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid / 64), lane = tid % 64, m = lane % 16, g = lane / 16;
    const int w = blockIdx.x / a.Hk, hk = blockIdx.x - w * a.Hk;
    const ChunkAt at = chunk_at(a.start, a.n_tokens, a.B, w);
    if (at.n == 0 || state_row(a.slot, a.n_slots, at.b) < 0)
        return;
    const uint32_t kst = a.k_stride * sizeof(TIn), qst = a.q_stride * sizeof(TIn), vst = a.v_stride * sizeof(TIn), ost = a.Hv * D * sizeof(TOut);
    const Buffer kb = head_rows<TIn, D>(static_cast<const TIn *>(a.k) + at.first * a.k_stride + hk * D, a.k_stride, at.n);
    const Buffer qb = head_rows<TIn, D>(static_cast<const TIn *>(a.q) + at.first * a.q_stride + hk * D, a.q_stride, at.n);
    Tok kt, qt;
    f32x4_t dq[2][4] = {}, dk[2][4] = {};
    const int mine = 32 * wave + 8 * g;   // the lane's first column: of the rows it stages and of what it stores
    Raw8<TIn> v[4];
    Raw8<TOut> o[4];
    Raw8<float> z[4], d[4], sraw[2][2], draw[2][2];
    float gamma[4], rest[4], beta[4], g1, parts[2][(D / 16 + NWV - 1) / NWV];   // (gamma .. of token 16 nt + m)
    auto load_head = [&](int h) {
        const int hv = hk * a.r + h;
        const size_t unit = (size_t)w * a.Hv + hv;
        const Buffer vb = head_rows<TIn, D>(static_cast<const TIn *>(a.v) + at.first * a.v_stride + hv * D, a.v_stride, at.n);
        const Buffer ob = head_rows<TOut, D>(static_cast<const TOut *>(ga.dout) + ((size_t)at.first * a.Hv + hv) * D, (int64_t)a.Hv * D, at.n);
        const Buffer zb(a.z + unit * SC * D, 4 * SC * D), db(ga.dd + unit * SC * D, 4 * SC * D), gb(a.prep + unit * GRAD_PREP, 4 * SCAN_GATES);
        const Buffer pb(ga.part + unit * GRAD_PARTS, 4 * GRAD_PARTS);
        g1 = a.g[(size_t)(at.first + min(lane, at.n - 1)) * a.Hv + hv];
#pragma unroll
        for (int rt = 0; rt < 4; ++rt) {
            const int i = 16 * rt + m;
            gamma[rt] = __uint_as_float(gb.load4(4 * i));
            rest[rt] = __uint_as_float(gb.load4(4 * (SC + i)));
            beta[rt] = __uint_as_float(gb.load4(4 * (2 * SC + i)));
            z[rt] = load_raw8<float>(zb, (i * D + mine) * 4);
            d[rt] = load_raw8<float>(db, (i * D + mine) * 4);
            v[rt] = load_raw8<TIn>(vb, i * vst + mine * (uint32_t)sizeof(TIn));
            o[rt] = load_raw8<TOut>(ob, i * ost + mine * (uint32_t)sizeof(TOut));
        }
#pragma unroll
        for (int i = 0; i < (D / 16 + NWV - 1) / NWV; ++i)   // (D / 16 is a multiple of NWV)
#pragma unroll
            for (int j = 0; j < 2; ++j)
                parts[j][i] = __uint_as_float(pb.load4(4 * (((wave + NWV * i) * 2 + j) * SC + lane)));
    };
    auto load_states = [&](size_t unit, int ks, int to) {
        const Buffer sb(a.s0 + unit * D * D, 4 * D * D), dsb(ga.ds + unit * D * D, 4 * D * D);
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const uint32_t from = (state_row_of(2 * wave + t, m / 4, m % 4) * D + 32 * ks + 8 * g) * 4;
            sraw[to][t] = load_raw8<float>(sb, from);
            draw[to][t] = load_raw8<float>(dsb, from);
        }
    };
    if constexpr (AHEAD) {
        kt.load(kb, kst, wave, lane);
        qt.load(qb, qst, wave, lane);
        load_head(0);
        kt.store(kimg, wave, lane);
        qt.store(qimg, wave, lane);
    }
    for (int h = 0; h < a.r; ++h) {
        const int hv = hk * a.r + h;
        const size_t unit = (size_t)w * a.Hv + hv;
        const float *gates = a.prep + unit * GRAD_PREP;
        if constexpr (!AHEAD)
            load_head(h);
        const float last = __shfl(gamma[3], 15);   // (of token 63)
        if constexpr (NP < FULL)
            load_states(unit, 0, 0);
        if (wave == 0)
            cs[lane] = sum_below(lane < at.n ? log2_gate(g1) : 0.0);
        {   // the tokens' rows: 16 columns of 32 a lane group, tile by tile
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                float x = 0.0f;
#pragma unroll
                for (int i = 0; i < (D / 16 + NWV - 1) / NWV; ++i)
                    x += parts[j][i];
                sums[3 + j][wave][lane] = x;
            }
#pragma unroll
            for (int rt = 0; rt < 4; ++rt) {
                float ex[8], dx[8], zx[8], ox[8], oe = 0.0f, zd = 0.0f;
                unpack8(z[rt], zx);
                unpack8(d[rt], dx);
                unpack8(v[rt], ex);
                unpack8(o[rt], ox);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    ex[j] += zx[j];
                    dx[j] *= beta[rt];
                    oe = fmaf(ox[j], ex[j], oe);
                    zd = fmaf(zx[j], dx[j], zd);
                }
                uint4 po[NO], pe[FULL], pv[LK];
                cut_raw(o[rt], po);
                cut8(ex, pe);
                cut8(dx, pv);
                const int to = (rt * KS + wave) * 64 + lane;
#pragma unroll
                for (int j = 0; j < NO; ++j)
                    oimg[j * ROWS + to] = po[j];
#pragma unroll
                for (int j = 0; j < FULL; ++j)
                    eimg[j * ROWS + to] = pe[j];
#pragma unroll
                for (int j = 0; j < LK; ++j)
                    vimg[j * ROWS + to] = pv[j];
                oe += __shfl_xor(oe, 16);
                zd += __shfl_xor(zd, 16);
                oe += __shfl_xor(oe, 32);
                zd += __shfl_xor(zd, 32);
                if (g == 0) {
                    sums[0][wave][16 * rt + m] = a.scale * oe;
                    sums[1][wave][16 * rt + m] = zd;
                }
            }
        }
        lds_barrier();
        // against the states: S0 dO', S0 dV', dS1 E'
        f32x4_t q0[2][4] = {}, k0[2][4] = {}, k1[2][4] = {};
        float sq = 0.0f;
#pragma unroll UNROLL   // (the register sets take turns)
        for (int ks = 0; ks < KS; ++ks) {
            if constexpr (NP == FULL)
                load_states(unit, ks, 0);
            else if (ks + 1 < KS)
                load_states(unit, ks + 1, (ks + 1) % 2);
            uint4 ps[2][FULL], pd[2][LK];
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                float x[8], y[8];
                unpack8(sraw[NP == FULL ? 0 : ks % 2][t], x);
                unpack8(draw[NP == FULL ? 0 : ks % 2][t], y);
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    sq = fmaf(x[j], y[j], sq);
                cut8(x, ps[t]);
                cut8(y, pd[t]);
            }
            uint4 po[4][NO], pe[4][LK], pv[4][LK];
#pragma unroll
            for (int nt = 0; nt < 4; ++nt) {
                const int from = (nt * KS + ks) * 64 + lane;
#pragma unroll
                for (int j = 0; j < NO; ++j)
                    po[nt][j] = oimg[j * ROWS + from];
#pragma unroll
                for (int j = 0; j < LK; ++j) {
                    pe[nt][j] = eimg[j * ROWS + from];
                    pv[nt][j] = vimg[j * ROWS + from];
                }
            }
            mma(q0, ps, po);
            mma<LK>(k0, ps, pv);
            mma<LK>(k1, pd, pe);
        }
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int nt = 0; nt < 4; ++nt) {
                q0[t][nt] *= a.scale * gamma[nt];
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    dk[t][nt][r] += rest[nt] * beta[nt] * k1[t][nt][r] - gamma[nt] * k0[t][nt][r];
            }
#pragma unroll
        for (int s = 1; s < 64; s *= 2)
            sq += __shfl_xor(sq, s);
        if (lane == 0)
            square[wave] = sq;
        auto put_matrices = [&](int it, const f32x4_t (&y1)[4], const f32x4_t (&y2)[4]) {
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                const int to = ((wave + NWV * it) * 2 + s) * 64 + lane;
                float x[8];
                uint4 p1[FULL], p2[LK];
                pair8(y1[2 * s], y1[2 * s + 1], x);
                cut8(x, p1);
                pair8(y2[2 * s], y2[2 * s + 1], x);
                cut8(x, p2);
#pragma unroll
                for (int j = 0; j < FULL; ++j)
                    w1[j * W + to] = p1[j];
#pragma unroll
                for (int j = 0; j < LK; ++j)
                    w2[j * W + to] = p2[j];
            }
        };
        // W1' (without its diagonal) and -W2', tile columns `wave`, wave + NWV ..: rows j, columns i
        f32x4_t x1[ITS][4] = {}, x2[ITS][4] = {};
#pragma unroll (APART ? 1 : ITS)
        for (int it = 0; it < ITS; ++it) {
            const int tile = wave + NWV * it;
#pragma unroll UNROLL
            for (int ks = 0; ks < KS; ++ks) {
                const int from = (tile * KS + ks) * 64 + lane;
                uint4 po[1][NO], pv[1][LK], pe[4][FULL];
#pragma unroll
                for (int j = 0; j < NO; ++j)
                    po[0][j] = oimg[j * ROWS + from];
#pragma unroll
                for (int j = 0; j < LK; ++j)
                    pv[0][j] = vimg[j * ROWS + from];
#pragma unroll
                for (int jt = 0; jt < 4; ++jt)
#pragma unroll
                    for (int j = 0; j < FULL; ++j)
                        pe[jt][j] = eimg[j * ROWS + (jt * KS + ks) * 64 + lane];
                f32x4_t c1[4][1], c2[4][1];
#pragma unroll
                for (int jt = 0; jt < 4; ++jt) {
                    c1[jt][0] = x1[it][jt];
                    c2[jt][0] = x2[it][jt];
                }
                mma(c1, pe, po);
                mma<LK>(c2, pe, pv);
#pragma unroll
                for (int jt = 0; jt < 4; ++jt) {
                    x1[it][jt] = c1[jt][0];
                    x2[it][jt] = c2[jt][0];
                }
            }
            const int i = 16 * tile + m;
            const double ci = cs[i];
#pragma unroll
            for (int jt = 0; jt < 4; ++jt) {
                const float4 b4 = *reinterpret_cast<const float4 *>(gates + 2 * SC + 16 * jt + 4 * g);
                const float bj[4] = {b4.x, b4.y, b4.z, b4.w};
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int j = 16 * jt + 4 * g + r;
                    const float d = decay(ci - cs[j]) * bj[r];
                    x1[it][jt][r] = i > j ? a.scale * d * x1[it][jt][r] : 0.0f;
                    x2[it][jt][r] = i > j ? -d * x2[it][jt][r] : 0.0f;
                }
            }
            if constexpr (APART)
                put_matrices(it, x1[it], x2[it]);
        }
        lds_barrier();
        if constexpr (!APART) {
#pragma unroll
            for (int it = 0; it < ITS; ++it)
                put_matrices(it, x1[it], x2[it]);
        }
        if constexpr (!AHEAD) {
            kt.load(kb, kst, wave, lane);
            qt.load(qb, qst, wave, lane);
            kt.store(kimg, wave, lane);
            qt.store(qimg, wave, lane);
        }
        const float beta_now[4] = {beta[0], beta[1], beta[2], beta[3]};
        if constexpr (AHEAD)
            load_head(min(h + 1, a.r - 1));
        lds_barrier();
        // dQ' += K' W1', dK' -= K' W2' (summed over j); dK' += Q' W1 - K' W2 (summed over i)
        static_for<2>([&](auto step) {
            constexpr int s = step(), FROM = 2 * s;   // columns from 32 s on have something in rows 32 s ..
            uint4 fk[2][NP], fq[2][NP];
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                Tok::columns(kimg, 2 * wave + t, s, lane, fk[t]);
                Tok::columns(qimg, 2 * wave + t, s, lane, fq[t]);
            }
            {
                uint4 b1[4 - FROM][FULL], b2[4 - FROM][LK];
                f32x4_t cq[2][4 - FROM], ck[2][4 - FROM];
#pragma unroll
                for (int it = FROM; it < 4; ++it) {
                    const int from = (it * 2 + s) * 64 + lane;
#pragma unroll
                    for (int j = 0; j < FULL; ++j)
                        b1[it - FROM][j] = w1[j * W + from];
#pragma unroll
                    for (int j = 0; j < LK; ++j)
                        b2[it - FROM][j] = w2[j * W + from];
#pragma unroll
                    for (int t = 0; t < 2; ++t) {
                        cq[t][it - FROM] = q0[t][it];
                        ck[t][it - FROM] = dk[t][it];
                    }
                }
                mma(cq, fk, b1);
                mma<LK>(ck, fk, b2);
#pragma unroll
                for (int it = FROM; it < 4; ++it)
#pragma unroll
                    for (int t = 0; t < 2; ++t) {
                        q0[t][it] = cq[t][it - FROM];
                        dk[t][it] = ck[t][it - FROM];
                    }
            }
            {
                constexpr int TO = 2 * s + 2;   // rows 32 s .. have something in columns up to 32 s + 31
                uint4 b1[TO][LK], b2[TO][LK];
                f32x4_t ck[2][TO];
#pragma unroll
                for (int jt = 0; jt < TO; ++jt) {
#pragma unroll
                    for (int j = 0; j < LK; ++j) {
                        b1[jt][j] = transposed(w1 + j * W, jt, s, lane);
                        b2[jt][j] = transposed(w2 + j * W, jt, s, lane);
                    }
#pragma unroll
                    for (int t = 0; t < 2; ++t)
                        ck[t][jt] = dk[t][jt];
                }
                mma<LK>(ck, fq, b1);
                mma<LK>(ck, fk, b2);
#pragma unroll
                for (int jt = 0; jt < TO; ++jt)
#pragma unroll
                    for (int t = 0; t < 2; ++t)
                        dk[t][jt] = ck[t][jt];
            }
        });
#pragma unroll
        for (int nt = 0; nt < 4; ++nt) {
            float x[8], y[8], dot = 0.0f, oe = 0.0f;
            if constexpr (AHEAD) {   // (their images as first operands: 8 columns of a token a lane)
                uint4 fq[1], fk[1];
                Tok::rows(qimg, nt, wave, lane, fq);
                Tok::rows(kimg, nt, wave, lane, fk);
                unpack8(Raw8<TIn>{fq[0]}, x);
                unpack8(Raw8<TIn>{fk[0]}, y);
            } else {
                unpack8(load_raw8<TIn>(qb, (16 * nt + m) * qst + mine * (uint32_t)sizeof(TIn)), x);
                unpack8(load_raw8<TIn>(kb, (16 * nt + m) * kst + mine * (uint32_t)sizeof(TIn)), y);
            }
#pragma unroll
            for (int v = 0; v < NWV; ++v)
                oe += sums[0][v][16 * nt + m];
            oe *= beta_now[nt];   // W1's diagonal
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                dot = fmaf(x[j], q0[j / 4][nt][j % 4], dot);
                dq[j / 4][nt][j % 4] += fmaf(oe, y[j], q0[j / 4][nt][j % 4]);
                dk[j / 4][nt][j % 4] = fmaf(oe, x[j], dk[j / 4][nt][j % 4]);
            }
            dot += __shfl_xor(dot, 16);
            dot += __shfl_xor(dot, 32);
            if (g == 0)
                sums[2][wave][16 * nt + m] = dot;
        }
        lds_barrier();
        if (wave == 0) {
            float oe = 0.0f, own_terms = 0.0f, total = 0.0f, in = 0.0f, on = 0.0f;
#pragma unroll
            for (int v = 0; v < NWV; ++v) {
                oe += sums[0][v][lane];
                own_terms += sums[1][v][lane] + sums[2][v][lane];
                total += square[v];
                in += sums[3][v][lane];
                on += sums[4][v][lane];
            }
            const float b1 = gates[2 * SC + lane];
            const float from_here = own_terms - b1 * in, before = b1 * on;   // (0 behind the chunk's end)
            const double upto = sum_below((double)from_here), all = __shfl(upto, 63), ahead = sum_below((double)before) - before;
            if (lane < at.n) {
                const size_t to = (size_t)(at.first + lane) * a.Hv + hv;
                ga.dbeta[to] = in + on + gates[3 * SC + lane] * oe;
                ga.dg[to] = (float)(all - upto + from_here + ahead + total * last);
            }
        }
        lds_barrier();
    }
    auto put = [&](void *to, int64_t stride, const f32x4_t (&x)[2][4]) {
        TIn *rows = static_cast<TIn *>(to) + at.first * stride + hk * D + mine;
#pragma unroll
        for (int nt = 0; nt < 4; ++nt)
            if (16 * nt + m < at.n) {
                TIn *p = rows + (16 * nt + m) * stride;
                if constexpr (sizeof(TIn) == 4) {
                    *reinterpret_cast<float4 *>(p) = make_float4(x[0][nt][0], x[0][nt][1], x[0][nt][2], x[0][nt][3]);
                    *reinterpret_cast<float4 *>(p + 4) = make_float4(x[1][nt][0], x[1][nt][1], x[1][nt][2], x[1][nt][3]);
                } else {
                    *reinterpret_cast<uint4 *>(p) = make_uint4(pack_pair<TIn>(x[0][nt][0], x[0][nt][1]), pack_pair<TIn>(x[0][nt][2], x[0][nt][3]),
                                                               pack_pair<TIn>(x[1][nt][0], x[1][nt][1]), pack_pair<TIn>(x[1][nt][2], x[1][nt][3]));
                }
            }
    };
    put(ga.dq, a.q_stride, dq);
    put(ga.dk, a.k_stride, dk);
}

template <typename TIn, typename TOut, int D>
void launch_scan_grad_sized(const GradArgs &a, hipStream_t stream)
{
    const int64_t chunks = scan_chunks(a.f.n_tokens, a.f.B);
    if (a.f.n_tokens > 0)
        launch_part(kvb_scan_prep_kernel<TIn, D, true>, true, false, chunks * a.f.Hv, 256, stream, a.f);
    if (a.f.n_tokens > 0)
        scan_split<TIn, D>(a.f, [&]<int NWV>(int64_t blocks) {
            launch_part(kvb_scan_kernel<TIn, float, D, NWV, true, false>, false, false, blocks, 64 * NWV, stream, a.f);
        });
    constexpr int NWV = D == 32 ? 2 : 4;   // (eight waves' slabs would not fit beside the images)
    launch_part(kvb_scan_reverse_kernel<TIn, TOut, D, NWV>, a.f.n_tokens == 0, a.f.n_tokens == 0, (int64_t)a.f.B * a.f.Hv * (D / (16 * NWV)), 64 * NWV, stream, a);
    if (a.f.n_tokens > 0)
        launch_part(kvb_scan_grad_kernel<TIn, TOut, D>, false, true, chunks * a.f.Hk, 2 * D, stream, a);
}
template <typename TIn, typename TOut>
void launch_scan_grad_typed(int d, const GradArgs &a, hipStream_t stream)
{
    if (d == 32)
        launch_scan_grad_sized<TIn, TOut, 32>(a, stream);
    else if (d == 64)
        launch_scan_grad_sized<TIn, TOut, 64>(a, stream);
    else
        launch_scan_grad_sized<TIn, TOut, 128>(a, stream);
}

}  // namespace kvb_impl
#endif  // KVB_SCAN_GRAD_KERNEL_H
