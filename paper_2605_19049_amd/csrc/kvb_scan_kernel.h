// kvb_scan: the gated delta rule over whole sequences (the mathematics and the images: kvb_scan_device.h).
#ifndef KVB_SCAN_KERNEL_H
#define KVB_SCAN_KERNEL_H

#include "kvb_scan_device.h"

namespace kvb_impl {

// M and P of one chunk for the v-heads of one qk-head: a workgroup of four waves.
// Products K K' and Q K' once for all of them: wave w has rows 16 w .. of both.  Then for each v-head G and P, and
// M = -(1 + G beta)^-1 G by 16 x 16 blocks: the diagonal blocks row by row in registers (each wave one), then wave J the blocks below
// its own,  M_IJ = -(1 + M_II beta) (G_IJ + sum_K G_IK beta M_KJ),  on the fp32 matrix instruction: the sums' registers
// are its second operand as they stand, if row 4 g + r is taken for what lane group g sums in its r-th step.
// c is summed in fp64, so that differences of it are good to fp32 whatever its size; a decay below exp(-1e5) counts as that (zero).
template <typename TIn, int D>
__global__ __launch_bounds__(256) void kvb_scan_prep_kernel(const ScanArgs a)
{
    constexpr int LD = SC + 4;
    __shared__ float gs[SC * LD], ps[SC * LD], td[4 * 16 * 20];
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid / 64), lane = tid % 64, m = lane % 16, g = lane / 16;
    const int w = blockIdx.x / a.Hk, hk = blockIdx.x - w * a.Hk;
    const ChunkAt at = chunk_at(a.start, a.n_tokens, a.B, w);
    if (at.n == 0)
        return;
    const TIn *k = static_cast<const TIn *>(a.k) + at.first * a.k_stride + hk * D;
    const TIn *q = static_cast<const TIn *>(a.q) + at.first * a.q_stride + hk * D;
    f32x4_t kk[4] = {}, qk[4] = {};
    const int own = min(16 * wave + m, at.n - 1);
#pragma unroll
    for (int ks = 0; ks < D / 32; ++ks) {
        const int col = 32 * ks + 8 * g;
        const Raw8<TIn> kr = load_raw8(k + own * a.k_stride + col), qr = load_raw8(q + own * a.q_stride + col);
        Raw8<TIn> br[4];
#pragma unroll
        for (int nt = 0; nt < 4; ++nt)
            br[nt] = load_raw8(k + min(16 * nt + m, at.n - 1) * a.k_stride + col);
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
    for (int h = 0; h < a.r; ++h) {
        const int hv = hk * a.r + h;
        float *prep = a.prep + ((size_t)w * a.Hv + hv) * SCAN_PREP;
        const size_t tok = (size_t)(at.first + min(lane, at.n - 1)) * a.Hv + hv;
        const float g1 = a.g[tok], b1 = a.beta[tok];
        const float gate = lane < at.n ? (g1 < -1e5f ? -1e5f : g1) : 0.0f, beta = lane < at.n ? b1 : 0.0f;
        double c = gate;
#pragma unroll
        for (int s = 1; s < 64; s *= 2) {
            const double below = __shfl_up(c, s);
            c += lane >= s ? below : 0.0;
        }
        if (wave == 0) {
            float *gates = prep + 2 * SCAN_MAT;
            const double last = __shfl(c, 63);
            gates[lane] = expf((float)c);
            gates[SC + lane] = lane < at.n ? expf((float)(last - c)) : 0.0f;
            gates[2 * SC + lane] = beta;
            gates[3 * SC + lane] = (float)c;
        }
        double ci[4];
#pragma unroll
        for (int r = 0; r < 4; ++r)
            ci[r] = __shfl(c, 16 * wave + 4 * g + r);
#pragma unroll
        for (int nt = 0; nt < 4; ++nt) {
            const int j = 16 * nt + m;
            const double cj = __shfl(c, j);
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int i = 16 * wave + 4 * g + r;
                const float decay = expf((float)(ci[r] - cj));
                gs[i * LD + j] = i > j && i < at.n ? decay * kk[nt][r] : 0.0f;
                ps[i * LD + j] = i >= j && i < at.n ? decay * qk[nt][r] : 0.0f;
            }
        }
        __syncthreads();
        // the diagonal block: lane m has column m of it (in all four lane groups)
        float x[16], y[16];
        const float *blk = gs + 16 * wave * (LD + 1);
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            float s = blk[i * LD + m];
#pragma unroll
            for (int l4 = 0; l4 < i; l4 += 4) {
                const float4 c4 = *reinterpret_cast<const float4 *>(blk + i * LD + l4);
                s = fmaf(c4.x, y[l4], s);
                s = l4 + 1 < i ? fmaf(c4.y, y[l4 + 1], s) : s;
                s = l4 + 2 < i ? fmaf(c4.z, y[l4 + 2], s) : s;
                s = l4 + 3 < i ? fmaf(c4.w, y[l4 + 3], s) : s;
            }
            x[i] = -s;
            y[i] = x[i] * __shfl(beta, 16 * wave + i);
        }
        const float bm = __shfl(beta, 16 * wave + m);
        f32x4_t diag;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            diag[r] = g == 0 ? x[r] : g == 1 ? x[4 + r] : g == 2 ? x[8 + r] : x[12 + r];
            td[(wave * 16 + 4 * g + r) * 20 + m] = (4 * g + r == m ? 1.0f : 0.0f) + diag[r] * bm;
        }
        __syncthreads();
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
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                mm[I][r] = I < wave ? 0.0f : I == wave ? diag[r] : -below[r];
                ym[I][r] = mm[I][r] * __shfl(beta, 16 * I + 4 * g + r);
            }
        }
        __syncthreads();
#pragma unroll
        for (int I = 0; I < 4; ++I)
#pragma unroll
            for (int r = 0; r < 4; ++r)
                gs[(16 * I + 4 * g + r) * LD + 16 * wave + m] = mm[I][r];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 3; ++i) {
            const int u = tid + 256 * i, of = u >= SCAN_UNITS, t = (of ? u - SCAN_UNITS : u) / 64;
            const int rt = t < 2 ? t : 1 + t / 2, s = t < 2 ? 0 : t % 2;
            const float *from = (of ? ps : gs) + (16 * rt + m) * LD + 32 * s + 4 * g;
            float4 *to = reinterpret_cast<float4 *>(prep + u * 8);
            to[0] = *reinterpret_cast<const float4 *>(from);
            to[1] = *reinterpret_cast<const float4 *>(from + 16);
        }
        __syncthreads();
    }
}

// The state from chunk to chunk: a workgroup has NWV waves of 16 NC columns each of one (sequence, v-head).
// A wave keeps its columns of the state in its sums' registers for the whole sequence; the chunk's
// K S and Q S, E and the state's update follow from each other within the wave (paired order).  Lane l % 16 = n has the columns
// NC n .. NC n + NC - 1 of the wave's.  What the next chunk needs from memory is requested a chunk ahead.
template <typename TIn, int D, int NC, int NWV>
__global__ __launch_bounds__(64 * NWV, 1) void kvb_scan_kernel(const ScanArgs a)
{
    constexpr int NTH = 64 * NWV, KT = D / 16, KS = D / 32, SPLIT = D / (16 * NC * NWV);
    using Tok = TokenTile<TIn, D, NWV>;
    using Mat = MatTile<2 * SCAN_UNITS, NTH>;
    __shared__ uint4 kimg[Tok::WORDS], qimg[Tok::WORDS], mats[FULL * 2 * SCAN_UNITS];
    __shared__ float4 gate[SCAN_GATES / 4];
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid / 64), lane = tid % 64, m = lane % 16, g = lane / 16;
    const int unit = blockIdx.x / SPLIT, part = blockIdx.x % SPLIT;
    const int b = unit / a.Hv, hv = unit - b * a.Hv, hk = hv / a.r;
    const int row = state_row(a.slot, a.n_slots, b);
    if (row < 0)
        return;
    const Span span = span_of(a.start, a.n_tokens, b);
    const int chunks = (span.len + SC - 1) / SC, col = (part * NWV + wave) * 16 * NC + NC * m;
    const size_t own = ((size_t)row * a.Hv + hv) * D * D + col;

    f32x4_t S[KT][NC];
#pragma unroll
    for (int t = 0; t < KT; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            if constexpr (NC == 2) {
                const float2 x = a.state0 ? *reinterpret_cast<const float2 *>(a.state0 + own + (16 * t + 4 * g + r) * D) : make_float2(0.0f, 0.0f);
                S[t][0][r] = x.x;
                S[t][1][r] = x.y;
            } else {
                S[t][0][r] = a.state0 ? a.state0[own + (16 * t + 4 * g + r) * D] : 0.0f;
            }
        }

    const TIn *kp = static_cast<const TIn *>(a.k) + span.first * a.k_stride + hk * D;
    const TIn *qp = static_cast<const TIn *>(a.q) + span.first * a.q_stride + hk * D;
    const TIn *vp = static_cast<const TIn *>(a.v) + span.first * a.v_stride + hv * D + col;
    const float *prep = a.prep + ((size_t)first_chunk(span, b) * a.Hv + hv) * SCAN_PREP;
    const size_t prep_step = (size_t)a.Hv * SCAN_PREP;

    Tok knext, qnext;
    Mat mnext;
    float gnext[SCAN_GATES / NTH];
    float vnext[4][4][NC];
    auto request = [&](int c) {
        const int n = min(SC, span.len - c * SC);
        knext.load(kp + (int64_t)c * SC * a.k_stride, a.k_stride, n, wave, lane);
        qnext.load(qp + (int64_t)c * SC * a.q_stride, a.q_stride, n, wave, lane);
        mnext.load(prep + c * prep_step, tid);
#pragma unroll
        for (int i = 0; i < SCAN_GATES / NTH; ++i)
            gnext[i] = prep[c * prep_step + 2 * SCAN_MAT + tid + NTH * i];
        const TIn *v = vp + (int64_t)c * SC * a.v_stride;
#pragma unroll
        for (int rt = 0; rt < 4; ++rt)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const TIn *p = v + min(16 * rt + 4 * g + r, n - 1) * a.v_stride;
                if constexpr (NC == 2) {
                    const float2 x = unpack2r(load_raw2(p));
                    vnext[rt][r][0] = x.x;
                    vnext[rt][r][1] = x.y;
                } else {
                    vnext[rt][r][0] = to_f32(*p);
                }
            }
    };
    if (chunks > 0)
        request(0);
    for (int c = 0; c < chunks; ++c) {
        const int n = min(SC, span.len - c * SC);
        knext.store(kimg, wave, lane);
        qnext.store(qimg, wave, lane);
        mnext.store(mats, tid);
#pragma unroll
        for (int i = 0; i < SCAN_GATES / NTH; ++i)
            reinterpret_cast<float *>(gate)[tid + NTH * i] = gnext[i];
        f32x4_t E[4][NC], O[4][NC], y[4][NC];
#pragma unroll
        for (int rt = 0; rt < 4; ++rt)
#pragma unroll
            for (int ct = 0; ct < NC; ++ct)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    E[rt][ct][r] = vnext[rt][r][ct];
                    O[rt][ct][r] = 0.0f;
                    y[rt][ct][r] = 0.0f;
                }
        __syncthreads();
        if (c + 1 < chunks)
            request(c + 1);
        // y = K S, O = Q S
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            uint4 s[NC][FULL];
#pragma unroll
            for (int ct = 0; ct < NC; ++ct) {
                float x[8];
                pair8(S[2 * ks][ct], S[2 * ks + 1][ct], x);
                cut8(x, s[ct]);
            }
#pragma unroll
            for (int rt = 0; rt < 4; ++rt) {
                uint4 f[PIECES<TIn>];
                Tok::rows(kimg, rt, ks, lane, f);
#pragma unroll
                for (int ct = 0; ct < NC; ++ct)
                    mma(y[rt][ct], f, s[ct]);
                Tok::rows(qimg, rt, ks, lane, f);
#pragma unroll
                for (int ct = 0; ct < NC; ++ct)
                    mma(O[rt][ct], f, s[ct]);
            }
        }
        // Y = V - gamma y, y = beta Y, E = Y + M y
#pragma unroll
        for (int rt = 0; rt < 4; ++rt) {
            const float4 ga = gate[4 * rt + g], be = gate[32 + 4 * rt + g];
            const float gm[4] = {ga.x, ga.y, ga.z, ga.w}, bt[4] = {be.x, be.y, be.z, be.w};
#pragma unroll
            for (int ct = 0; ct < NC; ++ct)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    E[rt][ct][r] = fmaf(-gm[r], y[rt][ct][r], E[rt][ct][r]);
                    O[rt][ct][r] *= gm[r];
                    y[rt][ct][r] = bt[r] * E[rt][ct][r];
                }
        }
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            uint4 p[NC][FULL];
#pragma unroll
            for (int ct = 0; ct < NC; ++ct) {
                float x[8];
                pair8(y[2 * s][ct], y[2 * s + 1][ct], x);
                cut8(x, p[ct]);
            }
#pragma unroll
            for (int rt = 0; rt < 4; ++rt)
                if (has_tile<false>(rt, s)) {
                    uint4 f[FULL];
                    Mat::tile(mats, tile_of<false>(rt, s), lane, f);
#pragma unroll
                    for (int ct = 0; ct < NC; ++ct)
                        mma(E[rt][ct], f, p[ct]);
                }
        }
        // O += P beta E, S = exp(c_last) S + K' rest beta E
        const float last = reinterpret_cast<const float *>(gate)[SC - 1];
#pragma unroll
        for (int t = 0; t < KT; ++t)
#pragma unroll
            for (int ct = 0; ct < NC; ++ct)
                S[t][ct] *= last;
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            uint4 p[NC][FULL], e[NC][FULL];
#pragma unroll
            for (int ct = 0; ct < NC; ++ct) {
                float x[8];
                pair8(E[2 * s][ct], E[2 * s + 1][ct], x);
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const float4 be = gate[32 + 8 * s + 4 * h + g];
                    x[4 * h] *= be.x;
                    x[4 * h + 1] *= be.y;
                    x[4 * h + 2] *= be.z;
                    x[4 * h + 3] *= be.w;
                }
                cut8(x, p[ct]);
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const float4 re = gate[16 + 8 * s + 4 * h + g];
                    x[4 * h] *= re.x;
                    x[4 * h + 1] *= re.y;
                    x[4 * h + 2] *= re.z;
                    x[4 * h + 3] *= re.w;
                }
                cut8(x, e[ct]);
            }
#pragma unroll
            for (int t = 0; t < KT; ++t) {
                uint4 f[PIECES<TIn>];
                Tok::columns(kimg, t, s, lane, f);
#pragma unroll
                for (int ct = 0; ct < NC; ++ct)
                    mma(S[t][ct], f, e[ct]);
            }
#pragma unroll
            for (int rt = 0; rt < 4; ++rt)
                if (has_tile<false>(rt, s)) {
                    uint4 f[FULL];
                    Mat::tile(mats, SCAN_TILES + tile_of<false>(rt, s), lane, f);
#pragma unroll
                    for (int ct = 0; ct < NC; ++ct)
                        mma(O[rt][ct], f, p[ct]);
                }
        }
        const Out<TIn> out{a.out, a.out_wide != 0};
#pragma unroll
        for (int rt = 0; rt < 4; ++rt)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int i = 16 * rt + 4 * g + r;
                const size_t to = ((size_t)(span.first + c * SC + i) * a.Hv + hv) * D + col;
                if (i < n) {
                    if constexpr (NC == 2)
                        out.put2(to, a.scale * O[rt][0][r], a.scale * O[rt][1][r]);
                    else
                        out.put1(to, a.scale * O[rt][0][r]);
                }
            }
        __syncthreads();
    }
    if (a.state1)
#pragma unroll
        for (int t = 0; t < KT; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                float *to = a.state1 + own + (16 * t + 4 * g + r) * D;
                if constexpr (NC == 2)
                    *reinterpret_cast<float2 *>(to) = make_float2(S[t][0][r], S[t][1][r]);
                else
                    *to = S[t][0][r];
            }
}

template <typename TIn, int D>
void launch_scan_sized(const ScanArgs &a, hipStream_t stream)
{
    constexpr int NWV = D >= 64 ? 4 : 2;
    if (a.n_tokens > 0)
        launch_part(kvb_scan_prep_kernel<TIn, D>, true, false, scan_chunks(a.n_tokens, a.B) * a.Hk, 256, stream, a);
    launch_part(kvb_scan_kernel<TIn, D, 1, NWV>, a.n_tokens == 0, true, (int64_t)a.B * a.Hv * (D / (16 * NWV)), 64 * NWV, stream, a);
}
template <typename TIn>
void launch_scan_typed(int d, const ScanArgs &a, hipStream_t stream)
{
    if (d == 32)
        launch_scan_sized<TIn, 32>(a, stream);
    else if (d == 64)
        launch_scan_sized<TIn, 64>(a, stream);
    else
        launch_scan_sized<TIn, 128>(a, stream);
}

}  // namespace kvb_impl
#endif  // KVB_SCAN_KERNEL_H
