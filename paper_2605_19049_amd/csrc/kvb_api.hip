// Host side of the library: argument checks (all before the first HIP call), the extern "C" entry
// points of include/kvb.h, the kernel timer.
#include "kvb_accept_device.h"
#include "kvb_layer_device.h"

#include <cmath>

namespace kvb_impl {

thread_local kvb_timer *g_armed = nullptr;
thread_local hipError_t g_launch_status = hipSuccess;

}  // namespace kvb_impl

using namespace kvb_impl;

namespace {

thread_local hipError_t g_last_hip_error = hipSuccess;

bool aligned(const void *p, size_t n) { return (reinterpret_cast<uintptr_t>(p) % n) == 0; }

int check_common(const kvb_shape *sh, const kvb_store *st, const int32_t *slot)
{
    if (!sh || !st || !slot)
        return KVB_EINVAL;
    if (sh->B < 0 || sh->Hk <= 0 || sh->Hv <= 0 || sh->Hv % sh->Hk != 0)
        return KVB_EINVAL;
    if (sh->dk <= 0 || sh->dv <= 0)
        return KVB_EINVAL;
    if (sh->cap < 1 || sh->cap > KVB_MAX_CAP)
        return KVB_EINVAL;
    if (st->n_slots <= 0 || !st->buf_k || !st->buf_u || !st->buf_G || !st->fill)
        return KVB_EINVAL;
    if (st->block_table) {   // paged record buffers
        const int bs = st->block_size;
        if (bs < 8 || bs > KVB_MAX_CAP || (bs & (bs - 1)) != 0)
            return KVB_EINVAL;
        if (st->max_blocks < 1 || st->max_blocks > KVB_MAX_BLOCKS || st->n_blocks < 1)
            return KVB_EINVAL;
        if ((long long)bs * st->max_blocks < sh->cap || !aligned(st->block_table, 4))
            return KVB_EINVAL;
    }
    if (!aligned(st->state, 16) || !aligned(st->buf_k, 16) || !aligned(st->buf_u, 16) ||
        !aligned(st->buf_G, 4) || !aligned(st->fill, 4) || !aligned(st->status, 4) || !aligned(slot, 4))
        return KVB_EINVAL;
    if ((long long)sh->B * sh->Hv > 0x7FFFFFFFLL)
        return KVB_EINVAL;
    if (sh->in_dtype != KVB_F32 && sh->in_dtype != KVB_BF16 && sh->in_dtype != KVB_F16)
        return KVB_EUNSUPPORTED;
    // records and outputs: fp32, or the 16-bit type of the inputs
    if (sh->out_dtype != KVB_F32 && (sh->in_dtype == KVB_F32 || sh->out_dtype != sh->in_dtype))
        return KVB_EUNSUPPORTED;
    if (sh->rec_dtype != KVB_F32 && (sh->in_dtype == KVB_F32 || sh->rec_dtype != sh->in_dtype))
        return KVB_EUNSUPPORTED;
    if (sh->dk != sh->dv || (sh->dk != 32 && sh->dk != 64 && sh->dk != 128))
        return KVB_EUNSUPPORTED;
    return KVB_OK;
}

int check_tokens(const void *q, const void *k, const void *v, const float *g, const float *beta, const void *out)
{
    if (!q || !k || !v || !g || !beta || !out)
        return KVB_EINVAL;
    if (!aligned(q, 16) || !aligned(k, 16) || !aligned(v, 16) || !aligned(out, 16) || !aligned(g, 4) ||
        !aligned(beta, 4))
        return KVB_EINVAL;
    return KVB_OK;
}

// Whether the state should be streamed past the caches: the caller's hint, else by this
// call's own state footprint against the 256 MB last-level cache.  For decoding and verification
// the switch sits at 288 MiB: a state of 256 MiB re-read every step still finds most of itself
// in the cache and runs faster with plain loads (kvb_decode_flush at C = 16: 49 against 53 us per
// step), at 288 MiB the two are level (59 us), at 320 MiB streaming wins (65 against 71).  kvb_flush
// reads and writes the state, twice the lines through the cache: measured, streaming wins from
// about 200 MiB of state on (16 records: 65 against 71 us at 192 MiB, 88 against 84 at 224 MiB;
// 64 records: 139 against 107 us at 256 MiB), so its switch sits at 192 MiB.
bool stream_state(const kvb_shape *sh, const kvb_store *st, double limit_mib = 288.0)
{
    if (st->flags & KVB_STORE_STREAM)
        return true;
    if (st->flags & KVB_STORE_RESIDENT)
        return false;
    const double bytes = 4.0 * sh->B * sh->Hv * sh->dk * sh->dv;
    return bytes > limit_mib * 1024 * 1024;
}

Store dev_store(const kvb_store *st)
{
    return Store{st->state, st->buf_k, st->buf_u, st->buf_G, st->fill, st->status, st->n_slots,
                 st->block_table, st->block_table ? st->block_size : 0, st->block_table ? st->max_blocks : 1,
                 st->block_table ? st->n_blocks : 0, st->flags & KVB_STORE_FILL_APART ? 5 : 0};
}

// The status of the launch this thread has just made (what the launch call itself returned:
// an error some other library left behind in the runtime is neither reported nor cleared).
int finish_launch()
{
    const hipError_t e = g_launch_status;
    if (e != hipSuccess) {
        g_last_hip_error = e;
        return KVB_EHIP;
    }
    return KVB_OK;
}

// Every compute entry point ends with no timer armed: a call that returns before it launches
// (bad arguments, B = 0) must not leave its timer to some later, unrelated launch.
struct DisarmOnExit {
    ~DisarmOnExit() { g_armed = nullptr; }
};

int step_common(const kvb_shape *sh, const kvb_store *st, const int32_t *slot, int T, const void *q,
                const void *k, const void *v, const float *g, const float *beta, void *out, void *stream,
                int advance, int threshold = 0, const int32_t *parent = nullptr)
{
    int rc = check_common(sh, st, slot);
    if (rc != KVB_OK)
        return rc;
    rc = check_tokens(q, k, v, g, beta, out);
    if (rc != KVB_OK)
        return rc;
    if (T < 1 || T > KVB_MAX_DRAFTS || T > sh->cap)
        return KVB_EINVAL;
    if (sh->B == 0)
        return KVB_OK;
    StepArgs a{dev_store(st), slot, q, k, v, g, beta, out, sh->out_dtype == KVB_F32, sh->Hk, sh->Hv, sh->Hv / sh->Hk, sh->cap, T,
               sh->scale, advance, threshold, stream_state(sh, st) ? 1 : 0,
               // chain: g stands in as a readable array of at least B*T words whose values are ignored
               parent ? parent : reinterpret_cast<const int32_t *>(g), parent ? 1 : 0};
    const int blocks = sh->B * sh->Hv;
    // (kvb_verify steps from draft to draft in 32 bits of bytes)
    if (T > 1 && (long long)sh->Hv * sh->dv * (sh->in_dtype == KVB_F32 ? 4 : 2) > 0xFFFFFFFFLL)
        return KVB_EINVAL;
    if (advance && step_workgroups(a, sh->dk, sh->in_dtype == KVB_F32, blocks) > MAX_FILL_WG)
        return KVB_EINVAL;
    hipStream_t hs = static_cast<hipStream_t>(stream);
    g_launch_status = hipSuccess;
    if (T > 1)   // several drafts: the matrix-core kernel (the head size was checked above)
        rc = dispatch_types(sh->in_dtype, sh->rec_dtype, [&]<typename TIn, typename TRec>() {
            launch_verify_typed<TIn, TRec>(sh->dk, a, blocks, hs);
        });
    else
        rc = dispatch_types(sh->in_dtype, sh->rec_dtype, [&]<typename TIn, typename TRec>() {
            launch_step_typed<TIn, TRec>(sh->dk, a, blocks, hs);
        });
    if (rc != KVB_OK)
        return rc;
    return finish_launch();
}

// The element types and head sizes of a scan (cap and rec_dtype of the shape mean nothing there), and its sequences.
int check_seqs(const kvb_shape *sh, const kvb_seqs *sq)
{
    if (!sh || !sq)
        return KVB_EINVAL;
    if (sh->B < 0 || sh->Hk <= 0 || sh->Hv <= 0 || sh->Hv % sh->Hk != 0 || sh->dk <= 0 || sh->dv <= 0)
        return KVB_EINVAL;
    if (sq->n_tokens < 0 || sq->n_slots < 0)
        return KVB_EINVAL;
    if (sh->in_dtype != KVB_F32 && sh->in_dtype != KVB_BF16 && sh->in_dtype != KVB_F16)
        return KVB_EUNSUPPORTED;
    if (sh->out_dtype != KVB_F32 && (sh->in_dtype == KVB_F32 || sh->out_dtype != sh->in_dtype))
        return KVB_EUNSUPPORTED;
    if (sh->dk != sh->dv || (sh->dk != 32 && sh->dk != 64 && sh->dk != 128))
        return KVB_EUNSUPPORTED;
    const int64_t size = sh->in_dtype == KVB_F32 ? 4 : 2, width[3] = {(int64_t)sh->Hk * sh->dk, (int64_t)sh->Hk * sh->dk, (int64_t)sh->Hv * sh->dv};
    const int64_t stride[3] = {sq->q_stride, sq->k_stride, sq->v_stride};
    for (int i = 0; i < 3; ++i)   // (64 rows of 2^26 bytes in 32 bits)
        if (width[i] * 4 > 1 << 26 || (stride[i] != 0 && (stride[i] < width[i] || stride[i] > 1 << 26 || stride[i] * size > 1 << 26 || stride[i] * size % 16 != 0)))
            return KVB_EINVAL;
    // one workgroup for each chunk and v-head, and up to eight for each sequence and v-head
    if (scan_chunks(sq->n_tokens, sh->B) > INT32_MAX / sh->Hv || (int64_t)sh->B * sh->Hv > INT32_MAX / 8)
        return KVB_EINVAL;
    return KVB_OK;
}
int check_seq_pointers(const kvb_shape *sh, const kvb_seqs *sq, const void *q, const void *k, const void *v, const float *g,
                       const float *beta, const float *state0, const void *work)
{
    if (!sq->start || !aligned(sq->start, 4) || !aligned(sq->slot, 4) || !aligned(state0, 16) || !aligned(work, 16))
        return KVB_EINVAL;
    if (sq->n_tokens > 0 && !work)
        return KVB_EINVAL;
    if (!aligned(q, 16) || !aligned(k, 16) || !aligned(v, 16) || !aligned(g, 4) || !aligned(beta, 4))
        return KVB_EINVAL;
    if (sq->n_tokens > 0 && (!q || !k || !v || !g || !beta))
        return KVB_EINVAL;
    return KVB_OK;
}

ScanArgs scan_args(const kvb_shape *sh, const kvb_seqs *sq, const void *q, const void *k, const void *v, const float *g, const float *beta,
                   const float *state0, float *state1, void *out, float *prep, float *s0, float *z)
{
    const int64_t qk = (int64_t)sh->Hk * sh->dk, vv = (int64_t)sh->Hv * sh->dv;
    return ScanArgs{q, k, v, g, beta, state0, state1, out, sq->start, sq->slot, prep, s0, z, sq->q_stride ? sq->q_stride : qk,
                    sq->k_stride ? sq->k_stride : qk, sq->v_stride ? sq->v_stride : vv, sh->B, sq->n_slots, sq->n_tokens, sh->Hk, sh->Hv,
                    sh->Hv / sh->Hk, sh->scale};
}

int64_t scan_work_bytes(const kvb_shape *sh, const kvb_seqs *sq)
{
    return 4 * scan_chunks(sq->n_tokens, sh->B) * sh->Hv * SCAN_PREP;
}

int64_t grad_work_bytes(const kvb_shape *sh, const kvb_seqs *sq)
{
    return 4 * scan_chunks(sq->n_tokens, sh->B) * sh->Hv * grad_floats(sh->dk);
}

int check_vocab(const kvb_vocab *vo)
{
    if (!vo || vo->B < 0 || vo->T < 1 || vo->T > KVB_MAX_DRAFTS || vo->V < 1 || vo->V > KVB_MAX_VOCAB)
        return KVB_EINVAL;
    if (vo->stride != 0 && (vo->stride < vo->V || vo->stride > INT32_MAX))
        return KVB_EINVAL;
    if (vo->dtype != KVB_F32 && vo->dtype != KVB_BF16 && vo->dtype != KVB_F16)
        return KVB_EUNSUPPORTED;
    if (vo->B > (1 << 20))
        return KVB_EINVAL;
    return KVB_OK;
}

int64_t conv_channels(const kvb_shape *sh) { return (int64_t)(2 * (int64_t)sh->Hk + sh->Hv) * sh->dk; }

// The shape (as far as it matters) and the taps of a convolution, without its tokens.
int check_taps(const kvb_shape *sh, const kvb_taps *ta)
{
    if (!sh || !ta || sh->B < 0 || sh->Hk <= 0 || sh->Hv <= 0 || sh->Hv % sh->Hk != 0 || sh->dk <= 0 || sh->dv <= 0)
        return KVB_EINVAL;
    if (sh->in_dtype != KVB_F32 && sh->in_dtype != KVB_BF16 && sh->in_dtype != KVB_F16)
        return KVB_EUNSUPPORTED;
    if (sh->dk != sh->dv || (sh->dk != 32 && sh->dk != 64 && sh->dk != 128))
        return KVB_EUNSUPPORTED;
    const int64_t C = conv_channels(sh), size = sh->in_dtype == KVB_F32 ? 4 : 2;
    if (C * 4 > 1 << 26)
        return KVB_EINVAL;
    if (!ta->weight || !aligned(ta->weight, 16) || !aligned(ta->bias, 16) || !aligned(ta->A_log, 4) || !aligned(ta->dt_bias, 4))
        return KVB_EINVAL;
    if (ta->x_stride != 0 && (ta->x_stride < C || ta->x_stride > 1 << 26 || ta->x_stride * size > 1 << 26 || ta->x_stride * size % 16 != 0))
        return KVB_EINVAL;
    for (const int64_t s : {ta->a_stride, ta->b_stride})
        if (s != 0 && (s < sh->Hv || s > 1 << 26))
            return KVB_EINVAL;
    if (ta->width < 1 || (ta->flags & ~KVB_CONV_UNIT) != 0 || !std::isfinite(ta->eps) || ((ta->flags & KVB_CONV_UNIT) && !(ta->eps >= KVB_MIN_EPS)))
        return KVB_EINVAL;
    return ta->width >= 2 && ta->width <= 4 ? KVB_OK : KVB_EUNSUPPORTED;
}
// The threads of a launch are counted in 32 bits: 4 waves each that the last workgroup of four may have too many
constexpr int64_t MOST_WAVES = UINT32_MAX / 64 - 4;
// A wave for each unit of each of them
bool conv_units_fit(const kvb_shape *sh, int64_t tokens) { return tokens <= MOST_WAVES / (conv_groups((int)conv_channels(sh)) + 1); }

// The inputs of a convolution's tokens, and whether there are gates
int check_conv_inputs(const kvb_shape *sh, const kvb_taps *ta, bool tokens, const void *x, const void *a, const void *b, const void *state0)
{
    const size_t size = sh->in_dtype == KVB_F32 ? 4 : 2;
    if (!aligned(x, 16) || !aligned(a, size) || !aligned(b, size) || !aligned(state0, 16) || (tokens && !x) || !a != !b)
        return KVB_EINVAL;
    return a && (!ta->A_log || !ta->dt_bias) ? KVB_EINVAL : KVB_OK;
}
int check_conv_outputs(bool tokens, bool gates, const void *q, const void *k, const void *v, const float *g, const float *beta)
{
    if (!aligned(q, 16) || !aligned(k, 16) || !aligned(v, 16) || !aligned(g, 4) || !aligned(beta, 4) || (tokens && (!q || !k || !v)))
        return KVB_EINVAL;
    return tokens && (gates != (g != nullptr) || gates != (beta != nullptr)) ? KVB_EINVAL : KVB_OK;
}

ConvArgs conv_args(const kvb_shape *sh, const kvb_taps *ta, const void *x, const void *a, const void *b, const void *state0)
{
    ConvArgs r{};
    const int64_t C = conv_channels(sh);
    r.x = x, r.a = a, r.b = b, r.weight = ta->weight, r.bias = ta->bias, r.A_log = ta->A_log, r.dt_bias = ta->dt_bias, r.state0 = state0;
    r.x_stride = ta->x_stride ? ta->x_stride : C, r.a_stride = ta->a_stride ? ta->a_stride : sh->Hv, r.b_stride = ta->b_stride ? ta->b_stride : sh->Hv;
    r.q_stride = r.k_stride = sh->Hk * sh->dk, r.v_stride = sh->Hv * sh->dv;
    r.B = sh->B, r.Hk = sh->Hk, r.Hv = sh->Hv, r.d = sh->dk, r.C = (int)C, r.gates = a != nullptr, r.unit = ta->flags & KVB_CONV_UNIT, r.eps = ta->eps;
    return r;
}
void conv_seqs(ConvArgs &r, const kvb_seqs *sq)
{
    r.start = sq->start, r.slot = sq->slot, r.n_slots = sq->n_slots, r.n_tokens = sq->n_tokens;
    r.q_stride = sq->q_stride ? sq->q_stride : r.q_stride, r.k_stride = sq->k_stride ? sq->k_stride : r.k_stride, r.v_stride = sq->v_stride ? sq->v_stride : r.v_stride;
}
int check_conv_seqs(const kvb_shape *sh, const kvb_taps *ta, const kvb_seqs *sq)
{
    int rc = check_taps(sh, ta);
    if (rc != KVB_OK)
        return rc;
    kvb_shape own = *sh;   // (types of outputs mean nothing here)
    own.out_dtype = KVB_F32;
    rc = check_seqs(&own, sq);
    if (rc != KVB_OK)
        return rc;
    return conv_units_fit(sh, conv_deal(sq->n_tokens, sh->B, conv_groups((int)conv_channels(sh)) + 1, sh->in_dtype == KVB_F32, false).stretches) ? KVB_OK : KVB_EINVAL;
}
// T tokens of each of B requests
int conv_tokens_common(const kvb_shape *sh, const kvb_taps *ta, const int32_t *slot, int32_t n_slots, int32_t T, const int32_t *parent, const void *x,
                       const void *a, const void *b, const void *state0, void *state1, void *q, void *k, void *v, float *g, float *beta, void *stream)
{
    int rc = check_taps(sh, ta);
    if (rc == KVB_OK)
        rc = check_conv_inputs(sh, ta, sh->B > 0, x, a, b, state0);
    if (rc == KVB_OK)
        rc = check_conv_outputs(sh->B > 0, a != nullptr, q, k, v, g, beta);
    if (rc != KVB_OK)
        return rc;
    if ((sh->B > 0 && !slot) || !aligned(slot, 4) || !aligned(parent, 4) || !aligned(state1, 16) || n_slots < 0 || T < 1 || T > KVB_MAX_DRAFTS)
        return KVB_EINVAL;
    if (!conv_units_fit(sh, (int64_t)sh->B * T))
        return KVB_EINVAL;
    if (sh->B == 0)
        return KVB_OK;
    ConvArgs r = conv_args(sh, ta, x, a, b, state0);
    r.slot = slot, r.n_slots = n_slots, r.state1 = state1;
    r.q = q, r.k = k, r.v = v, r.g = g, r.beta = beta;
    g_launch_status = hipSuccess;
    if (T > 1)
        launch_conv_drafts(sh->in_dtype, ta->width, ConvDraftArgs{r, parent, T}, static_cast<hipStream_t>(stream));
    else
        launch_conv_token(sh->in_dtype, ta->width, r, static_cast<hipStream_t>(stream));
    return finish_launch();
}

int64_t conv_columns(const ConvArgs &r, int width) { return (int64_t)(width + (r.bias != nullptr)) * r.C + (r.gates ? 2 * r.Hv : 0); }

// Workspace for the gates' columns too: what there is of them is not known here
int64_t conv_grad_work_bytes(const kvb_shape *sh, const kvb_taps *ta, const kvb_seqs *sq)
{
    const int64_t C = conv_channels(sh), columns = (ta->width + 1) * C + 2 * sh->Hv;
    const bool wide = sh->in_dtype == KVB_F32;
    return 4 * columns * conv_most_parts(sq->n_tokens, sh->B, grad_groups((int)C, wide ? GRAD_CHANNELS<float> : GRAD_CHANNELS<bf16_t>), wide);
}

int check_rows(const kvb_rows *ro)
{
    if (!ro || ro->n_tokens < 0 || ro->heads < 1 || ro->width < 8 || ro->width > KVB_MAX_WIDTH || ro->width % 8 != 0)
        return KVB_EINVAL;
    for (const int t : {ro->dtype, ro->x_dtype})
        if (t != KVB_F32 && t != KVB_BF16 && t != KVB_F16)
            return KVB_EUNSUPPORTED;
    if (ro->x_dtype != KVB_F32 && ro->x_dtype != ro->dtype)
        return KVB_EUNSUPPORTED;
    if (!(ro->eps >= KVB_MIN_EPS) || !std::isfinite(ro->eps) || !std::isfinite(ro->scale))
        return KVB_EINVAL;
    const int64_t w = (int64_t)ro->heads * ro->width, size[2] = {ro->x_dtype == KVB_F32 ? 4 : 2, ro->dtype == KVB_F32 ? 4 : 2}, stride[2] = {ro->x_stride, ro->gate_stride};
    for (int i = 0; i < 2; ++i)
        if (w * 4 > 1 << 26 || (stride[i] != 0 && (stride[i] < w || stride[i] > 1 << 26 || stride[i] * size[i] > 1 << 26 || stride[i] * size[i] % 16 != 0)))
            return KVB_EINVAL;
    return (int64_t)ro->n_tokens * ro->heads > INT32_MAX ? KVB_EINVAL : KVB_OK;
}
NormArgs norm_args(const kvb_rows *ro, const void *x, const void *res, const void *gate, const void *weight, void *sum, void *out)
{
    const int64_t w = (int64_t)ro->heads * ro->width;
    return NormArgs{x, res, gate, weight, sum, out, ro->x_stride ? ro->x_stride : w, ro->gate_stride ? ro->gate_stride : w, (int64_t)ro->n_tokens * ro->heads,
                    ro->heads, ro->width, ro->eps, ro->scale};
}
// (dispatch_types has the pairs the other way round: the narrower type first)
template <typename F>
int norm_types(const kvb_rows *ro, F &&f)
{
    return dispatch_types(ro->dtype, ro->x_dtype, [&]<typename T, typename TX>() { f.template operator()<TX, T>(); });
}

int check_list(const kvb_list *li)
{
    if (!li || li->n < 0 || li->blocks < 0 || li->blocks > MOST_WAVES / 4 || (li->n == 0 && li->blocks > 0))
        return KVB_EINVAL;
    if (li->n > 0 && (!li->data || !li->size || !li->type || !li->first))
        return KVB_EINVAL;
    return aligned(li->data, 8) && aligned(li->size, 8) && aligned(li->type, 4) && aligned(li->first, 4) ? KVB_OK : KVB_EINVAL;
}

}  // namespace

extern "C" {

int kvb_conv(const kvb_shape *shape, const kvb_taps *taps, const kvb_seqs *seqs, const void *x, const void *a, const void *b, const void *state0,
             void *state1, void *q, void *k, void *v, float *g, float *beta, void *stream)
{
    DisarmOnExit disarm;
    int rc = check_conv_seqs(shape, taps, seqs);
    if (rc == KVB_OK)
        rc = check_conv_inputs(shape, taps, seqs->n_tokens > 0, x, a, b, state0);
    if (rc == KVB_OK)
        rc = check_conv_outputs(seqs->n_tokens > 0, a != nullptr, q, k, v, g, beta);
    if (rc != KVB_OK)
        return rc;
    if (!seqs->start || !aligned(seqs->start, 4) || !aligned(seqs->slot, 4) || !aligned(state1, 16))
        return KVB_EINVAL;
    if (shape->B == 0)
        return KVB_OK;
    ConvArgs r = conv_args(shape, taps, x, a, b, state0);
    conv_seqs(r, seqs);
    r.state1 = state1, r.q = q, r.k = k, r.v = v, r.g = g, r.beta = beta;
    g_launch_status = hipSuccess;
    launch_conv(shape->in_dtype, taps->width, r, static_cast<hipStream_t>(stream));
    return finish_launch();
}

int kvb_conv_decode(const kvb_shape *shape, const kvb_taps *taps, const int32_t *slot, int32_t n_slots, const void *x, const void *a, const void *b,
                    const void *state0, void *state1, void *q, void *k, void *v, float *g, float *beta, void *stream)
{
    DisarmOnExit disarm;
    return conv_tokens_common(shape, taps, slot, n_slots, 1, nullptr, x, a, b, state0, state1, q, k, v, g, beta, stream);
}

int kvb_conv_verify(const kvb_shape *shape, const kvb_taps *taps, const int32_t *slot, int32_t n_slots, int32_t T, const int32_t *parent, const void *x,
                    const void *a, const void *b, const void *state, void *q, void *k, void *v, float *g, float *beta, void *stream)
{
    DisarmOnExit disarm;
    return conv_tokens_common(shape, taps, slot, n_slots, T, parent, x, a, b, state, nullptr, q, k, v, g, beta, stream);
}

int kvb_conv_commit(const kvb_shape *shape, const kvb_taps *taps, const int32_t *slot, int32_t n_slots, int32_t T, const int32_t *path,
                    const int32_t *accepted, const void *x, const void *state0, void *state1, void *stream)
{
    DisarmOnExit disarm;
    int rc = check_taps(shape, taps);
    if (rc == KVB_OK)
        rc = check_conv_inputs(shape, taps, shape->B > 0, x, nullptr, nullptr, state0);
    if (rc != KVB_OK)
        return rc;
    if ((shape->B > 0 && (!slot || !accepted || !state1)) || !aligned(slot, 4) || !aligned(path, 4) || !aligned(accepted, 4) || !aligned(state1, 16) || n_slots < 0 || T < 1 ||
        T > KVB_MAX_DRAFTS || !conv_units_fit(shape, shape->B))
        return KVB_EINVAL;
    if (shape->B == 0)
        return KVB_OK;
    const ConvArgs r = conv_args(shape, taps, x, nullptr, nullptr, state0);
    g_launch_status = hipSuccess;
    launch_conv_commit(shape->in_dtype, taps->width, ConvCommitArgs{x, state0, state1, slot, path, accepted, r.x_stride, shape->B, T, n_slots, r.C},
                       static_cast<hipStream_t>(stream));
    return finish_launch();
}

int64_t kvb_conv_backward_work(const kvb_shape *shape, const kvb_taps *taps, const kvb_seqs *seqs)
{
    const int rc = check_conv_seqs(shape, taps, seqs);
    return rc != KVB_OK ? rc : conv_grad_work_bytes(shape, taps, seqs);
}

int kvb_conv_backward(const kvb_shape *shape, const kvb_taps *taps, const kvb_seqs *seqs, const void *x, const void *a, const void *b,
                      const void *state0, const void *dq, const void *dk, const void *dv, const float *dg, const float *dbeta, const void *dstate1,
                      void *dx, void *da, void *db, float *dweight, float *dbias, float *dA_log, float *ddt_bias, void *dstate0, void *work, void *stream)
{
    DisarmOnExit disarm;
    int rc = check_conv_seqs(shape, taps, seqs);
    const bool tokens = rc == KVB_OK && seqs->n_tokens > 0, gates = tokens ? a != nullptr : dA_log != nullptr;
    if (rc == KVB_OK)
        rc = check_conv_inputs(shape, taps, tokens, x, a, b, state0);
    if (rc == KVB_OK)
        rc = check_conv_outputs(tokens, gates, dq, dk, dv, dg, dbeta);
    if (rc != KVB_OK)
        return rc;
    const size_t size = shape->in_dtype == KVB_F32 ? 4 : 2;
    if (!seqs->start || !aligned(seqs->start, 4) || !aligned(seqs->slot, 4) || !aligned(dstate1, 16) || !aligned(dx, 16) || !aligned(da, size) || !aligned(db, size) ||
        !aligned(dweight, 4) || !aligned(dbias, 4) || !aligned(dA_log, 4) || !aligned(ddt_bias, 4) || !aligned(dstate0, 16) || !aligned(work, 16))
        return KVB_EINVAL;
    if ((tokens && (!dx || gates != (da != nullptr) || gates != (db != nullptr))) || !dweight || !work || (dbias != nullptr) != (taps->bias != nullptr) ||
        gates != (dA_log != nullptr) || gates != (ddt_bias != nullptr) || (dstate0 && dstate0 == dstate1))
        return KVB_EINVAL;
    ConvGradArgs r{};
    r.f = conv_args(shape, taps, x, a, b, state0);
    conv_seqs(r.f, seqs);
    r.f.gates = gates;
    r.dq = dq, r.dk = dk, r.dv = dv, r.dg = dg, r.dbeta = dbeta, r.dstate1 = dstate1, r.dx = dx, r.da = da, r.db = db, r.dstate0 = dstate0;
    const bool wide = shape->in_dtype == KVB_F32;
    const ConvParts parts = conv_parts(seqs->n_tokens, shape->B, grad_groups(r.f.C, wide ? GRAD_CHANNELS<float> : GRAD_CHANNELS<bf16_t>) + gates, wide);
    r.part = static_cast<float *>(work), r.parts = parts.parts, r.columns = (int)conv_columns(r.f, taps->width);
    g_launch_status = hipSuccess;
    hipStream_t hs = static_cast<hipStream_t>(stream);
    if (shape->in_dtype == KVB_F32)
        launch_conv_grad_typed<float>(taps->width, r, parts.length, dweight, dbias, dA_log, ddt_bias, hs);
    else if (shape->in_dtype == KVB_BF16)
        launch_conv_grad_typed<bf16_t>(taps->width, r, parts.length, dweight, dbias, dA_log, ddt_bias, hs);
    else
        launch_conv_grad_typed<f16_t>(taps->width, r, parts.length, dweight, dbias, dA_log, ddt_bias, hs);
    return finish_launch();
}

int kvb_norm(const kvb_rows *rows, const void *x, const void *res, const void *gate, const void *weight, void *sum, void *out, void *stream)
{
    DisarmOnExit disarm;
    int rc = check_rows(rows);
    if (rc != KVB_OK)
        return rc;
    if (!aligned(x, 16) || !aligned(res, 16) || !aligned(gate, 16) || !aligned(weight, 16) || !aligned(sum, 16) || !aligned(out, 16))
        return KVB_EINVAL;
    if (rows->n_tokens == 0)   // (arrays of no elements may be NULL)
        return KVB_OK;
    if (!x || !weight || !out || (!res && (sum || rows->scale != 1.0f)))
        return KVB_EINVAL;
    const NormArgs a = norm_args(rows, x, res, gate, weight, sum, out);
    if (rows->width > 2048 && a.rows > MOST_WAVES / (rows->width > 8192 ? 8 : 4))   // a workgroup a row
        return KVB_EINVAL;
    g_launch_status = hipSuccess;
    rc = norm_types(rows, [&]<typename TX, typename T>() { launch_norm_typed<TX, T>(a, static_cast<hipStream_t>(stream)); });
    if (rc != KVB_OK)
        return rc;
    return finish_launch();
}

int64_t kvb_norm_backward_work(const kvb_rows *rows)
{
    const int rc = check_rows(rows);
    return rc != KVB_OK ? rc : 4 * (int64_t)rows->width * norm_most_parts((int64_t)rows->n_tokens * rows->heads, rows->width);
}

int kvb_norm_backward(const kvb_rows *rows, const void *x, const void *gate, const void *weight, const void *dout, const void *dsum, void *dx, void *dres,
                      void *dgate, float *dweight, void *work, void *stream)
{
    DisarmOnExit disarm;
    int rc = check_rows(rows);
    if (rc != KVB_OK)
        return rc;
    if (!aligned(x, 16) || !aligned(gate, 16) || !aligned(weight, 16) || !aligned(dout, 16) || !aligned(dsum, 16) || !aligned(dx, 16) || !aligned(dres, 16) ||
        !aligned(dgate, 16) || !aligned(dweight, 4) || !aligned(work, 16))
        return KVB_EINVAL;
    if (!dweight || (rows->n_tokens > 0 && !weight) || (gate != nullptr) != (dgate != nullptr) || (rows->n_tokens > 0 && (!x || !dout || !dx || !work)))
        return KVB_EINVAL;
    NormGradArgs a{norm_args(rows, x, nullptr, gate, weight, nullptr, nullptr), dout, dsum, dx, dres, dgate, static_cast<float *>(work), 0, rows->scale};
    a.parts = norm_parts(a.f.rows, a.f.width);
    g_launch_status = hipSuccess;
    rc = norm_types(rows, [&]<typename TX, typename T>() { launch_norm_grad_typed<TX, T>(a, dweight, static_cast<hipStream_t>(stream)); });
    if (rc != KVB_OK)
        return rc;
    return finish_launch();
}

int64_t kvb_grad_norm_work(const kvb_list *list)
{
    const int rc = check_list(list);
    return rc != KVB_OK ? rc : 8 * list_most_sums(list->blocks);
}

int kvb_grad_norm(const kvb_list *list, float *norm, void *work, void *stream)
{
    DisarmOnExit disarm;
    const int rc = check_list(list);
    if (rc != KVB_OK)
        return rc;
    if (!norm || !aligned(norm, 4) || !aligned(work, 8) || (list->blocks > 0 && !work))
        return KVB_EINVAL;
    g_launch_status = hipSuccess;
    launch_grad_norm(ListArgs{list->data, nullptr, list->size, list->type, list->first, list->n, list->blocks}, norm, static_cast<double *>(work),
                     static_cast<hipStream_t>(stream));
    return finish_launch();
}

int kvb_clip(const kvb_list *list, const kvb_list *to, const float *norm, float largest, void *stream)
{
    DisarmOnExit disarm;
    int rc = check_list(list);
    if (rc == KVB_OK && to)
        rc = check_list(to);
    if (rc != KVB_OK)
        return rc;
    if (!norm || !aligned(norm, 4) || !(largest >= 0.0f) || (to && (to->n != list->n || to->blocks != list->blocks)))
        return KVB_EINVAL;
    if (list->blocks == 0)
        return KVB_OK;
    g_launch_status = hipSuccess;
    launch_clip(ListArgs{list->data, to ? to->data : list->data, list->size, list->type, list->first, list->n, list->blocks}, norm, largest,
                static_cast<hipStream_t>(stream));
    return finish_launch();
}

int64_t kvb_accept_work(const kvb_vocab *vocab)
{
    const int rc = check_vocab(vocab);
    return rc != KVB_OK ? rc : accept_work_bytes(vocab->B, vocab->V);
}

int kvb_accept(const kvb_vocab *vocab, const int32_t *n_drafts, const int32_t *parent, const int32_t *tokens, const void *target,
               const void *draft, const float *u, const float *s, int32_t *path, int32_t *accepted, int32_t *token, void *work, void *stream)
{
    DisarmOnExit disarm;
    const int rc = check_vocab(vocab);
    if (rc != KVB_OK)
        return rc;
    if (vocab->B == 0)
        return KVB_OK;
    const size_t size = vocab->dtype == KVB_F32 ? 4 : 2;
    if (!tokens || !target || !u || !s || !path || !accepted || !token || !work)
        return KVB_EINVAL;
    if (!aligned(n_drafts, 4) || !aligned(parent, 4) || !aligned(tokens, 4) || !aligned(target, size) || !aligned(draft, size) ||
        !aligned(u, 4) || !aligned(s, 4) || !aligned(path, 4) || !aligned(accepted, 4) || !aligned(token, 4) || !aligned(work, 8))
        return KVB_EINVAL;
    const int segments = accept_segments(vocab->B, vocab->V);
    const AcceptArgs a{n_drafts, parent, tokens, target, draft, u, s, path, accepted, token, static_cast<double *>(work), reinterpret_cast<AcceptWalk *>(static_cast<double *>(work) + (int64_t)vocab->B * segments),
                       vocab->stride ? vocab->stride : vocab->V, vocab->B, vocab->T, vocab->V, segments, accept_segment(vocab->V, segments)};
    g_launch_status = hipSuccess;
    launch_accept(vocab->dtype, a, static_cast<hipStream_t>(stream));
    return finish_launch();
}

int64_t kvb_scan_work(const kvb_shape *shape, const kvb_seqs *seqs)
{
    const int rc = check_seqs(shape, seqs);
    return rc != KVB_OK ? rc : scan_work_bytes(shape, seqs);
}

int kvb_scan(const kvb_shape *shape, const kvb_seqs *seqs, const void *q, const void *k, const void *v, const float *g, const float *beta,
             const float *state0, float *state1, void *out, void *work, void *stream)
{
    DisarmOnExit disarm;
    int rc = check_seqs(shape, seqs);
    if (rc == KVB_OK)
        rc = check_seq_pointers(shape, seqs, q, k, v, g, beta, state0, work);
    if (rc != KVB_OK)
        return rc;
    if (!aligned(state1, 16) || !aligned(out, 16) || (seqs->n_tokens > 0 && !out))
        return KVB_EINVAL;
    if (shape->B == 0)
        return KVB_OK;
    const ScanArgs a = scan_args(shape, seqs, q, k, v, g, beta, state0, state1, out, static_cast<float *>(work), nullptr, nullptr);
    hipStream_t hs = static_cast<hipStream_t>(stream);
    g_launch_status = hipSuccess;
    rc = dispatch_types(shape->in_dtype, shape->out_dtype, [&]<typename TIn, typename TOut>() { launch_scan_typed<TIn, TOut>(shape->dk, a, hs); });
    if (rc != KVB_OK)
        return rc;
    return finish_launch();
}

int64_t kvb_scan_backward_work(const kvb_shape *shape, const kvb_seqs *seqs)
{
    const int rc = check_seqs(shape, seqs);
    return rc != KVB_OK ? rc : grad_work_bytes(shape, seqs);
}

int kvb_scan_backward(const kvb_shape *shape, const kvb_seqs *seqs, const void *q, const void *k, const void *v, const float *g,
                      const float *beta, const float *state0, const void *dout, const float *dstate1, void *dq, void *dk, void *dv,
                      float *dg, float *dbeta, float *dstate0, void *work, void *stream)
{
    DisarmOnExit disarm;
    int rc = check_seqs(shape, seqs);
    if (rc == KVB_OK)
        rc = check_seq_pointers(shape, seqs, q, k, v, g, beta, state0, work);
    if (rc != KVB_OK)
        return rc;
    if (!aligned(dout, 16) || !aligned(dstate1, 16) || !aligned(dq, 16) || !aligned(dk, 16) || !aligned(dv, 16) || !aligned(dg, 4) ||
        !aligned(dbeta, 4) || !aligned(dstate0, 16))
        return KVB_EINVAL;
    if (seqs->n_tokens > 0 && (!dout || !dq || !dk || !dv || !dg || !dbeta))
        return KVB_EINVAL;
    if (shape->B == 0)
        return KVB_OK;
    const int64_t chunks = scan_chunks(seqs->n_tokens, shape->B) * shape->Hv, d = shape->dk;
    float *prep = static_cast<float *>(work);   // (every part a multiple of 16 bytes)
    float *s0 = prep + chunks * GRAD_PREP, *ds = s0 + chunks * d * d, *z = ds + chunks * d * d, *dd = z + chunks * SC * d, *part = dd + chunks * SC * d;
    const GradArgs a{scan_args(shape, seqs, q, k, v, g, beta, state0, nullptr, nullptr, prep, s0, z), dout, dstate1, dq, dk, dv, dg, dbeta, dstate0, ds, dd, part};
    hipStream_t hs = static_cast<hipStream_t>(stream);
    g_launch_status = hipSuccess;
    rc = dispatch_types(shape->in_dtype, shape->out_dtype, [&]<typename TIn, typename TOut>() { launch_scan_grad_typed<TIn, TOut>(shape->dk, a, hs); });
    if (rc != KVB_OK)
        return rc;
    return finish_launch();
}

int kvb_decode(const kvb_shape *shape, const kvb_store *store, const int32_t *slot, const void *q, const void *k,
               const void *v, const float *g, const float *beta, void *out, void *stream)
{
    DisarmOnExit disarm;
    return step_common(shape, store, slot, 1, q, k, v, g, beta, out, stream, 1);
}

int kvb_decode_flush(const kvb_shape *shape, const kvb_store *store, const int32_t *slot, const void *q,
                     const void *k, const void *v, const float *g, const float *beta, void *out,
                     int32_t threshold, void *stream)
{
    DisarmOnExit disarm;
    if (!shape || !store)
        return KVB_EINVAL;
    if (!store->state || threshold < 1 || threshold > shape->cap)
        return KVB_EINVAL;
    return step_common(shape, store, slot, 1, q, k, v, g, beta, out, stream, 1, threshold);
}

int kvb_verify(const kvb_shape *shape, const kvb_store *store, const int32_t *slot, int32_t T, const void *q,
               const void *k, const void *v, const float *g, const float *beta, void *out, void *stream)
{
    DisarmOnExit disarm;
    return step_common(shape, store, slot, T, q, k, v, g, beta, out, stream, 0);
}

int kvb_verify_tree(const kvb_shape *shape, const kvb_store *store, const int32_t *slot, int32_t T,
                    const int32_t *parent, const void *q, const void *k, const void *v, const float *g,
                    const float *beta, void *out, void *stream)
{
    DisarmOnExit disarm;
    if (!parent || !aligned(parent, 4))
        return KVB_EINVAL;
    return step_common(shape, store, slot, T, q, k, v, g, beta, out, stream, 0, 0, parent);
}

int kvb_compact(const kvb_shape *shape, const kvb_store *store, const int32_t *slot, int32_t T,
                const int32_t *path, const int32_t *path_len, void *stream)
{
    DisarmOnExit disarm;
    int rc = check_common(shape, store, slot);
    if (rc != KVB_OK)
        return rc;
    if (!path || !path_len || !aligned(path, 4) || !aligned(path_len, 4))
        return KVB_EINVAL;
    if (T < 1 || T > KVB_MAX_DRAFTS || T > shape->cap)
        return KVB_EINVAL;
    if (shape->B == 0)
        return KVB_OK;
    CompactArgs a{dev_store(store), slot, path, path_len, shape->Hk, shape->Hv, shape->Hv / shape->Hk, shape->cap, T};
    const int blocks = shape->B * shape->Hv;
    hipStream_t hs = static_cast<hipStream_t>(stream);
    g_launch_status = hipSuccess;
    rc = launch_compact(shape->dk, shape->in_dtype, shape->rec_dtype, a, blocks, hs);
    if (rc != KVB_OK)
        return rc;
    return finish_launch();
}

int kvb_flush(const kvb_shape *shape, const kvb_store *store, const int32_t *slot, const int32_t *accepted,
              int32_t threshold, void *stream)
{
    DisarmOnExit disarm;
    int rc = check_common(shape, store, slot);
    if (rc != KVB_OK)
        return rc;
    if (!aligned(accepted, 4))
        return KVB_EINVAL;
    if (!store->state && !accepted)   // nothing to fold into and nothing to commit
        return KVB_EINVAL;
    if (threshold < 1 || threshold > shape->cap)
        return KVB_EINVAL;
    if (shape->B == 0)
        return KVB_OK;
    if (shape->Hv > MAX_FILL_WG)
        return KVB_EINVAL;
    FlushArgs a{dev_store(store), slot, accepted, shape->Hk, shape->Hv, shape->Hv / shape->Hk, shape->cap, threshold,
                store->state && stream_state(shape, store, 192.0) ? 1 : 0};
    const int blocks = shape->B * shape->Hv;
    hipStream_t hs = static_cast<hipStream_t>(stream);
    g_launch_status = hipSuccess;
    rc = launch_flush(shape->dk, shape->in_dtype, shape->rec_dtype, a, blocks, hs);
    if (rc != KVB_OK)
        return rc;
    return finish_launch();
}

int kvb_direct(const kvb_shape *shape, const kvb_store *store, const int32_t *slot, const int32_t *len,
               int32_t Lmax, const void *q, const void *k, const void *v, const float *g, const float *beta,
               void *out, void *stream)
{
    DisarmOnExit disarm;
    int rc = check_common(shape, store, slot);
    if (rc != KVB_OK)
        return rc;
    rc = check_tokens(q, k, v, g, beta, out);
    if (rc != KVB_OK)
        return rc;
    if (!len || !aligned(len, 4))
        return KVB_EINVAL;
    if (Lmax < 1 || Lmax > shape->cap || Lmax > KVB_MAX_DIRECT_LEN)
        return KVB_EINVAL;
    if (shape->B == 0)
        return KVB_OK;
    // offsets in 32 bits: of the elements of a context, and of the bytes of 16 rows in fp32
    if ((long long)shape->Hv * shape->dv * (Lmax > 64 ? Lmax : 64) > 1LL << 32)
        return KVB_EINVAL;
    DirectArgs a{dev_store(store), slot, len, q, k, v, g, beta, out, shape->out_dtype == KVB_F32, shape->Hk,
                 shape->Hv, shape->Hv / shape->Hk, shape->cap, Lmax, shape->scale};
    const int blocks = shape->B * shape->Hv;
    hipStream_t hs = static_cast<hipStream_t>(stream);
    g_launch_status = hipSuccess;
    rc = launch_direct(shape->dk, shape->in_dtype, shape->rec_dtype, a, blocks, hs);
    if (rc != KVB_OK)
        return rc;
    return finish_launch();
}

int kvb_timer_create(kvb_timer **timer)
{
    if (!timer)
        return KVB_EINVAL;
    kvb_timer *t = new kvb_timer{nullptr, nullptr};
    hipError_t e = hipEventCreate(&t->start);
    if (e == hipSuccess)
        e = hipEventCreate(&t->stop);
    if (e != hipSuccess) {
        g_last_hip_error = e;
        (void)hipGetLastError();   // (as in kvb_timer_read)
        if (t->start)
            (void)hipEventDestroy(t->start);
        delete t;
        return KVB_EHIP;
    }
    *timer = t;
    return KVB_OK;
}

int kvb_timer_arm(kvb_timer *timer)
{
    g_armed = timer;
    return KVB_OK;
}

int kvb_timer_read(kvb_timer *timer, float *microseconds)
{
    if (!timer || !microseconds)
        return KVB_EINVAL;
    hipError_t e = hipEventSynchronize(timer->stop);
    float ms = 0.0f;
    if (e == hipSuccess)
        e = hipEventElapsedTime(&ms, timer->start, timer->stop);
    if (e != hipSuccess) {
        g_last_hip_error = e;
        (void)hipGetLastError();   // this call's own error: not left behind for the caller's next HIP call
        return KVB_EHIP;
    }
    *microseconds = ms * 1000.0f;
    return KVB_OK;
}

void kvb_timer_destroy(kvb_timer *timer)
{
    if (!timer)
        return;
    if (g_armed == timer)
        g_armed = nullptr;
    (void)hipEventDestroy(timer->start);
    (void)hipEventDestroy(timer->stop);
    delete timer;
}

const char *kvb_strerror(int code)
{
    switch (code) {
    case KVB_OK:
        return "ok";
    case KVB_EINVAL:
        return "invalid argument (null or misaligned pointer, or a size out of range)";
    case KVB_EUNSUPPORTED:
        return "unsupported head size or dtype";
    case KVB_EHIP:
        return hipGetErrorString(g_last_hip_error);
    }
    return "unknown kvb error code";
}

int kvb_version(void) { return KVB_VERSION; }

}  // extern "C"
