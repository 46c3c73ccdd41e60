/*
 * kvb -- KVBuffer-style Gated DeltaNet decoding for AMD MI355X (gfx950).
 *
 * C ABI of the library.  Every pointer marked "device" is device memory owned
 * by the caller; the compute calls never allocate, free or synchronise, and
 * enqueue all work on the caller's HIP stream (`stream` is a hipStream_t passed
 * as void*; NULL = the default stream).  The structs are host memory and are
 * read only during the call.  The only state the library keeps is two
 * thread-local words on the host: the timer armed for the calling thread's next
 * launch (kvb_timer_arm) and the HIP error code behind the last KVB_EHIP.
 *
 * Notation (paper Sec. 2.1, Sec. 3, App. A.1).  For one request and one v-head:
 *   S0    the committed state, dk x dv, fp32                (the "state slot", Sec. 2.2)
 *   f     number of records in the request's buffer         ("fill")
 *   record l (0 <= l < f) = ( k_l, u_l, G_l ):
 *         k_l  key of the l-th token since the last flush
 *         u_l  its delta value (the quantity the paper buffers instead of v)
 *         G_l  sum of the log decays g of tokens 0..l of the chunk, so that
 *              gamma_l = exp(G_l) and Gamma_{il} = exp(G_i - G_l) <= 1 for i >= l
 *   For a new token at chunk position i (App. A.1, Eq. 16):
 *         u_i = beta_i ( v_i - gamma_i k_i S0 - sum_{l<i}  Gamma_{il} (k_i.k_l) u_l )
 *         o_i = scale  ( gamma_i q_i S0       + sum_{l<=i} Gamma_{il} (q_i.k_l) u_l )
 *         S   = gamma_m-1 S0 + sum_{l<m} Gamma_{m-1,l} k_l^T u_l          (flush of m records)
 *   which is exactly the token-by-token recurrence of Eq. 11-12 regrouped.
 *
 * Grouped heads: v-head h uses the q and k of qk-head h / (Hv / Hk).
 * The gate is passed as a log decay g <= 0 (alpha = exp(g)); gamma ratios are
 * never formed, only exp of differences.
 */
#ifndef KVB_H
#define KVB_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define KVB_VERSION 120 /* 120: fp16 inputs, 16-bit delta-value records and outputs (kvb_shape.rec_dtype) */

/* return codes */
#define KVB_OK            0
#define KVB_EINVAL       (-1) /* null / misaligned pointer, size out of range          */
#define KVB_EUNSUPPORTED (-2) /* head size or dtype combination that is not compiled    */
#define KVB_EHIP         (-3) /* the HIP runtime refused the launch                     */

/* element types: of q, k, v and the buffered keys (in_dtype), of the buffered delta values
 * (rec_dtype) and of the outputs (out_dtype).  The paper's implementation keeps a fp32 state
 * and fp16 vectors and records (Sec. 4.1; caption of the GDN memory-profile table, App. A.2):
 * that is in = rec = out = KVB_F16.  A 16-bit rec_dtype or out_dtype must equal in_dtype;
 * KVB_F32 is always allowed for both.  The state is fp32 throughout. */
#define KVB_F32  0
#define KVB_BF16 1
#define KVB_F16  2
/* Which (in_dtype, head size) pairs are tuned.  d = 128 with KVB_BF16 or KVB_F16 inputs (any
 * allowed rec_dtype / out_dtype) is the pair the kernels are built and measured for: matrix-
 * instruction kernels for kvb_verify, kvb_verify_tree, kvb_flush and kvb_direct, the streaming
 * decode kernel for kvb_decode / kvb_decode_flush.  KVB_F32 inputs at any head size, and
 * d = 32 or 64 with any input type, run on the fp32 matrix instruction (single-token decoding:
 * the vector ALU): same results, and kvb_direct is limited to 64 tokens there. */

#define KVB_MAX_CAP        128 /* largest `cap` (the paper buffers at most d records, Sec. 3.4) */
#define KVB_MAX_DRAFTS       8 /* largest T of kvb_verify (Sec. 4.2 sweeps up to 8)             */
#define KVB_MAX_DIRECT_LEN 128 /* largest Lmax of kvb_direct (Sec. 3.4: contexts up to d tokens);
                                  16-bit inputs with d = 128; the other compiled pairs take 64   */
#define KVB_MAX_BLOCKS      16 /* longest block-table row (KVB_MAX_CAP / smallest block)        */

/* kvb_store.flags: how the state should travel through the caches.  With neither bit the
 * library streams (non-temporal loads, and non-temporal stores when the state is written
 * back) when the states one call touches, 4 * B * Hv * dk * dv bytes, exceed 288 MiB: a little
 * more than the 256 MB last-level cache, because a state of 256 MiB that is re-read every
 * step still finds most of itself there; kvb_flush, which passes the state through the cache
 * in both directions, switches at 192 MiB.  A model with many GDN layers should set
 * KVB_STORE_STREAM: each layer's state is next read one token later, after every other
 * layer's has passed through. */
#define KVB_STORE_STREAM   1
#define KVB_STORE_RESIDENT 2
/* kvb_store.flags, where the fills lie: without this bit `fill` is [n_slots], with it
 * [n_slots][KVB_FILL_APART] and the fill of a slot is the first word of its row (the others are
 * neither read nor written).  All workgroups of a request add to its fill in calls that change
 * it, and additions to one 128-byte line pass one at a time: with a line to each slot, calls of
 * a few hundred to a few thousand workgroups are up to 30 % faster.  Use it in new programs. */
#define KVB_STORE_FILL_APART 4
#define KVB_FILL_APART      32

/* bits set in status[slot]: a call would have overrun that request's buffer; a draft tree or
 * an accepted path handed to kvb_verify_tree / kvb_compact was not well formed */
#define KVB_STATUS_OVERFLOW 1
#define KVB_STATUS_BADPATH  2

typedef struct kvb_shape {
    int32_t B;         /* requests in this call (0 = no-op)                                */
    int32_t Hk;        /* q/k heads                                                        */
    int32_t Hv;        /* v heads, Hv % Hk == 0.  At most (KVB_EINVAL beyond): 32768 for   */
                       /* calls that change `fill`, for kvb_decode without a state counted */
                       /* as Hk * ceil(Hv / Hk / 2); less than 4 GiB of v a draft for      */
                       /* several drafts of kvb_verify; Hv * dv * max(Lmax, 64) <= 2^32    */
                       /* for kvb_direct                                                   */
    int32_t dk;        /* key/query head size;   compiled: dk == dv in {32, 64, 128}       */
    int32_t dv;        /* value head size                                                  */
    int32_t cap;       /* records one request's buffer can hold, 1..KVB_MAX_CAP            */
    int32_t in_dtype;  /* KVB_F32, KVB_BF16 or KVB_F16: type of q, k, v and of buf_k       */
    int32_t out_dtype; /* type of `out`: KVB_F32, or in_dtype if that is a 16-bit type     */
    int32_t rec_dtype; /* type of buf_u: KVB_F32, or in_dtype if that is a 16-bit type.    */
                       /* A 16-bit record holds the delta value rounded to nearest even;   */
                       /* every later use (the token's own output included) reads that     */
                       /* rounded value, so a record is all that later calls depend on.    */
    float   scale;     /* multiplies every output (1.0 = the paper's formulas)             */
} kvb_shape;

typedef struct kvb_store {
    float   *state;   /* device [n_slots, Hv, dk, dv] fp32, dv contiguous.  May be NULL for
                         kvb_decode / kvb_verify: KV-only mode, S0 taken as zero (Sec. 3.4). */
    void    *buf_k;   /* device [n_slots, Hk, cap, dk] in_dtype                             */
    void    *buf_u;   /* device [n_slots, Hv, cap, dv] rec_dtype                            */
    float   *buf_G;   /* device [n_slots, Hv, cap]     fp32                                 */
    int32_t *fill;    /* device [n_slots] (KVB_STORE_FILL_APART: [n_slots][KVB_FILL_APART], the
                         first word of a row); 0..cap between calls.  While a call that changes
                         fill runs, the word belongs to its workgroups: bits 16.. count
                         them, it may be negative, and the low half may hold the new count
                         before the records exist.  Neither count can be read from it until
                         the call's kernel has ended, when it is a plain count again.        */
    int32_t *status;  /* device [n_slots] sticky KVB_STATUS_* bits, or NULL                 */
    int32_t  n_slots; /* slots in the arrays above; requests whose slot is outside
                         0..n_slots-1 are skipped                                           */
    int32_t  flags;   /* KVB_STORE_* hints, 0 = let the library decide                      */
    /* Paged record buffers (Sec. 3.1: a request's buffer is made of blocks of 8 or 16 records
     * drawn from a pool shared by all requests).  block_table == NULL (and the three sizes 0):
     * the layout above, one block of cap records per slot.  Otherwise record l of slot s lives
     * in block block_table[s][l / block_size] at position l % block_size, and the record
     * arrays are pools of n_blocks blocks:
     *   buf_k [n_blocks, Hk, block_size, dk]   buf_u [n_blocks, Hv, block_size, dv]
     *   buf_G [n_blocks, Hv, block_size]
     * state, fill and status stay per slot.  Only the entries that cover records 0..cap-1 are
     * read; ids outside 0..n_blocks-1 are clamped into the pool.  Two requests of one call must
     * not share a block.                                                                     */
    const int32_t *block_table; /* device [n_slots, max_blocks] or NULL                       */
    int32_t  block_size;        /* 8, 16, 32, 64 or 128 records                               */
    int32_t  max_blocks;        /* 1..KVB_MAX_BLOCKS, block_size * max_blocks >= cap          */
    int32_t  n_blocks;          /* blocks in the pools                                        */
} kvb_store;

/*
 * All compute calls take `slot`: device int32 [B], the store slot of request b.
 * A slot must not appear twice in one call.  Infinities and NaN reach what the formulas pass
 * them to, with two exceptions for 16-bit inputs at d = 128: kvb_flush makes NaN of the state
 * column of an infinite delta value and of the state row of an infinite key (kvb_decode_flush
 * keeps them infinite), and in kvb_verify / kvb_verify_tree a draft whose key is not finite may
 * make the request's other drafts NaN.  state, buf_k, buf_u, q, k, v and
 * out must be 16-byte aligned; the int32 / float vectors 4-byte aligned.
 */

/*
 * kvb_decode -- chunkwise decoding of ONE new token per request (Sec. 3.2; the
 * single-token chunkwise form, App. A.1 Eq. 16; with store->state == NULL the
 * single-token parallel form, Eq. 14).  Reads S0 and records 0..f-1, writes the
 * output and record f = (k, u, G_f), then fill = f + 1.  Never writes `state`.
 *   q, k  device [B, Hk, dk] in_dtype      v    device [B, Hv, dv] in_dtype
 *   g     device [B, Hv] fp32 log decay    beta device [B, Hv] fp32
 *   out   device [B, Hv, dv] out_dtype
 * A request with f == cap is skipped: its out row and buffer are left as they
 * are and status[slot] gets KVB_STATUS_OVERFLOW.
 */
int kvb_decode(const kvb_shape *shape, const kvb_store *store, const int32_t *slot,
               const void *q, const void *k, const void *v,
               const float *g, const float *beta, void *out, void *stream);

/*
 * kvb_decode_flush -- kvb_decode followed by kvb_flush(accepted = NULL, threshold), in one
 * pass (the paper launches the state update as a second kernel, Sec. 4.2; here a request
 * whose buffer reaches `threshold` records with this token has its state updated from the
 * tile the decode step has already read, which saves re-reading it).  Same arguments,
 * results and error behaviour as the two calls in sequence; state must not be NULL;
 * threshold 1..cap (threshold 1 is the fused recurrent step: every token is folded at once).
 */
int kvb_decode_flush(const kvb_shape *shape, const kvb_store *store, const int32_t *slot,
                     const void *q, const void *k, const void *v,
                     const float *g, const float *beta, void *out,
                     int32_t threshold, void *stream);

/*
 * kvb_flush -- the deferred, batched state update (Sec. 3.2, Eq. 5; for GDN the
 * last line of App. A.1 Eq. 16; with `accepted` the accepted-only update of
 * Sec. 3.3 Eq. 8).  For request b: m = fill + (accepted ? accepted[b] : 0); if
 * m >= threshold and m > 0:  S <- exp(G_{m-1}) S + sum_l exp(G_{m-1} - G_l) k_l^T u_l
 * and fill = 0; otherwise fill = m and the state is untouched.  Besides
 * kvb_decode_flush the only call that writes `state`.
 * On a zeroed state this is the KV-only -> state transition of Sec. 3.4.
 * state == NULL (a KV-only context): nothing is folded, the call only commits the accepted
 * drafts of a preceding kvb_verify (fill = m); `accepted` must then be given.
 *   accepted  device int32 [B] (each 0..T of the preceding kvb_verify) or NULL
 *   threshold 1..cap; 1 flushes every non-empty buffer
 * m > cap sets KVB_STATUS_OVERFLOW and is treated as cap.
 */
int kvb_flush(const kvb_shape *shape, const kvb_store *store, const int32_t *slot,
              const int32_t *accepted, int32_t threshold, void *stream);

/*
 * kvb_verify -- parallel verification of T sequential draft tokens per request
 * (Sec. 3.3, Eq. 7; for GDN the chunkwise matrix form App. A.1 Eq. 15 restricted
 * to rows f..f+T-1).  One pass over S0 serves all T drafts; no temporary state
 * is formed.  Writes T outputs and records f..f+T-1 but leaves `fill` (and
 * `state`) untouched: committing is kvb_flush(accepted, ...).
 *   T     1..KVB_MAX_DRAFTS
 *   q, k  device [B, T, Hk, dk]   v device [B, T, Hv, dv]   g, beta device [B, T, Hv]
 *   out   device [B, T, Hv, dv] out_dtype
 * A request with f + T > cap is skipped with KVB_STATUS_OVERFLOW.
 */
int kvb_verify(const kvb_shape *shape, const kvb_store *store, const int32_t *slot, int32_t T,
               const void *q, const void *k, const void *v,
               const float *g, const float *beta, void *out, void *stream);

/*
 * kvb_verify_tree -- kvb_verify for drafts that form a tree (Sec. 3.3: the mask M and the
 * prefix set Par(t) of App. A.1 admit any draft structure; the figure of Sec. 3.3 accepts
 * drafts 0 and 2 of three).  Draft i continues the committed context and then exactly its
 * ancestors among the T drafts: its decay, its delta value and its output are those of the
 * root path that ends in i.  With parent[b][i] = i - 1 this is kvb_verify.
 *   parent  device int32 [B, T]: parent[b][i] in {-1, 0 .. i-1}; -1 = the draft follows the last
 *           committed token.  Parents precede their children.  An entry outside that range is
 *           taken as -1 and status[slot] gets KVB_STATUS_BADPATH.  T = 1: not read.
 * Everything else as kvb_verify: record f + i holds draft i (its G is cumulative along its own
 * path), fill and state are untouched.  Committing an accepted root path is kvb_compact followed
 * by kvb_flush(accepted = path_len).
 */
int kvb_verify_tree(const kvb_shape *shape, const kvb_store *store, const int32_t *slot, int32_t T,
                    const int32_t *parent, const void *q, const void *k, const void *v,
                    const float *g, const float *beta, void *out, void *stream);

/*
 * kvb_compact -- makes the accepted drafts of a tree a prefix of the T new records (Sec. 3.3,
 * Eq. 8: only accepted tokens reach the state).  For request b the records at f + path[b][j]
 * move to f + j, j = 0 .. path_len[b]-1; the caller then commits them with
 * kvb_flush(accepted = path_len, ...).  Neither fill nor state changes here.
 *   T         the T of the preceding kvb_verify_tree
 *   path      device int32 [B, T]: the accepted root path, oldest draft first, strictly increasing
 *             node indices in 0 .. T-1 (the caller passes a path of the tree; only its order and
 *             range are checked)
 *   path_len  device int32 [B]: 0 .. T accepted drafts
 * A path that is not increasing, a length outside 0..T, or f + T > cap leaves the request's
 * records as they are and sets KVB_STATUS_BADPATH.
 */
int kvb_compact(const kvb_shape *shape, const kvb_store *store, const int32_t *slot, int32_t T,
                const int32_t *path, const int32_t *path_len, void *stream);

/*
 * kvb_direct -- state-free computation of a whole short context from its keys
 * and values (Sec. 3.4; the parallel form App. A.1 Eq. 13).  For request b the
 * first len[b] tokens are processed from a zero state: outputs for every
 * position, records 0..len[b]-1, fill = len[b] (whatever the buffer held before
 * is discarded).  `state` is neither read nor written.  Decoding then continues
 * with kvb_decode (state NULL), and kvb_flush on a zeroed state folds the
 * records into a state once the context outgrows the buffer.
 *   len   device int32 [B], 0..Lmax        Lmax 1..min(cap, KVB_MAX_DIRECT_LEN); above 64 only for
 *         16-bit inputs with d = 128 (KVB_EUNSUPPORTED otherwise)
 *   q, k  device [B, Lmax, Hk, dk]  v device [B, Lmax, Hv, dv]  g, beta device [B, Lmax, Hv]
 *   out   device [B, Lmax, Hv, dv] out_dtype; rows >= len[b] are not written
 * len[b] outside 0..Lmax is clamped to Lmax with KVB_STATUS_OVERFLOW.
 * With a 16-bit rec_dtype the outputs read the records as stored (rounded), like everywhere
 * else; a row's delta value reads the stored records of the rows solved before it, and the
 * rows solved with it as follows.  d = 128: 64 rows are solved for in fp32 and rounded
 * afterwards, so none sees the rounding of the others.  d = 32 and 64: 16 rows are solved for in
 * fp32, and once more from the rounded values of that first solution; the second solution is
 * rounded and stored (it differs from solving row by row only where rounding the first one
 * differs from rounding the second).
 * A head of a context whose outputs are not all finite is solved token by token (slower).
 */
int kvb_direct(const kvb_shape *shape, const kvb_store *store, const int32_t *slot,
               const int32_t *len, int32_t Lmax,
               const void *q, const void *k, const void *v,
               const float *g, const float *beta, void *out, void *stream);

/*
 * Whole sequences: ragged, packed along one token axis.  Sequence b's tokens are rows start[b] .. start[b+1]-1 of
 * every token array (an empty sequence is fine).  shape: B sequences; cap and rec_dtype are not looked at.
 */
typedef struct kvb_seqs {
    const int32_t *start;    /* device [B+1], ascending, within 0..n_tokens (cut off to that)          */
    const int32_t *slot;     /* device [B]: sequence b's states are row slot[b] of the state arrays; a
                                sequence whose slot is outside 0..n_slots-1 is skipped, no slot may
                                appear twice.  NULL: row b                                             */
    int64_t  q_stride;       /* elements from one token's row of q to the next, so that q, k and v may */
    int64_t  k_stride;       /* be parts of the rows of one projection: at least the row, in bytes a   */
    int64_t  v_stride;       /* multiple of 16, at most 2^26; 0: packed.  Heads of a token are contiguous */
    int32_t  n_tokens;       /* rows of the token arrays                                               */
    int32_t  n_slots;        /* rows of the state arrays                                               */
} kvb_seqs;

/*
 * kvb_scan -- the recurrence over whole sequences of any length, the way a prompt that no record
 * buffer holds enters a state (and the forward pass of training).  From state0, for each token in order,
 *      e_t = v_t - alpha_t k_t S,  S <- alpha_t S + beta_t k_t^T e_t,  o_t = scale q_t S       (Eq. 11-12)
 * in chunks of 64 tokens (a few tokens: one by one) with all arithmetic to fp32 (16-bit inputs are exact).
 *   q, k    device [n_tokens, Hk, dk] in_dtype     v  device [n_tokens, Hv, dv] in_dtype
 *   g, beta device [n_tokens, Hv] fp32
 *   state0  device [n_slots, Hv, dk, dv] fp32, or NULL: zero
 *   state1  the same, written: the state behind the last token (an empty sequence's is its state0); NULL:
 *           not wanted.  May be state0.  With a store's state array and the requests' slots, kvb_decode
 *           and the other calls go on from there (the record buffers must be empty, fill 0).
 *   out     device [n_tokens, Hv, dv] out_dtype, packed
 *   work    device, kvb_scan_work(shape, seqs) bytes, 16-byte aligned; what it holds means nothing
 *           before and after the call.  kvb_scan_work depends on B, Hv and n_tokens alone, grows with
 *           them, and returns one of the error codes for what the call would refuse.
 * Head sizes and types as elsewhere: dk == dv in {32, 64, 128}, fp32, bf16 or fp16.
 * Whether tokens go one by one or in chunks is decided by their average number a sequence (up to 4: one by one): a long sequence among
 * many that are empty or short is better given a call of its own.
 * A value that is not finite may make NaN of any output of its head in the 64-token chunk that holds it (counted from the
 * sequence's start) and behind it; log decays down to -infinity are fine.
 */
int64_t kvb_scan_work(const kvb_shape *shape, const kvb_seqs *seqs);
int kvb_scan(const kvb_shape *shape, const kvb_seqs *seqs,
             const void *q, const void *k, const void *v, const float *g, const float *beta,
             const float *state0, float *state1, void *out, void *work, void *stream);

/*
 * kvb_scan_backward -- the gradients of kvb_scan, from those of its outputs and last states.  The forward pass leaves
 * nothing for it: states and triangular systems are worked out once more from the inputs.
 *   q .. state0  as kvb_scan was given them (n_slots, slots and strides too)
 *   dout     device [n_tokens, Hv, dv] out_dtype, packed
 *   dstate1  device [n_slots, Hv, dk, dv] fp32, or NULL: zero
 *   dq, dk, dv  device, written: in_dtype, strides of q, k and v.  q and k of a qk-head get the sum over its v-heads
 *   dg, dbeta   device [n_tokens, Hv] fp32, written; dg is the gradient of the log decay
 *   dstate0  device [n_slots, Hv, dk, dv] fp32, written, or NULL: not wanted.  May be dstate1
 *   work     device, kvb_scan_backward_work(shape, seqs) bytes, 16-byte aligned: at d = 128 some 257 KB for each 64 tokens
 *            of a v-head, the state and its gradient at each chunk's start above all (kvb_scan: 37 KB)
 * Rows of skipped sequences are not written.  The same inputs give the same bits.  16-bit gradients are rounded once from sums to
 * within 2^-16 of their terms (dq: 2^-24), all else is held to fp32.
 */
int64_t kvb_scan_backward_work(const kvb_shape *shape, const kvb_seqs *seqs);
int kvb_scan_backward(const kvb_shape *shape, const kvb_seqs *seqs,
                      const void *q, const void *k, const void *v, const float *g, const float *beta, const float *state0,
                      const void *dout, const float *dstate1, void *dq, void *dk, void *dv,
                      float *dg, float *dbeta, float *dstate0, void *work, void *stream);

#define KVB_MAX_VOCAB (1 << 24) /* largest V of kvb_accept */

typedef struct kvb_vocab {
    int32_t B;       /* requests                                              */
    int32_t T;       /* drafts a request has room for, 1..KVB_MAX_DRAFTS         */
    int32_t V;       /* tokens of the vocabulary, 1..KVB_MAX_VOCAB               */
    int32_t dtype;   /* of the probabilities: KVB_F32, KVB_BF16 or KVB_F16       */
    int64_t stride;  /* elements from one row of probabilities to the next; 0: V */
} kvb_vocab;

/*
 * kvb_accept -- which of the drafted tokens the target model accepts, from given random numbers, and the token that
 * follows them: what comes between kvb_verify (whose outputs lead to the target's probabilities) and the commit.  Together
 * the accepted drafts and the token are distributed as the target's own samples.
 *   n_drafts device int32 [B]: drafts that request b has, 0..T (cut off to that); NULL: T each
 *   parent   device int32 [B, T], as kvb_verify_tree's; NULL: a chain.  An entry outside -1 .. i-1 is taken as -1
 *   tokens   device int32 [B, T]: the drafted tokens.  One outside 0..V-1 is never accepted
 *   target   device [B, T+1, V] dtype: row 0 the target's probabilities behind the last committed token, row i + 1 those
 *            behind draft i
 *   draft    device [B, T, V] dtype: row i the probabilities that draft i was drawn from (siblings: independently); NULL: drafts
 *            that were not drawn but chosen (the best tokens of a draft head, say), as if each was certain
 *   u        device fp32 [B, T], s  device fp32 [B]: random numbers, uniform in [0, 1)
 *   path     device int32 [B, T]: the accepted drafts, oldest first, then -1: kvb_compact's path
 *   accepted device int32 [B]: how many: kvb_compact's path_len, kvb_flush's accepted
 *   token    device int32 [B]: the token that follows the last accepted draft
 *   work     device, kvb_accept_work(vocab) bytes, 8-byte aligned; what it holds means nothing before and after the call.
 *            kvb_accept_work grows with B and V: what it gives for the largest batch serves smaller ones
 * The walk starts at row 0 with r = the row and Z = 1 and looks at the drafts in order; draft i is tested if its parent is where
 * the walk stands.  It is accepted if u_i q_i(x_i) Z < r(x_i); then the walk stands at it, r is its row and Z = 1.
 * Otherwise r becomes max(r - Z q_i, 0) and Z its sum; for chosen drafts r(x_i) becomes 0 and Z loses what it was.  The token is
 * drawn from r (from the row itself if nothing is left of r, -1 if that has nothing either): weights are r cut off to 0..1
 * in whole multiples of 2^-48, rounded down, and the token is the first whose running sum exceeds floor(s W) in fp64, W their sum.
 * Each operation is one rounding in fp32, sums are exact: the results do not depend on the launch.  (Rows that sum to more than 32 are
 * no probabilities; they get one of their tokens, but which of those next to s W may depend on it.)  A probability of the target
 * that is not a number counts as 0, one of a draft as infinity: a draft whose own is none is not accepted (as 0 it always would be).
 */
int64_t kvb_accept_work(const kvb_vocab *vocab);
int kvb_accept(const kvb_vocab *vocab, const int32_t *n_drafts, const int32_t *parent, const int32_t *tokens,
               const void *target, const void *draft, const float *u, const float *s,
               int32_t *path, int32_t *accepted, int32_t *token, void *work, void *stream);

/*
 * Around the recurrence: what makes a layer's q, k, v, g and beta from the rows of its projection (kvb_conv and its forms), the norms ahead of a
 * block and behind the recurrence (kvb_norm), and the norm of all gradients together (kvb_grad_norm, kvb_clip).
 */
#define KVB_MIN_EPS   1e-30f   /* least eps of kvb_taps and kvb_rows */
#define KVB_CONV_UNIT 1   /* kvb_taps.flags: q and k are divided by sqrt(sum of squares over the head + eps) */

typedef struct kvb_taps {
    const void  *weight;     /* device [C, width] in_dtype, C = (2 Hk + Hv) dk channels: q's, k's, v's, head by head.  The last    */
                             /* tap is the token's own                                                                           */
    const void  *bias;       /* device [C] in_dtype, or NULL: none                                                               */
    const float *A_log;      /* device [Hv] fp32, for the gates                                                                  */
    const float *dt_bias;    /* device [Hv] fp32, for the gates                                                                  */
    int64_t      x_stride;   /* elements from one token's row of x to the next: at least C, in bytes a multiple of 16, at most 2^26;
                                0: packed.  So that x may be part of the rows of one projection                                  */
    int64_t      a_stride;   /* the same of a and b: at least Hv, at most 2^26; 0: packed                                        */
    int64_t      b_stride;
    int32_t      width;      /* 2, 3 or 4 taps                                                                                   */
    int32_t      flags;      /* KVB_CONV_UNIT                                                                                    */
    float        eps;        /* at least KVB_MIN_EPS with KVB_CONV_UNIT                                                          */
} kvb_taps;

/*
 * kvb_conv -- whole sequences (kvb_seqs, ragged and packed).  With E the width - 1 rows of the sequence's state followed by its inputs,
 *      z_t = bias + sum_i weight_i E_{t+i}      y = z / (1 + exp(-z))      q, k, v = y, q and k of length one (KVB_CONV_UNIT)
 *      g = -exp(A_log) log(1 + exp(a + dt_bias))      beta = 1 / (1 + exp(-b))
 *   shape   B, Hk, Hv, dk == dv in {32, 64, 128}, in_dtype; the rest is not looked at
 *   x       device [n_tokens, C] in_dtype         a, b  device [n_tokens, Hv] in_dtype; both NULL: no gates are wanted, g and beta are NULL too
 *   state0  device [n_slots, width - 1, C] in_dtype, the last inputs, oldest first; NULL: zero
 *   state1  the same, written: the state behind the last token (an empty sequence's is its state0); NULL: not wanted.  May be state0
 *   q, k, v device, written: [n_tokens, Hk or Hv, dk] in_dtype, strides of seqs
 *   g, beta device, written: [n_tokens, Hv] fp32
 * All arithmetic is fp32, results are rounded once.  What is written must not overlap x, a and b.
 * Rows of skipped sequences (slot outside 0..n_slots-1) are not written.  Where start does not ascend, what its sequences give, and which of their tokens
 * are done, is not said, here and in kvb_conv_backward; nothing outside them is read or written.
 * A call that would take 2^32 threads is refused, here and below: 64 for each 512
 * channels, and for the gates, of each token or draft, here of up to 64 tokens (each sequence is as much as 8 more).
 */
int kvb_conv(const kvb_shape *shape, const kvb_taps *taps, const kvb_seqs *seqs, const void *x, const void *a, const void *b,
             const void *state0, void *state1, void *q, void *k, void *v, float *g, float *beta, void *stream);

/*
 * kvb_conv_decode -- kvb_conv for one token of each request, as kvb_decode wants them.  slot device int32 [B] (not NULL, none twice), rows of n_slots
 * states; x [B, C], a, b [B, Hv]; q, k, v, g, beta packed; state0 and state1 as above (state1 may be state0).
 */
int kvb_conv_decode(const kvb_shape *shape, const kvb_taps *taps, const int32_t *slot, int32_t n_slots, const void *x, const void *a, const void *b,
                    const void *state0, void *state1, void *q, void *k, void *v, float *g, float *beta, void *stream);

/*
 * kvb_conv_verify -- the same for T drafts of each request, as kvb_verify and kvb_verify_tree want them: draft i's taps reach back over its ancestors
 * and then the state.  The state is left alone.
 *   T       1..KVB_MAX_DRAFTS       x device [B, T, C], a, b [B, T, Hv] (the strides from draft to draft, requests follow each other); q .. beta packed
 *   parent  device int32 [B, T] as kvb_verify_tree's, or NULL: a chain.  An entry outside -1 .. i-1 is taken as -1
 */
int kvb_conv_verify(const kvb_shape *shape, const kvb_taps *taps, const int32_t *slot, int32_t n_slots, int32_t T, const int32_t *parent,
                    const void *x, const void *a, const void *b, const void *state, void *q, void *k, void *v, float *g, float *beta, void *stream);

/*
 * kvb_conv_commit -- the accepted drafts of a preceding kvb_conv_verify enter the state: state1 becomes the last width - 1 rows of state0 and theirs.
 *   path     device int32 [B, T], kvb_accept's or kvb_compact's: the accepted drafts, oldest first; NULL: drafts 0, 1, .. of a chain
 *   accepted device int32 [B]: how many, 0..T
 *   x        as kvb_conv_verify was given it
 *   state0, state1  as above, state1 not NULL.  May be the same
 * A path that is not increasing within 0..T-1 or a number outside 0..T commits nothing: state1 becomes state0 (kvb_compact reports these).
 */
int kvb_conv_commit(const kvb_shape *shape, const kvb_taps *taps, const int32_t *slot, int32_t n_slots, int32_t T, const int32_t *path,
                    const int32_t *accepted, const void *x, const void *state0, void *state1, void *stream);

/*
 * kvb_conv_backward -- the gradients of kvb_conv, from those of its outputs and last states.
 *   x .. state0     as kvb_conv was given them (a and b NULL: no gates; dg, dbeta, da, db, dA_log and ddt_bias are NULL too.  Without any
 *                   tokens dA_log and ddt_bias alone count, which become 0)
 *   dq, dk, dv      device in_dtype, strides of q, k and v in seqs         dg, dbeta  device [n_tokens, Hv] fp32
 *   dstate1         device [n_slots, width - 1, C] in_dtype, or NULL: zero
 *   dx, da, db      device, written: in_dtype, strides of x, a and b
 *   dweight, dbias  device [C, width], [C] fp32, written; dbias is NULL if and only if there is no bias
 *   dA_log, ddt_bias  device [Hv] fp32, written
 *   dstate0         device [n_slots, width - 1, C] in_dtype, written, or NULL: not wanted.  Not dstate1
 *   work            device, kvb_conv_backward_work(shape, taps, seqs) bytes, 16-byte aligned; what it holds means nothing before and after the call.
 *                   It grows with B and n_tokens; another shape or other taps have sizes of their own, which may be more for fewer channels
 * What is written must not overlap what is read.  Rows of skipped sequences are neither written nor counted in the sums.  The same inputs give the
 * same bits.
 */
int64_t kvb_conv_backward_work(const kvb_shape *shape, const kvb_taps *taps, const kvb_seqs *seqs);
int kvb_conv_backward(const kvb_shape *shape, const kvb_taps *taps, const kvb_seqs *seqs, const void *x, const void *a, const void *b,
                      const void *state0, const void *dq, const void *dk, const void *dv, const float *dg, const float *dbeta, const void *dstate1,
                      void *dx, void *da, void *db, float *dweight, float *dbias, float *dA_log, float *ddt_bias, void *dstate0, void *work,
                      void *stream);

#define KVB_MAX_WIDTH 16384 /* longest row of kvb_norm */

typedef struct kvb_rows {
    int64_t x_stride;     /* elements from one token's rows of x to the next, of gate: at least heads * width, in bytes a multiple of 16,  */
    int64_t gate_stride;  /* at most 2^26; 0: packed.  A token's heads follow each other                                                  */
    int32_t n_tokens;
    int32_t heads;        /* rows of a token, each with a norm of its own                                                                 */
    int32_t width;        /* elements of a row: a multiple of 8, 8..KVB_MAX_WIDTH                                                         */
    int32_t dtype;        /* of gate, weight and out: KVB_F32, KVB_BF16 or KVB_F16                                                        */
    int32_t x_dtype;      /* of x, res and sum: KVB_F32 or dtype                                                                          */
    float   eps;          /* at least KVB_MIN_EPS                                                                                        */
    float   scale;        /* of x where there is a residual, 1 where there is none                                                        */
} kvb_rows;

/*
 * kvb_norm -- the root mean square norm of rows, with the residual ahead of it and the gate behind it:
 *      s = res + scale x, rounded to x_dtype (x itself without a residual)      out = s / sqrt(mean s^2 + eps) weight gate / (1 + exp(-gate))
 * Behind the recurrence: x its outputs (fp32 or 16 bits), heads = Hv, width = dv, gate from the layer's projection.  Ahead of a block: heads = 1, x what
 * the block before put out, res the stream that it is added to.
 *   x       device [n_tokens, heads, width] x_dtype         res   the same, packed, or NULL: none
 *   gate    device [n_tokens, heads, width] dtype, or NULL: none       weight  device [width] dtype
 *   sum     device, written: s, packed, or NULL: not wanted.  Without a residual NULL.  May be res, or x where that lies packed
 *   out     device, written: [n_tokens, heads, width] dtype, packed.  May be x (of the same type) or gate where they lie packed
 * All arithmetic is fp32; squares above the range of fp32 make a row 0.  Rows above 2048 elements: at most 2^24 - 2, above 8192 half as many.
 */
int kvb_norm(const kvb_rows *rows, const void *x, const void *res, const void *gate, const void *weight, void *sum, void *out, void *stream);

/*
 * kvb_norm_backward -- the gradients of kvb_norm.
 *   x        what the norm was taken of: kvb_norm's sum where there was a residual, else its x; x_stride is this array's
 *   gate, weight  as kvb_norm was given them          dout  device [n_tokens, heads, width] dtype, packed
 *   dsum     device x_dtype, packed: the gradient of sum from what else it went to; NULL: zero
 *   dx       device, written: x_dtype, lies as x does; scale times the gradient of s
 *   dres     device, written: x_dtype, packed: the gradient of s; NULL: not wanted.  May be dsum
 *   dgate    device, written: dtype, lies as gate does; NULL if and only if there is no gate
 *   dweight  device [width] fp32, written
 *   work     device, kvb_norm_backward_work(rows) bytes, 16-byte aligned; means nothing before and after the call.  It grows with n_tokens
 *            and heads; other widths have sizes of their own, which may be more for a narrower row
 * What is written must not overlap what is read otherwise.  The same inputs give the same bits.
 */
int64_t kvb_norm_backward_work(const kvb_rows *rows);
int kvb_norm_backward(const kvb_rows *rows, const void *x, const void *gate, const void *weight, const void *dout, const void *dsum, void *dx,
                      void *dres, void *dgate, float *dweight, void *work, void *stream);

#define KVB_LIST_BLOCK 16384

typedef struct kvb_list {       /* some tensors, none of which share memory; all arrays are on the device            */
    void *const   *data;        /* [n] addresses, each aligned to its elements                                       */
    const int64_t *size;        /* [n] elements, 0 is fine                                                           */
    const int32_t *type;        /* [n] KVB_F32, KVB_BF16 or KVB_F16                                                  */
    const int32_t *first;       /* [n+1] running sum of ceil(size / KVB_LIST_BLOCK), from 0                          */
    int32_t        n;
    int32_t        blocks;      /* first[n]; below 2^24 - 1: 256 threads a block                                     */
} kvb_list;

/*
 * kvb_grad_norm -- norm = the root of the sum of squares of all elements (summed in fp64).
 *   norm  device fp32 [1], written       work  device, kvb_grad_norm_work(list) bytes, 8-byte aligned; means nothing before and after the call.  It grows with
 *                                              blocks and depends on nothing else: what it gives for the longest list serves shorter ones
 */
int64_t kvb_grad_norm_work(const kvb_list *list);
int kvb_grad_norm(const kvb_list *list, float *norm, void *work, void *stream);

/*
 * kvb_clip -- every element times min(1, largest / (norm + 1e-6)), in fp32, rounded once.
 *   to       tensors of the same sizes and types (only data is looked at), or NULL: in place.  None may overlap another's source
 *   norm     device fp32 [1]: kvb_grad_norm's, or what ranks that hold a part each have made of theirs
 *   largest  at least 0
 * A result that lies otherwise among 16 bytes than its source is written element by element, in about twice the time.
 * Where nothing is to be cut, nothing is written in place.  A norm that is infinite makes every finite element 0, one that is not a number all NaN.
 */
int kvb_clip(const kvb_list *list, const kvb_list *to, const float *norm, float largest, void *stream);

/*
 * Kernel timer (measurement aid, no part of the method).  A timer owns two HIP events.
 * kvb_timer_arm makes the NEXT kernel that the calling thread launches through this
 * library record its own begin and end timestamps into them; kvb_timer_read waits for that
 * kernel and returns its duration (a call of several kernels: from the first one's begin to the last one's end).  Timers are host objects: create / destroy allocate and
 * free them, the only allocation this library ever performs.  Do not arm during stream capture.
 */
typedef struct kvb_timer kvb_timer;
int  kvb_timer_create(kvb_timer **timer);
int  kvb_timer_arm(kvb_timer *timer);          /* NULL disarms */
int  kvb_timer_read(kvb_timer *timer, float *microseconds);
void kvb_timer_destroy(kvb_timer *timer);

/* Static text for a return code (for KVB_EHIP: the last HIP error string of this thread). */
const char *kvb_strerror(int code);

/* KVB_VERSION of the built library. */
int kvb_version(void);

#ifdef __cplusplus
}
#endif
#endif /* KVB_H */
