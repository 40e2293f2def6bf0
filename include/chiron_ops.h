/*
 * chiron_ops.h: the individual kernels of the decode step, exported so that each can be
 * checked against the plain definition and timed on its own.  chiron_decode_step (chiron.h)
 * is the product call; these run exactly the kernels it runs.
 *
 * Same conventions as chiron.h: int32 status return, dev/host pointers, `stream` is a
 * hipStream_t as void*, calls enqueue and do not synchronise.  Activations are fp32,
 * weights/gains/cache are bf16 bit patterns.
 */
#ifndef CHIRON_OPS_H
#define CHIRON_OPS_H

#include <stdint.h>

#include "chiron.h"

#ifdef __cplusplus
extern "C" {
#endif

/* out[r][j] = h[r][j] * gain[j] / sqrt(mean_j(h[r][j]^2) + eps); h, out dev fp32 [rows, n]; gain dev bf16 [n]. */
int32_t chiron_op_rmsnorm(const float *h, const void *gain, int32_t rows, int32_t n, float eps, float *out,
                          void *stream);

/* A weight matrix repacked into matrix-core tile order (library-owned device copy). */
typedef struct chiron_linear chiron_linear;
/* w dev bf16 [N, K] (out, in) row-major; any N >= 1 (padded to 32 inside), K a multiple of 16. */
int32_t chiron_linear_create(const void *w, int32_t N, int32_t K, void *stream, chiron_linear **out);
int32_t chiron_linear_destroy(chiron_linear *l);

/* y[M,N] = x[M,K] * W^T (accumulate == 0) or y += x * W^T (accumulate != 0, the residual add).
 * x, y dev fp32 row-major; they may overlap (a square matrix applied in place), which costs a pass over the result.
 * x is split into two bf16 terms, products accumulate in fp32. */
int32_t chiron_op_linear(const chiron_linear *l, const float *x, int32_t M, float *y, int32_t accumulate,
                         void *stream);

/* The fused gate/up matrix of a feed-forward block: w_gate, w_up dev bf16 [F, K] each, row-major, F and K multiples
 * of 16.  The library's copy interleaves the two so that gate column j and up column j are produced by one wave; it
 * goes with the two SwiGLU entry points below only (chiron_op_linear refuses it). */
int32_t chiron_linear_create_gate_up(const void *w_gate, const void *w_up, int32_t F, int32_t K, void *stream,
                                     chiron_linear **out);

/* SwiGLU fused into the gate/up projection's epilogue:
 *     act[m][j] = silu(gate[m][j]) * up[m][j],  gate = x * Wg^T,  up = x * Wu^T,  silu(z) = z / (1 + exp(-z)).
 * x dev fp32 [M, K]; act dev fp32 [M, F], caller-owned. */
int32_t chiron_op_gate_up_swiglu(const chiron_linear *gate_up, const float *x, int32_t M, float *act, void *stream);

/* The feed-forward block as the decode step runs it, two launches:  y (+)= act * Wd^T  with act as above.
 * down is a plain chiron_linear over Wd [N, F].  The intermediate never leaves the library: fp32 rows with few rows,
 * and from the row count of the linear_big_min_m knob on the two bf16 terms of act in the tile order that the down
 * projection copies straight into LDS.  x dev fp32 [M, K]; y dev fp32 [M, N]. */
int32_t chiron_op_swiglu_ffn(const chiron_linear *gate_up, const chiron_linear *down, const float *x, int32_t M,
                             float *y, int32_t accumulate, void *stream);

/* Rotary embedding in place: x dev fp32 [rows, n_heads, d]; row r is rotated for position pos[r]
 * (pairs (j, j+d/2), angle pos*base^(-2j/d), angles evaluated in fp64). */
int32_t chiron_op_rope(float *x, int32_t rows, int32_t n_heads, int32_t d, const int32_t *pos, float base,
                       void *stream);

/* chiron_op_rope for callers that cannot allocate device memory (code under HIP graph capture, tight serving
 * loops, harnesses that forbid hipMalloc): same arguments, same kernels, bit-identical result, but the cos/sin
 * table the two kernels share lives in a fixed 1 MiB device array inside the library (one per GPU, held until the
 * process ends) instead of a stream-ordered allocation.  The call itself allocates nothing.  Limit: rows * d <=
 * 262144 (e.g. 2048 rows at head_dim 128); beyond it CHIRON_ERR_SHAPE and nothing is launched.  All calls on one
 * GPU share the array: calls that overlap there (different streams or threads) race; calls on one stream do not. */
int32_t chiron_op_rope_noalloc(float *x, int32_t rows, int32_t n_heads, int32_t d, const int32_t *pos, float base,
                               void *stream);

/* Paged GQA decode attention of one layer: for request i and query head a (KV head a / G)
 *     out[i][a] = softmax_t(q[i][a] . K_t / sqrt(d)) . V_t   over positions t < ctx_lens[i]
 * of the request's paged cache.  q, out dev fp32 [batch, n_q_heads*head_dim]; ctx_lens dev
 * int32 [batch], each >= 1.  Uses the model's attention workspace (split-K partials). */
int32_t chiron_op_paged_attention(chiron_model *m, const chiron_kvpool *p, int32_t layer, const float *q,
                                  const int32_t *block_table, const int32_t *ctx_lens, int32_t batch, float *out,
                                  void *stream);

/* cos/sin [rows, d/2] dev fp32 of the angles pos[r]*base^(-2j/d), evaluated in fp64: the table that chiron_append_kv_rope
 * takes, one for all layers of a step. */
int32_t chiron_op_rope_table(const int32_t *pos, int32_t rows, int32_t d, float base, float *cos, float *sin, void *stream);

/* ---- block-sparse attention of new tokens: select pages by a cheap score, attend over those only --------------
 *
 * Row r is one new token: of request row_seq[r] (dev int32 [rows], null: of request r), seeing the first ctx_lens[r]
 * (dev int32 [rows], >= 0) positions of it, its own among them.  q dev fp32 [rows, n_q_heads*head_dim], rotated.
 *
 * Selection, for each row and KV head c, over the pages 0 .. ceil(ctx_lens[r]/16)-1:
 *     q8[h]    = round(q[h] / 2^f), ties to even, 2^f as an index record's 2^e over the G query heads of c
 *     score(p) = 2^e(p) * max_h sum_j (q8[h][j] > 0 ? q8[h][j]*hi(p)[j] : q8[h][j]*lo(p)[j])
 * which (but for the rounding of q) bounds q . k from above for every token of the page.  The first n_first and the last
 * n_last pages are always taken, then the pages of the highest scores, equal ones by the lower page, `top` in all.  Whole
 * number arithmetic: a selection does not depend on the batch or on how the work was split.  NaN in q counts as 0 and
 * infinities as the largest finite value.
 *   pages   dev int32 [rows, n_kv_heads, top]: page indices of the request (columns of its block table), ascending, then -1
 *   counts  dev int32 [rows] (optional): min(top, pages of the row)
 * n_first, n_last >= 0, n_first + n_last <= top. */
int32_t chiron_op_select_pages(chiron_model *m, const chiron_kvpool *p, const chiron_kvindex *x, int32_t layer, const float *q,
                               const int32_t *block_table, const int32_t *row_seq, const int32_t *ctx_lens, int32_t rows,
                               int32_t top, int32_t n_first, int32_t n_last, int32_t *pages, int32_t *counts, void *stream);

/* out[r][a] = softmax_t(q[r][a] . K_t / sqrt(d)) . V_t over the tokens t < ctx_lens[r] of the pages listed for (r, a / G)
 * in pages[r][a / G][0 .. counts[r]-1] (counts null: all `top` entries).  Lists may be any, in any order, without an
 * entry twice; entries that name no page of the row (negative, or behind ctx_lens[r]) count for nothing; a row that sees
 * no token gets zeros.  out dev fp32 [rows, n_q_heads*head_dim].
 * Slots behind ctx_lens[r] may hold anything.  NaN and infinities that a row does attend, and in q, leave undefined what they
 * meet and nothing else: one in a key the row's outputs of its KV head, one in a value its own dim of these (which is then no
 * finite number), one in q its own head's.  (q and the weights go through the products in three terms, of which some are 0.) */
int32_t chiron_op_sparse_attention(chiron_model *m, const chiron_kvpool *p, int32_t layer, const float *q,
                                   const int32_t *block_table, const int32_t *row_seq, const int32_t *ctx_lens, int32_t rows,
                                   const int32_t *pages, const int32_t *counts, int32_t top, float *out, void *stream);
/* Both use the model's attention workspace (rows <= max_batch; calls on one model must not overlap).  Tables of more than
 * (8192 + 2 max_batch) * G * head_dim columns, 8 million tokens at the least, have no room in it for one row's scores: the selection
 * refuses them. */

/* ---- verification of drafted tokens ---------------------------------------------------------------------------
 *
 * Request i drafted n_i = draft_lens[i] (0 .. max_draft; null: max_draft) tokens x_t = tokens[i][t]; logits[i][t] are the
 * target's after the token before x_t (chiron_decode_step_multi fed with the last token and the drafts), draft_logits[i][t]
 * the draft's at the same place.  With p, q the softmax of logits / temperature[i] (null: 1) over the vocabulary:
 *     prob[i][t] = min(1, p_t(x_t) / q_t(x_t))         (q(x) = 0: 1 if p(x) > 0, else 0; t >= n_i: 0)
 *     a          = the first t < n_i with uniforms[i][t] >= prob[i][t], or n_i: the number of accepted tokens
 *     new token  = argmax_x r(x) / noise[i][x],  r = max(p_a - q_a, 0) if a < n_i (p_a where that is 0 everywhere), else p_a
 *     out_tokens[i] = x_0 .. x_{a-1}, new token, -1, ...
 * With uniforms uniform in [0,1) and noise from the unit exponential distribution the tokens are distributed as the target's
 * own samples.  draft_logits null: drafts that were not sampled (q is 1 at x_t).  temperature 0 (or no number above it): the greedy choice:
 * prob is 1 where x_t has the highest logit (of equal ones the lowest token), else 0, and the new token has the highest.  temperature
 * +inf: the same share for every token whose logit is above -inf.
 * NaN logits count as -inf, +inf as the largest finite value; in a row without any logit above -inf every p is 0 and the new token -1.
 * A drafted token outside 0 .. vocab-1 has prob 0.
 *   logits        dev fp32 [batch][max_draft+1][vocab], row (i,t) at logits + (i*(max_draft+1)+t)*logits_stride
 *   draft_logits  dev fp32 [batch][max_draft][vocab], row stride draft_stride, or null
 *   tokens        dev int32 [batch, max_draft];  uniforms dev fp32 [batch, max_draft];  noise dev fp32 [batch][vocab] (contiguous)
 *   out_tokens    dev int32 [batch, max_draft+1];  accepted dev int32 [batch];  prob dev fp32 [batch, max_draft] (optional)
 *   workspace     dev, chiron_verify_workspace_bytes() bytes, 16-byte aligned, caller-owned, in use until the stream has passed
 * 0 <= max_draft <= 127; batch * (2 max_draft + 1) <= 65535, with draft_logits or without (more requests: several calls). */
int64_t chiron_verify_workspace_bytes(int32_t batch, int32_t max_draft, int32_t vocab);
typedef struct {
    const float *logits, *draft_logits;
    int64_t logits_stride, draft_stride;
    const int32_t *tokens, *draft_lens;
    const float *uniforms, *noise, *temperature;
} chiron_draft_batch;
int32_t chiron_op_verify_drafts(const chiron_draft_batch *in /* host */, int32_t batch, int32_t max_draft, int32_t vocab,
                                int32_t *out_tokens, int32_t *accepted, float *prob, void *workspace, void *stream);

/* ---- products with 4-bit weights ------------------------------------------------------------------------------
 *
 * W[n][k] = (w4[n][k] - z[n][k/group]) * scale[n][k/group], w4 in 0 .. 15, z in 0 .. 64 (null: 8 everywhere; one above 64 is an
 * invalid argument, and with zero points the call waits for the stream to find out).
 *   w4      dev uint8 [N, K/2]: k even in the low four bits, k odd in the high four
 *   scales  dev bf16 [N, K/group];  zeros dev uint8 [N, K/group] or null
 * group 32, 64 or 128, K a multiple of group below 2^23, any N >= 1.  The library keeps its own repacked copy. */
typedef struct chiron_linear4 chiron_linear4;
int32_t chiron_linear4_create(const void *w4, const void *scales, const void *zeros, int32_t N, int32_t K, int32_t group,
                              void *stream, chiron_linear4 **out);
int32_t chiron_linear4_destroy(chiron_linear4 *l);

/* y[M,N] = x[M,K] * W^T, or y += (accumulate != 0).  x, y dev fp32 row-major, not overlapping.  An element of x enters with an
 * error of at most 2^-22 of itself and 2^-30.9 of the largest of its row's 128 inputs (or 2^-128): few rows as whole multiples of a
 * power of two in four 8-bit digits, many rows as two fp16 terms.  Sums over the groups are fp32.  A NaN or an infinity in a
 * row of x makes that row of y NaN.  M <= 65535. */
int32_t chiron_op_linear4(const chiron_linear4 *l, const float *x, int32_t M, float *y, int32_t accumulate, void *workspace,
                          void *stream);
/* workspace: dev, that many bytes, 16-byte aligned, caller-owned, in use until the stream has passed; 0 (null
 * will do) for few rows of few inputs. */
int64_t chiron_linear4_workspace_bytes(const chiron_linear4 *l, int32_t M);

/* Performance knobs of the kernels, process-wide (0 restores the built-in heuristic where one exists):
 *   linear_nf (1|2|4), linear_mt (1|2|3|4), linear_xcd_remap (0|1), linear_ksplit, linear_target_blocks,
 *   linear_big_min_m (rows from which the gate/up projection hands the down projection tiled bf16 terms; <0 never),
 *   linear_big_all (1: from that row count on every other projection's input is split into such terms first),
 *   linear_ks (4|8|16: k-steps per chunk, the depth of the weight ring),
 *   attn_grid, attn_target_waves, attn_chunk_pages.
 * They change launch shapes only, never results beyond summation order (up to 16 rows a forced linear_nf, linear_mt,
 * linear_ksplit, linear_ks or linear_big_all also keeps the tiled kernels instead of the few-row ones). Unknown keys are
 * an error. */
int32_t chiron_set_tuning(const char *key, int32_t value);

#ifdef __cplusplus
}
#endif
#endif /* CHIRON_OPS_H */
