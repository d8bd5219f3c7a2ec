/*
 * cx_lm.h -- C ABI of the language-model operators of the MI355X (gfx950) library: what a simulated worker's training step
 * computes before and after its matrix products, so that its gradient row is ready for the optimizer steps of cx_mix.h.
 *
 *   cx_embed_lookup, cx_embed_grad      embedding tables inside the workers' flat rows, and gradients into them
 *   cx_gated_scan, cx_gated_scan_grad   a gated linear recurrence over long sequences; its single-token step
 *   cx_token_scores                     log probabilities of given tokens, entropy, the largest logits
 *   cx_distill_loss / _grad / _step     distillation from a teacher's top logits, with the label's cross entropy
 *
 * Common conventions
 *   types      every operator has three entry points: float32, bfloat16 (suffix _bf16) and IEEE binary16 (suffix _f16);
 *              16-bit elements are passed as uint16_t bit patterns.  Elements are widened exactly, sums, states and
 *              statistics are fp32, every result is rounded once (nearest even).
 *   matrices   DEVICE memory, row-major, `ld` elements from row to row (ld >= columns); rows may begin at any element: no
 *              alignment beyond the element's own is asked for (CX_ERR_ALIGN).  Columns beyond those named are neither read
 *              nor written.
 *   stream     a hipStream_t passed as void* (NULL = the default stream).  Calls only enqueue kernels: they never
 *              synchronise, allocate or free, and may be captured into a graph.  The caller owns every buffer and keeps it
 *              alive until the stream has passed the call.
 *   workspace  scratch memory of the caller, 16-byte aligned, at least as large as the matching cx_*_workspace call says for the same
 *              sizes (of any element type; 0: NULL will do).  Nothing has to be cleared, nothing is kept in it from call to
 *              call; calls that may run at the same time need one each.
 *   results    depend on the arguments alone: no atomics on memory, sums in a fixed order.
 *   overlap    outputs overlap neither inputs nor each other (CX_ERR_ALIAS) except where a call says so.  Parts of the rows of one wider
 *              matrix do not overlap; a flat row counts from its first column to its table's end, and of two matrices of several rows
 *              and of different ld everything between the first and the last element.
 *   empty      sizes of zero tokens, rows, steps or sequences are valid; pointers to empty arrays may be NULL.
 *   return     CX_OK or a negative cx_status of cx_mix.h.  Argument errors are detected on the host before anything is
 *              enqueued: CX_ERR_NULL, CX_ERR_SHAPE (a size, a stride, a weight or the workspace's size out of range),
 *              CX_ERR_ALIGN, CX_ERR_ALIAS; CX_ERR_HIP if the runtime refuses a launch.
 */
#ifndef CX_LM_H
#define CX_LM_H

#include "cx_mix.h"

#ifdef __cplusplus
extern "C" {
#endif

#define CX_MAX_TOKENS (1 << 26)     /* tokens of a worker, rows of logits, steps of a sequence */
#define CX_MAX_SEQUENCES (1 << 22)
#define CX_MAX_VOCAB (1 << 26)
#define CX_MAX_WIDTH (1 << 20)
#define CX_MAX_TOP 64               /* alternatives of cx_token_scores */
#define CX_MAX_TEACHER 256          /* teacher's logits a row of cx_distill_* */
#define CX_SCAN_CHUNK 16            /* steps between two states that cx_gated_scan keeps for its gradient */

/* Version of this header (bumped on any signature change): 1. */
int cx_lm_abi_version(void);

/* ------------------------------------------------------------------------------------
 * cx_embed_lookup -- embedding lookup with scaling, for all W workers at once:
 *     out[w * N + n][0..D) = round(scale * table_w[tokens[w][n]][0..D))
 * where table_w is float [V][D] in columns [offset, offset + V * D) of worker w's flat parameter row x[w] (ld >= offset + V * D).
 *   tokens   int32 [W][N] DEVICE; a token outside [0, V) (padding) gives a row of zeros
 *   out      [W * N][ld_out], D columns
 * W <= CX_MAX_ROWS.
 */
int cx_embed_lookup(const float *x, int64_t ld, int32_t W, int64_t offset, int32_t V, int32_t D, const int32_t *tokens,
                    int64_t N, float scale, float *out, int64_t ld_out, void *stream);
int cx_embed_lookup_bf16(const uint16_t *x, int64_t ld, int32_t W, int64_t offset, int32_t V, int32_t D, const int32_t *tokens,
                         int64_t N, float scale, uint16_t *out, int64_t ld_out, void *stream);
int cx_embed_lookup_f16(const uint16_t *x, int64_t ld, int32_t W, int64_t offset, int32_t V, int32_t D, const int32_t *tokens,
                        int64_t N, float scale, uint16_t *out, int64_t ld_out, void *stream);

/* ------------------------------------------------------------------------------------
 * cx_embed_grad -- its gradient by sorted tokens, into the same columns of the workers' flat gradient rows:
 *     g_out[w][v] = round(g_in[w][v] + scale * sum over n with tokens[w][n] = v of dout[w * N + n])
 * summed in fp32 in an order that the tokens, the sizes and the element type alone fix: by ascending n, in parts where a token's
 * places cross one of the cuts that the sorted tokens have at equal distances, so that two occurrences may be in two parts.
 *   g_in     NULL: nothing is added, and rows that no token names become zeros;
 *            = g_out: added in place, rows that no token names are not touched (the gradient of a table that is
 *            also the output projection);  otherwise a second matrix with the same ld
 * Padding tokens are skipped; their rows of dout are not read.  Other columns of g_out are not touched.
 * The workspace holds the sorted tokens and the sums of pieces.
 */
int cx_embed_workspace(int32_t W, int64_t N, int32_t V, int32_t D, int64_t *bytes);
int cx_embed_grad(const float *dout, int64_t ld_dout, const int32_t *tokens, int32_t W, int64_t N, const float *g_in,
                  float *g_out, int64_t ld, int64_t offset, int32_t V, int32_t D, float scale, void *workspace,
                  int64_t workspace_bytes, void *stream);
int cx_embed_grad_bf16(const uint16_t *dout, int64_t ld_dout, const int32_t *tokens, int32_t W, int64_t N, const uint16_t *g_in,
                       uint16_t *g_out, int64_t ld, int64_t offset, int32_t V, int32_t D, float scale, void *workspace,
                       int64_t workspace_bytes, void *stream);
int cx_embed_grad_f16(const uint16_t *dout, int64_t ld_dout, const int32_t *tokens, int32_t W, int64_t N, const uint16_t *g_in,
                      uint16_t *g_out, int64_t ld, int64_t offset, int32_t V, int32_t D, float scale, void *workspace,
                      int64_t workspace_bytes, void *stream);

/* ------------------------------------------------------------------------------------
 * cx_gated_scan -- gated linear recurrence of B sequences of T steps and D columns:
 *     a_t = sigmoid(f_t) ;  h_t = a_t * (reset_t ? 0 : h_{t-1}) + (1 - a_t) * x_t ;  y_t = round(h_t)
 * f, x, y are matrices of B * T rows (sequence b has rows [b * T, (b + 1) * T)), each with its own ld; they may be parts of the
 * rows of one wider matrix.
 *   reset    uint8 [B][T] or NULL: nonzero where a document begins; nothing of the state before it is used, NaN
 *            and infinities included
 *   h0       float [B][D] or NULL (zeros): the state before the first step
 *   h_last   float [B][D] or NULL: receives the state after the last one; may be h0 (generation: T = 1, state in place)
 *   states   float [B][ceil(T / CX_SCAN_CHUNK)][D] or NULL: receives the state that enters every CX_SCAN_CHUNK-th step, which
 *            the gradient needs
 * Long sequences are computed as compositions of affine maps, so an infinite state may turn into a NaN.  Sequences of no more than
 * CX_SCAN_CHUNK steps need no workspace.
 */
int cx_scan_workspace(int64_t B, int64_t T, int32_t D, int64_t *bytes);
int cx_gated_scan(const float *f, int64_t ldf, const float *x, int64_t ldx, float *y, int64_t ldy, int64_t B, int64_t T,
                  int32_t D, const uint8_t *reset, const float *h0, float *h_last, float *states, void *workspace,
                  int64_t workspace_bytes, void *stream);
int cx_gated_scan_bf16(const uint16_t *f, int64_t ldf, const uint16_t *x, int64_t ldx, uint16_t *y, int64_t ldy, int64_t B, int64_t T,
                       int32_t D, const uint8_t *reset, const float *h0, float *h_last, float *states, void *workspace,
                       int64_t workspace_bytes, void *stream);
int cx_gated_scan_f16(const uint16_t *f, int64_t ldf, const uint16_t *x, int64_t ldx, uint16_t *y, int64_t ldy, int64_t B, int64_t T,
                      int32_t D, const uint8_t *reset, const float *h0, float *h_last, float *states, void *workspace,
                      int64_t workspace_bytes, void *stream);

/* ------------------------------------------------------------------------------------
 * cx_gated_scan_grad -- its gradient.  With r_t = dL/dh_t and keep_t = (reset_t ? 0 : 1):
 *     r_t = dy_t + keep_{t+1} a_{t+1} r_{t+1} ;  r_{T-1} = dy_{T-1} + dh_last
 *     dx_t = round((1 - a_t) r_t) ;  df_t = round(r_t (keep_t h_{t-1} - x_t) a_t (1 - a_t)) ;  dh0 = keep_0 a_0 r_0
 * States between those kept are computed again in fp32; y is not read.
 *   states   as the forward call left them for the same f, x, reset and h0
 *   dh_last  float [B][D] or NULL (zeros);  dh0: float [B][D] or NULL (not wanted); may be dh_last
 */
int cx_gated_scan_grad(const float *f, int64_t ldf, const float *x, int64_t ldx, const float *dy, int64_t lddy, float *df,
                       int64_t lddf, float *dx, int64_t lddx, int64_t B, int64_t T, int32_t D, const uint8_t *reset,
                       const float *states, const float *dh_last, float *dh0, void *workspace, int64_t workspace_bytes,
                       void *stream);
int cx_gated_scan_grad_bf16(const uint16_t *f, int64_t ldf, const uint16_t *x, int64_t ldx, const uint16_t *dy, int64_t lddy, uint16_t *df,
                            int64_t lddf, uint16_t *dx, int64_t lddx, int64_t B, int64_t T, int32_t D, const uint8_t *reset,
                            const float *states, const float *dh_last, float *dh0, void *workspace, int64_t workspace_bytes,
                            void *stream);
int cx_gated_scan_grad_f16(const uint16_t *f, int64_t ldf, const uint16_t *x, int64_t ldx, const uint16_t *dy, int64_t lddy, uint16_t *df,
                           int64_t lddf, uint16_t *dx, int64_t lddx, int64_t B, int64_t T, int32_t D, const uint8_t *reset,
                           const float *states, const float *dh_last, float *dh0, void *workspace, int64_t workspace_bytes,
                           void *stream);

/* ------------------------------------------------------------------------------------
 * cx_token_scores -- of N rows of V logits (scale = 1 / temperature > 0, log2(e) scale finite), p = softmax(scale * z):
 *     logp[n] = log p[tokens[n]]  (0 for a token outside [0, V)) ;  entropy[n] = -sum_v p_v log p_v
 *     top_ids[n][k], top_logp[n][k]: the K largest logits, largest first, the lower id first among equal ones, and their log p
 *   logp (with tokens, int32 [N]) and entropy: float [N] or NULL;  top_ids int32, top_logp float: [N][K], 0 <= K <= CX_MAX_TOP, K <= V
 * A logit of -inf has probability 0 and adds nothing to the entropy.  A row of -inf alone: logp and top_logp -inf, entropy 0.  A row
 * with a NaN or +inf: NaN for logp, entropy and top_logp; a NaN is no alternative (places left over: id -1).
 */
int cx_scores_workspace(int64_t N, int32_t V, int32_t K, int64_t *bytes);
int cx_token_scores(const float *z, int64_t ld, int64_t N, int32_t V, const int32_t *tokens, float scale, float *logp,
                    float *entropy, int32_t K, int32_t *top_ids, float *top_logp, void *workspace, int64_t workspace_bytes,
                    void *stream);
int cx_token_scores_bf16(const uint16_t *z, int64_t ld, int64_t N, int32_t V, const int32_t *tokens, float scale, float *logp,
                         float *entropy, int32_t K, int32_t *top_ids, float *top_logp, void *workspace, int64_t workspace_bytes,
                         void *stream);
int cx_token_scores_f16(const uint16_t *z, int64_t ld, int64_t N, int32_t V, const int32_t *tokens, float scale, float *logp,
                        float *entropy, int32_t K, int32_t *top_ids, float *top_logp, void *workspace, int64_t workspace_bytes,
                        void *stream);

/* ------------------------------------------------------------------------------------
 * cx_distill_loss / _grad / _step -- distillation of N rows of V student logits z from a teacher's K top logits:
 *     q = softmax(t / tau) over the row's valid ids ;  p = softmax(z / tau) ;  p1 = softmax(z)
 *     loss = w_kl tau^2 sum_k q_k (log q_k - log p[id_k])  -  w_ce log p1[label]
 *     dz   = round(gout (w_kl tau (p - q) + w_ce (p1 - onehot(label))))
 *   ids      int32 [N][K], t float [N][K] (logits or log probabilities: a constant per row changes nothing); an id outside [0, V)
 *            or a t of -inf counts for nothing, a row without valid ids has no first term.  0 <= K <= CX_MAX_TEACHER.
 *            An id that occurs twice counts twice.
 *   labels   int32 [N] or NULL; outside [0, V): no second term
 *   gout     float [N]: the gradient of what is trained on with respect to each row's loss
 *   stats    float [N][4]: written by _loss (may be NULL there), read by _grad with the same tau, w_kl and w_ce
 *   loss     float [N];  dz [N][ld_dz], may be z (with the same ld)
 * _loss computes the loss, _grad the gradient from the statistics that _loss left, _step both in one call.
 * tau > 0, w_kl >= 0, w_ce >= 0; they, log2(e) / tau and w_kl tau are finite.  A row that no term counts in has loss 0 and gradient 0,
 * whatever its logits; so has a row of -inf alone.  NaN and +inf in a row that counts make its loss and gradient NaN.  A probability
 * below 2^-126 is 0 in the gradient.
 */
int cx_distill_workspace(int64_t N, int32_t V, int64_t *bytes);
int cx_distill_loss(const float *z, int64_t ld, int64_t N, int32_t V, int32_t K, const int32_t *ids, const float *t,
                    const int32_t *labels, float tau, float w_kl, float w_ce, float *loss, float *stats, void *workspace,
                    int64_t workspace_bytes, void *stream);
int cx_distill_loss_bf16(const uint16_t *z, int64_t ld, int64_t N, int32_t V, int32_t K, const int32_t *ids, const float *t,
                         const int32_t *labels, float tau, float w_kl, float w_ce, float *loss, float *stats, void *workspace,
                         int64_t workspace_bytes, void *stream);
int cx_distill_loss_f16(const uint16_t *z, int64_t ld, int64_t N, int32_t V, int32_t K, const int32_t *ids, const float *t,
                        const int32_t *labels, float tau, float w_kl, float w_ce, float *loss, float *stats, void *workspace,
                        int64_t workspace_bytes, void *stream);
int cx_distill_grad(const float *z, int64_t ld, int64_t N, int32_t V, int32_t K, const int32_t *ids, const float *t,
                    const int32_t *labels, float tau, float w_kl, float w_ce, const float *stats, const float *gout, float *dz,
                    int64_t ld_dz, void *stream);
int cx_distill_grad_bf16(const uint16_t *z, int64_t ld, int64_t N, int32_t V, int32_t K, const int32_t *ids, const float *t,
                         const int32_t *labels, float tau, float w_kl, float w_ce, const float *stats, const float *gout,
                         uint16_t *dz, int64_t ld_dz, void *stream);
int cx_distill_grad_f16(const uint16_t *z, int64_t ld, int64_t N, int32_t V, int32_t K, const int32_t *ids, const float *t,
                        const int32_t *labels, float tau, float w_kl, float w_ce, const float *stats, const float *gout,
                        uint16_t *dz, int64_t ld_dz, void *stream);
int cx_distill_step(const float *z, int64_t ld, int64_t N, int32_t V, int32_t K, const int32_t *ids, const float *t,
                    const int32_t *labels, float tau, float w_kl, float w_ce, const float *gout, float *loss, float *dz,
                    int64_t ld_dz, void *workspace, int64_t workspace_bytes, void *stream);
int cx_distill_step_bf16(const uint16_t *z, int64_t ld, int64_t N, int32_t V, int32_t K, const int32_t *ids, const float *t,
                         const int32_t *labels, float tau, float w_kl, float w_ce, const float *gout, float *loss,
                         uint16_t *dz, int64_t ld_dz, void *workspace, int64_t workspace_bytes, void *stream);
int cx_distill_step_f16(const uint16_t *z, int64_t ld, int64_t N, int32_t V, int32_t K, const int32_t *ids, const float *t,
                        const int32_t *labels, float tau, float w_kl, float w_ce, const float *gout, float *loss,
                        uint16_t *dz, int64_t ld_dz, void *workspace, int64_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif

#endif /* CX_LM_H */
