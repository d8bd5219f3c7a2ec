/*
 * cx_lm.h -- C ABI of the language-model operators of the MI355X (gfx950) library: what a simulated worker's training step
 * computes before and after its matrix products, so that its gradient row is ready for the optimizer steps of cx_mix.h.
 *
 *   cx_embed_lookup, cx_embed_grad      embedding tables inside the workers' flat rows, and gradients into them
 *   cx_gated_scan, cx_gated_scan_grad   a gated linear recurrence over long sequences; its single-token step
 *   cx_token_scores                     log probabilities of given tokens, entropy, the largest logits
 *   cx_distill_loss / _grad / _step     distillation from a teacher's top logits, with the label's cross entropy
 *   cx_dropout                          dropout whose mask a counter-based generator names and nothing stores
 *   cx_add_norm, cx_add_norm_grad       residual addition (with dropout) and root-mean-square norm; output in 8 bits with scales
 *   cx_short_conv, cx_short_conv_grad   short causal convolution of every column; its single-token step
 *   cx_select_scan, cx_select_scan_grad selective state space scan over long sequences; its single-token step
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
#define CX_SCAN_CHUNK 16            /* steps between two states that cx_gated_scan and cx_select_scan keep for their gradients */
#define CX_MAX_NORM_WIDTH 16384     /* columns of cx_add_norm */
#define CX_MAX_TAPS 4               /* inputs that a step of cx_short_conv sees */
#define CX_MAX_STATES 16            /* states of a column of cx_select_scan */

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

/* ------------------------------------------------------------------------------------
 * cx_dropout -- dropout, added to a residual where there is one:
 *     out = round(residual + keep x s)     s = 2^16 / (2^16 - k),  k = round(p 2^16) <= 65535, 0 <= p < 1
 * keep of row n and column d: at least k is the 16-bit half (d mod 8) of block (n ceil(D / 8) + floor(d / 8), rng[1]) of Philox4x32 with ten
 * rounds (Salmon et al. 2011) and key rng[0]: halves of the four words in turn, the lower one first; of each 64-bit number the lower word first.
 *   x, out   [N][D], N <= 2^31, N ceil(D / 8) < 2^33; residual: the same or NULL.  out may be x or residual
 *   rng      int64 [2] DEVICE: key and draw; another draw is another mask.  Read when the kernel runs, so that a captured call whose
 *            caller adds to rng[1] between replays draws anew
 * The gradient is the same call on the result's gradient, with the same rng.  A dropped element counts for nothing, NaN and infinities included.
 */
int cx_dropout(const float *x, int64_t ldx, const float *residual, int64_t ldr, float *out, int64_t ldo, int64_t N, int32_t D,
               const int64_t *rng, float p, void *stream);
int cx_dropout_bf16(const uint16_t *x, int64_t ldx, const uint16_t *residual, int64_t ldr, uint16_t *out, int64_t ldo, int64_t N,
                    int32_t D, const int64_t *rng, float p, void *stream);
int cx_dropout_f16(const uint16_t *x, int64_t ldx, const uint16_t *residual, int64_t ldr, uint16_t *out, int64_t ldo, int64_t N, int32_t D,
                   const int64_t *rng, float p, void *stream);

/* ------------------------------------------------------------------------------------
 * cx_add_norm -- residual addition and root-mean-square norm of N rows of each of W workers:
 *     t = residual + drop(x) ;  s = round(t) ;  inv = 1 / sqrt(mean(t^2) + eps) ;  y = round(t inv w)
 *     scale = max(max |t inv w| / 448, 2^-126) ;  q = t inv w / scale in float32, rounded to e4m3 (4 exponent, 3 mantissa bits, largest 448)
 * drop as cx_dropout with p, rng and the row's number in 0 .. W N - 1 (p = 0: nothing is dropped, rng may be NULL); t is not rounded between.
 * w is [D] in columns [offset, offset + D) of the worker's flat row weights[w].
 *   x        [W * N][D], D <= CX_MAX_NORM_WIDTH; residual: the same or NULL (zeros)
 *   s, y     the same or NULL; s may be x or residual, y may be x;  inv: float [W * N] or NULL, which the gradient needs
 *   q, scale bytes [W * N][ldq], D columns, with float [W * N]; or both NULL.  One of s, y and q at least is wanted
 * 0 <= eps < infinity.  Squares whose sum leaves float32's range make inv and the row's y 0; an infinity's own y is NaN.  A NaN in a row makes
 * all of its y NaN, and so does eps = 0 in a row of zeros.  A NaN among a row's y makes its scale and its q NaN; an infinite y
 * without one an infinite scale, q NaN in its place and 0 elsewhere.
 */
int cx_add_norm(const float *x, int64_t ldx, const float *residual, int64_t ldr, const float *weights, int64_t ldw, int32_t W,
                int64_t offset, int64_t N, int32_t D, float eps, const int64_t *rng, float p, float *s, int64_t lds, float *y, int64_t ldy,
                float *inv, uint8_t *q, int64_t ldq, float *scale, void *stream);
int cx_add_norm_bf16(const uint16_t *x, int64_t ldx, const uint16_t *residual, int64_t ldr, const uint16_t *weights, int64_t ldw,
                     int32_t W, int64_t offset, int64_t N, int32_t D, float eps, const int64_t *rng, float p, uint16_t *s, int64_t lds,
                     uint16_t *y, int64_t ldy, float *inv, uint8_t *q, int64_t ldq, float *scale, void *stream);
int cx_add_norm_f16(const uint16_t *x, int64_t ldx, const uint16_t *residual, int64_t ldr, const uint16_t *weights, int64_t ldw, int32_t W,
                    int64_t offset, int64_t N, int32_t D, float eps, const int64_t *rng, float p, uint16_t *s, int64_t lds, uint16_t *y,
                    int64_t ldy, float *inv, uint8_t *q, int64_t ldq, float *scale, void *stream);

/* ------------------------------------------------------------------------------------
 * cx_add_norm_grad -- its gradient.  With g = dy w and the s and inv that the forward call left:
 *     ds = round(inv (g - s inv mean(g s inv)) + ds_in) ;  dx = round(drop of the same before its rounding)
 *     dw = round(g_in + sum over the worker's rows of dy s inv), into columns [offset, offset + D) of its flat gradient row g_out[w]
 * s is t rounded to the rows' type, so that with 16 bits each term of dw carries that rounding beside the sum's own: half a step, 2^-8 of it at
 * most in bfloat16 and 2^-11 in binary16.  No matrix of wider rows is kept for it.
 *   ds_in    gradient of s from elsewhere (the residual path behind the norm), or NULL
 *   ds       gradient of residual; dx: gradient of x; one of them may be NULL.  Each may be dy or ds_in
 *   g_in     NULL (nothing is added), g_out (added in place) or a second matrix with the same ld
 * Sums are fp32 in an order that the sizes fix.
 */
int cx_norm_workspace(int32_t W, int64_t N, int32_t D, int64_t *bytes);
int cx_add_norm_grad(const float *dy, int64_t lddy, const float *s, int64_t lds, const float *inv, const float *weights, int64_t ldw,
                     int32_t W, int64_t offset, int64_t N, int32_t D, const float *ds_in, int64_t ldi, const int64_t *rng, float p,
                     float *ds, int64_t ldds, float *dx, int64_t lddx, const float *g_in, float *g_out, int64_t ldg, void *workspace,
                     int64_t workspace_bytes, void *stream);
int cx_add_norm_grad_bf16(const uint16_t *dy, int64_t lddy, const uint16_t *s, int64_t lds, const float *inv, const uint16_t *weights,
                          int64_t ldw, int32_t W, int64_t offset, int64_t N, int32_t D, const uint16_t *ds_in, int64_t ldi,
                          const int64_t *rng, float p, uint16_t *ds, int64_t ldds, uint16_t *dx, int64_t lddx, const uint16_t *g_in,
                          uint16_t *g_out, int64_t ldg, void *workspace, int64_t workspace_bytes, void *stream);
int cx_add_norm_grad_f16(const uint16_t *dy, int64_t lddy, const uint16_t *s, int64_t lds, const float *inv, const uint16_t *weights,
                         int64_t ldw, int32_t W, int64_t offset, int64_t N, int32_t D, const uint16_t *ds_in, int64_t ldi,
                         const int64_t *rng, float p, uint16_t *ds, int64_t ldds, uint16_t *dx, int64_t lddx, const uint16_t *g_in,
                         uint16_t *g_out, int64_t ldg, void *workspace, int64_t workspace_bytes, void *stream);

/* ------------------------------------------------------------------------------------
 * cx_short_conv -- causal convolution of every column with K taps of its own, B sequences of T steps and D columns:
 *     v_t = bias + sum_{k < K} w[k] x_{t - K + 1 + k} ;  y_t = round(silu != 0 ? v_t sigmoid(v_t) : v_t)
 * 1 <= K <= CX_MAX_TAPS.  W workers have B / W sequences each (B a multiple of W); a worker's taps [D][K] and, behind them, biases [D] are in
 * columns [offset, offset + D (K + 1)) of its flat row.
 *   reset    uint8 [B][T] or NULL: nonzero where a document begins; its steps see nothing of the steps before
 *   before   [B][K - 1][D] or NULL (zeros): the inputs before the first step, the oldest first
 *   after    [B][K - 1][D] or NULL: receives what the step after the last one sees of these inputs, zeros where a reset lies between;
 *            may be before (generation: T = 1, state in place)
 */
int cx_short_conv(const float *x, int64_t ldx, const float *weights, int64_t ldw, int32_t W, int64_t offset, float *y, int64_t ldy,
                  int64_t B, int64_t T, int32_t D, int32_t K, int32_t silu, const uint8_t *reset, const float *before, float *after,
                  void *stream);
int cx_short_conv_bf16(const uint16_t *x, int64_t ldx, const uint16_t *weights, int64_t ldw, int32_t W, int64_t offset, uint16_t *y,
                       int64_t ldy, int64_t B, int64_t T, int32_t D, int32_t K, int32_t silu, const uint8_t *reset, const uint16_t *before,
                       uint16_t *after, void *stream);
int cx_short_conv_f16(const uint16_t *x, int64_t ldx, const uint16_t *weights, int64_t ldw, int32_t W, int64_t offset, uint16_t *y,
                      int64_t ldy, int64_t B, int64_t T, int32_t D, int32_t K, int32_t silu, const uint8_t *reset, const uint16_t *before,
                      uint16_t *after, void *stream);

/* ------------------------------------------------------------------------------------
 * cx_short_conv_grad -- its gradient over x, and over taps and biases into the same columns of the workers' flat gradient rows (g_in as
 * in cx_add_norm_grad).  v is computed again; `before` is a constant.  dx is [B * T][lddx].
 */
int cx_conv_workspace(int32_t W, int64_t B, int64_t T, int32_t D, int32_t K, int64_t *bytes);
int cx_short_conv_grad(const float *x, int64_t ldx, const float *dy, int64_t lddy, const float *weights, int64_t ldw, int32_t W,
                       int64_t offset, float *dx, int64_t lddx, const float *g_in, float *g_out, int64_t ldg, int64_t B, int64_t T,
                       int32_t D, int32_t K, int32_t silu, const uint8_t *reset, const float *before, void *workspace,
                       int64_t workspace_bytes, void *stream);
int cx_short_conv_grad_bf16(const uint16_t *x, int64_t ldx, const uint16_t *dy, int64_t lddy, const uint16_t *weights, int64_t ldw,
                            int32_t W, int64_t offset, uint16_t *dx, int64_t lddx, const uint16_t *g_in, uint16_t *g_out, int64_t ldg,
                            int64_t B, int64_t T, int32_t D, int32_t K, int32_t silu, const uint8_t *reset, const uint16_t *before,
                            void *workspace, int64_t workspace_bytes, void *stream);
int cx_short_conv_grad_f16(const uint16_t *x, int64_t ldx, const uint16_t *dy, int64_t lddy, const uint16_t *weights, int64_t ldw,
                           int32_t W, int64_t offset, uint16_t *dx, int64_t lddx, const uint16_t *g_in, uint16_t *g_out, int64_t ldg,
                           int64_t B, int64_t T, int32_t D, int32_t K, int32_t silu, const uint8_t *reset, const uint16_t *before,
                           void *workspace, int64_t workspace_bytes, void *stream);

/* ------------------------------------------------------------------------------------
 * cx_select_scan -- selective state space scan of B sequences of T steps, D columns and N states a column:
 *     delta_t = softplus(dt_t + bias) ;  a_t[n] = exp(-delta_t exp(A_log[n]))
 *     h_t[n] = a_t[n] (reset_t ? 0 : h_{t-1}[n]) + delta_t B_t[n] u_t
 *     y_t = round((sum_n C_t[n] h_t[n] + skip u_t) (z ? z_t sigmoid(z_t) : 1))
 * u, dt, z, y are matrices of B * T rows and D columns, bm (B) and cm (C) of N columns, each with its own ld <= 2^24; 1 <= N <= CX_MAX_STATES,
 * B D <= 2^29.
 * W workers have B / W sequences each (B a multiple of W); A_log [D][N], bias [D] and skip [D] lie one behind the other in columns
 * [offset, offset + D (N + 2)) of the worker's flat row.
 *   z        NULL: no gate
 *   reset    uint8 [B][T] or NULL: nonzero where a document begins; nothing of the state before it is used, NaN and infinities included
 *   h0       float [B][D][N] or NULL (zeros);  h_last: the same or NULL, may be h0 (generation: T = 1, state in place)
 *   states   float [B][ceil(T / CX_SCAN_CHUNK)][D][N] or NULL: the state that enters every CX_SCAN_CHUNK-th step, which the gradient needs
 * A dt of -inf (padding) leaves the state as it is, whatever u holds; in a row of nothing else whatever B and C hold too.  Long sequences are
 * computed as compositions of maps, so an infinite state may turn into a NaN.  A single step needs no workspace.
 */
int cx_select_workspace(int64_t B, int64_t T, int32_t D, int32_t N, int64_t *bytes);
int cx_select_scan(const float *u, int64_t ldu, const float *dt, int64_t lddt, const float *bm, int64_t ldb, const float *cm, int64_t ldc,
                   const float *z, int64_t ldz, const float *params, int64_t ldp, int32_t W, int64_t offset, float *y, int64_t ldy,
                   int64_t B, int64_t T, int32_t D, int32_t N, const uint8_t *reset, const float *h0, float *h_last, float *states,
                   void *workspace, int64_t workspace_bytes, void *stream);
int cx_select_scan_bf16(const uint16_t *u, int64_t ldu, const uint16_t *dt, int64_t lddt, const uint16_t *bm, int64_t ldb,
                        const uint16_t *cm, int64_t ldc, const uint16_t *z, int64_t ldz, const uint16_t *params, int64_t ldp, int32_t W,
                        int64_t offset, uint16_t *y, int64_t ldy, int64_t B, int64_t T, int32_t D, int32_t N, const uint8_t *reset,
                        const float *h0, float *h_last, float *states, void *workspace, int64_t workspace_bytes, void *stream);
int cx_select_scan_f16(const uint16_t *u, int64_t ldu, const uint16_t *dt, int64_t lddt, const uint16_t *bm, int64_t ldb,
                       const uint16_t *cm, int64_t ldc, const uint16_t *z, int64_t ldz, const uint16_t *params, int64_t ldp, int32_t W,
                       int64_t offset, uint16_t *y, int64_t ldy, int64_t B, int64_t T, int32_t D, int32_t N, const uint8_t *reset,
                       const float *h0, float *h_last, float *states, void *workspace, int64_t workspace_bytes, void *stream);

/* ------------------------------------------------------------------------------------
 * cx_select_scan_grad -- its gradient over u, dt, B, C, z and, into the same columns of the workers' flat gradient rows (g_in as in
 * cx_add_norm_grad), over A_log, bias and skip.  States between those kept are computed again in fp32; y is not read.
 *   states   as the forward call left them for the same inputs
 *   z, dz    both or neither
 *   dh_last  float [B][D][N] or NULL (zeros);  dh0: float [B][D][N] or NULL (not wanted); may be dh_last
 * A row whose dt are all -inf and whose dy are 0 (padding) has gradients of 0 and adds nothing to others, whatever u, B, C and z hold there.
 * Gradients of what columns and sequences share (B, C and the parameters) are sums in fp32, in an order that the sizes fix.
 */
int cx_select_grad_workspace(int64_t B, int64_t T, int32_t D, int32_t N, int64_t *bytes);
int cx_select_scan_grad(const float *u, int64_t ldu, const float *dt, int64_t lddt, const float *bm, int64_t ldb, const float *cm,
                        int64_t ldc, const float *z, int64_t ldz, const float *params, int64_t ldp, int32_t W, int64_t offset,
                        const float *dy, int64_t lddy, float *du, int64_t lddu, float *ddt, int64_t ldddt, float *dbm, int64_t lddb,
                        float *dcm, int64_t lddc, float *dz, int64_t lddz, const float *g_in, float *g_out, int64_t ldg, int64_t B,
                        int64_t T, int32_t D, int32_t N, const uint8_t *reset, const float *states, const float *dh_last, float *dh0,
                        void *workspace, int64_t workspace_bytes, void *stream);
int cx_select_scan_grad_bf16(const uint16_t *u, int64_t ldu, const uint16_t *dt, int64_t lddt, const uint16_t *bm, int64_t ldb,
                             const uint16_t *cm, int64_t ldc, const uint16_t *z, int64_t ldz, const uint16_t *params, int64_t ldp,
                             int32_t W, int64_t offset, const uint16_t *dy, int64_t lddy, uint16_t *du, int64_t lddu, uint16_t *ddt,
                             int64_t ldddt, uint16_t *dbm, int64_t lddb, uint16_t *dcm, int64_t lddc, uint16_t *dz, int64_t lddz,
                             const uint16_t *g_in, uint16_t *g_out, int64_t ldg, int64_t B, int64_t T, int32_t D, int32_t N,
                             const uint8_t *reset, const float *states, const float *dh_last, float *dh0, void *workspace,
                             int64_t workspace_bytes, void *stream);
int cx_select_scan_grad_f16(const uint16_t *u, int64_t ldu, const uint16_t *dt, int64_t lddt, const uint16_t *bm, int64_t ldb,
                            const uint16_t *cm, int64_t ldc, const uint16_t *z, int64_t ldz, const uint16_t *params, int64_t ldp,
                            int32_t W, int64_t offset, const uint16_t *dy, int64_t lddy, uint16_t *du, int64_t lddu, uint16_t *ddt,
                            int64_t ldddt, uint16_t *dbm, int64_t lddb, uint16_t *dcm, int64_t lddc, uint16_t *dz, int64_t lddz,
                            const uint16_t *g_in, uint16_t *g_out, int64_t ldg, int64_t B, int64_t T, int32_t D, int32_t N,
                            const uint8_t *reset, const float *states, const float *dh_last, float *dh0, void *workspace,
                            int64_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif

#endif /* CX_LM_H */
