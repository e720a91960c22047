/*
 * simple_vocab.h -- C boundary of the operators at a model's vocabulary, for AMD MI355X (gfx950): what stands before and behind
 * the sampling call of simple_sample.h in a decoding step (final norm, 8-bit head, embedding of the drawn ids), and the loss
 * and gradients of the training step over the same matrices.
 *
 * Conventions, as in simple_sample.h: *_dev is a device pointer that the caller owns; work is enqueued on hip_stream on the
 * current device and not synchronised; nothing is allocated (an operator that needs a workspace says how many bytes by a
 * function of its own, and writes nothing outside them; the workspace may be used for anything else once the stream has
 * passed the call).  Status codes and SIMPLE_F32 / SIMPLE_BF16 are those of simple_sample.h.  Matrices are row-major with a row
 * stride in elements that is at least the row's length; any alignment of an element's own size is taken, 16-byte aligned
 * rows are faster.  T = 0 is a no-op except for gradients of weights, which become zeros (or stay as they are where the call adds
 * to them).  Results do not depend on the order in which workgroups run.
 */
#ifndef SIMPLE_VOCAB_H
#define SIMPLE_VOCAB_H

#include <stdint.h>

#include "simple_sample.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * Root-mean-square norm of T rows of D values (D <= 32768), with an optional addition ahead of it:
 *   h = x + residual (one rounding to dtype; h = x where residual_dev is NULL)
 *   s = 1 / sqrt(mean(h^2) + eps),   out = h * s * weight (float32 arithmetic, one rounding)
 * x, residual, weight, h_out and out have type dtype; sums are float32.  h_out_dev receives h and may be residual_dev or x_dev
 * with the same stride; it may be NULL if residual_dev is.  out_dev may be x_dev with the same stride unless h_out_dev is.
 * rstd_dev (float[T]) receives s, which the gradient wants; may be NULL.
 */
int simple_rms_norm(const void* x_dev, int64_t x_stride, const void* residual_dev, int64_t residual_stride, const void* weight_dev,
                    int64_t T, int64_t D, int dtype, float eps, void* h_out_dev, int64_t h_stride, void* out_dev, int64_t out_stride,
                    float* rstd_dev, void* hip_stream);

/*
 * The same norm with its output in 8 bits: codes_dev[t, j] = rint(u_j * (127 / a)) in [-127, 127] and scales_dev[t] = a * s / 127, with
 * u = h * weight and a = max |u| of the row, so that code * scale is the norm's output.  s cancels out of the codes: they depend on
 * no sum.  A row of zeros (or one with a below 2^-120) has codes and scale 0; a row that holds a NaN or an infinity has codes 0
 * and scale NaN, which a product with it passes on.
 */
int simple_rms_norm_int8(const void* x_dev, int64_t x_stride, const void* residual_dev, int64_t residual_stride, const void* weight_dev,
                         int64_t T, int64_t D, int dtype, float eps, void* h_out_dev, int64_t h_stride, int8_t* codes_dev,
                         int64_t code_stride, float* scales_dev, void* hip_stream);

/* Rows in 8 bits without a norm: u = x, scales_dev[t] = a / 127.  For the weights of simple_linear_int8, once. */
int simple_quantize_rows(const void* x_dev, int64_t x_stride, int64_t T, int64_t D, int dtype, int8_t* codes_dev, int64_t code_stride,
                         float* scales_dev, void* hip_stream);

/*
 * Gradient of simple_rms_norm: with n = h * s, g = dy * weight,
 *   dx = s * (g - n * mean(g * n)) (+ dh),   dweight[j] = sum over t of dy[t, j] * n[t, j]   (float, written, not added to)
 * dx is the gradient of x and of residual alike; dh_dev (may be NULL) is what reaches h past the norm.  rstd_dev is s as the forward call
 * wrote it.  dx_dev may be dy_dev or dh_dev with the same stride.  workspace_dev: simple_rms_norm_grad_workspace(T, D) bytes, 16-byte
 * aligned.
 */
int simple_rms_norm_grad(const void* dy_dev, int64_t dy_stride, const void* h_dev, int64_t h_stride, const void* weight_dev,
                         const float* rstd_dev, const void* dh_dev, int64_t dh_stride, int64_t T, int64_t D, int dtype, void* dx_dev,
                         int64_t dx_stride, float* dweight_dev, void* workspace_dev, int64_t workspace_bytes, void* hip_stream);
int64_t simple_rms_norm_grad_workspace(int64_t T, int64_t D);

/*
 * Embedding lookup: out[t, :] = table[ids[t], :] * scale (float32 arithmetic, one rounding; table and out have type dtype).  A row whose id
 * is outside [0, V) becomes zeros (the sampling calls return id -1 for a row with an error).
 */
int simple_embed(const int32_t* ids_dev, const void* table_dev, int64_t table_stride, int64_t T, int64_t V, int64_t D, int dtype,
                 float scale, void* out_dev, int64_t out_stride, void* hip_stream);

/*
 * Its gradient: dtable[v, :] = scale * (sum of dout[t, :] over the tokens t with ids[t] = v), written whole (rows without a token
 * become zeros), or with accumulate != 0 added to what dtable holds (rows without a token are not touched).  A row's sum is formed
 * in float32 in an order that depends on ids and T alone (a table formed by blocks of columns has the bits of the whole one).  Ids outside [0, V) are
 * ignored.  dout has type dtype, dtable table_dtype.  workspace_dev: simple_embed_grad_workspace(T, V, D) bytes, 16-byte aligned.
 * T < 2^31, V < 2^31 - 1.
 */
int simple_embed_grad(const int32_t* ids_dev, const void* dout_dev, int64_t dout_stride, int64_t T, int64_t V, int64_t D, int dtype,
                      float scale, void* dtable_dev, int64_t dtable_stride, int table_dtype, int accumulate, void* workspace_dev,
                      int64_t workspace_bytes, void* hip_stream);
int64_t simple_embed_grad_workspace(int64_t T, int64_t V, int64_t D);

/*
 * The head in 8 bits: out[t, v] = (sum over k of codes[t, k] * w_codes[v, k]) * scales[t] * w_scales[v] for T tokens, V channels and rows
 * of K codes (K <= 131071, so that the 32-bit sums cannot overflow; they are exact).  Scales are float32, one rounding to out_dtype.
 * The output is a logits matrix as simple_sample reads it.  T <= 2^24, V <= 2^28.  workspace_dev (16-byte aligned,
 * simple_linear_int8_workspace() bytes) serves calls of more than 512 tokens whose codes' rows are not all 16-byte aligned multiples of 16;
 * it may be NULL, which makes those slower.
 */
int simple_linear_int8(const int8_t* codes_dev, int64_t code_stride, const float* scales_dev, const int8_t* w_codes_dev, int64_t w_code_stride,
                       const float* w_scales_dev, int64_t T, int64_t V, int64_t K, void* out_dev, int64_t out_stride, int out_dtype,
                       void* workspace_dev, int64_t workspace_bytes, void* hip_stream);
int64_t simple_linear_int8_workspace(int64_t T, int64_t V, int64_t K);

/*
 * Cross entropy of logits z = logit_scale * hidden * weight^T (hidden [T, D], weight [V, D], both bfloat16; sums float32), of which no [T, V]
 * matrix is kept:
 *   lse[t] = log(sum over v of exp z[t, v]),   loss[t] = lse[t] - z[t, targets[t]]
 * loss is the negative log-probability of the target, 0 where the target is outside [0, V) (a token that is masked).  logit_scale (positive) is
 * 1 / temperature for tokens that were drawn at one.  workspace_dev: simple_xent_workspace(T, V, D) bytes, 16-byte aligned; where the rows of hidden and weight are
 * 16-byte aligned (D and the strides multiples of 8, strides of 2^21 at most) nothing is copied and simple_xent_workspace_aligned(T, V, D) do.  T <= 2^20, V <= 2^28, D <= 65536, and
 * T * V < 2^41.
 */
int simple_xent(const void* hidden_dev, int64_t hidden_stride, const void* weight_dev, int64_t weight_stride, const int32_t* targets_dev,
                int64_t T, int64_t V, int64_t D, float logit_scale, float* loss_dev, float* lse_dev, void* workspace_dev,
                int64_t workspace_bytes, void* hip_stream);
int64_t simple_xent_workspace(int64_t T, int64_t V, int64_t D);
int64_t simple_xent_workspace_aligned(int64_t T, int64_t V, int64_t D);

/*
 * Its gradient for a loss of sum over t of dloss[t] * loss[t]: with G[t, v] = logit_scale * dloss[t] * (exp(z[t, v] - lse[t]) - [v = targets[t]]),
 *   dhidden = G * weight (bfloat16),   dweight = transposed G * hidden (dweight_dtype; accumulate != 0 adds it to what is there)
 * lse_dev is what simple_xent wrote.  Logits are formed again, a piece of the vocabulary at a time, and G is rounded for the products: of up to 64
 * tokens to 16 bits at any size; of more to 11 bits down to 2^-28 of the token's largest element (1 - p at its target), and to steps of 2^-38 of that
 * below, so that a row of weight which is less probable under every token gets a row of zeros.  For dweight the states of more than 64 tokens, times logit_scale, dloss and 1 - p
 * of their token, are rounded likewise, to 11 bits down to 2^-28 of the largest of all tokens (which should be above 2^-60); for dhidden
 * weights are exact down to 2^-28 of the largest.
 * A token whose target is outside [0, V) or whose dloss is 0 takes no part whatever its states hold: its row of dhidden is zeros.
 * Either output may be NULL: then it is not formed.  workspace_dev: simple_xent_grad_workspace() bytes for the outputs wanted, 16-byte aligned
 * (simple_xent_grad_workspace_aligned() where the rows of hidden and weight are, as above).
 */
int simple_xent_grad(const float* dloss_dev, const void* hidden_dev, int64_t hidden_stride, const void* weight_dev, int64_t weight_stride,
                     const int32_t* targets_dev, const float* lse_dev, int64_t T, int64_t V, int64_t D, float logit_scale, void* dhidden_dev,
                     int64_t dhidden_stride, void* dweight_dev, int64_t dweight_stride, int dweight_dtype, int accumulate,
                     void* workspace_dev, int64_t workspace_bytes, void* hip_stream);
int64_t simple_xent_grad_workspace(int64_t T, int64_t V, int64_t D, int want_dhidden, int want_dweight);
int64_t simple_xent_grad_workspace_aligned(int64_t T, int64_t V, int64_t D, int want_dhidden, int want_dweight);

#ifdef __cplusplus
}
#endif
#endif /* SIMPLE_VOCAB_H */
