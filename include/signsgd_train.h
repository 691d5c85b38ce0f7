/*
 * signsgd_train.h -- the operators of a training step that make the gradients which signsgd.h
 * compresses: losses over a language model's logits with their gradient, and activations kept in
 * 8 bits between the forward and the backward pass. Same library, same conventions as signsgd.h:
 * caller-owned DEVICE memory, work enqueued on cuda_stream, int status, every argument checked
 * before anything is enqueued, nothing allocated, nothing kept after the call.
 *
 * Matrices.    Row-major with unit column stride; a row stride is given in elements and is at
 *              least the number of columns (any value for fewer than two rows). Strides need not
 *              be multiples of anything: rows that do not start on a 16-byte boundary take
 *              kernels with narrower loads, with the same results.
 * Sizes.       0 <= rows, cols <= 2^31 - 1 and rows * stride <= SS_MAX_COORDS. A call with no
 *              element to work on enqueues no kernel unless its outputs need a value (sums of
 *              nothing are 0).
 * Arithmetic.  Inputs are widened exactly to fp32; sums, softmax statistics and gradients are
 *              held in fp32 (sums over a sequence in fp64) and rounded once where they are
 *              stored. Sums are taken in a fixed order: the same call gives the same bits.
 * Workspace.   Scratch device memory of the size that the matching *_workspace function gives,
 *              256-byte aligned; it needs no initial content and keeps nothing between calls.
 *              Calls that may overlap on the GPU need one each.
 * Aliasing.    As in signsgd.h, no buffer that a call writes may overlap another buffer of the
 *              call, with one exception: an output may be an input of the same shape in place
 *              (same address, same stride, same type) where a function says so. Columns of one
 *              wider matrix (two halves of each row) do not overlap.
 */
#ifndef SIGNSGD_TRAIN_H_
#define SIGNSGD_TRAIN_H_

#include <stdint.h>

#include "signsgd.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ------------------------------------------------------------------------------------------------
 * Activations kept in 8 bits.
 *
 * Format. The columns of a row are taken in groups of SS_ACT8_GROUP = 32 (the last group of a row
 * may be shorter). With a = max |x| over a group, e is the smallest integer >= -126 with
 * a <= 127 * 2^e, and x is kept as q = x / 2^e rounded to the nearest integer, ties to even; so
 * |q| <= 127 and |q 2^e - x| <= 2^(e-1) <= a / 127. A group whose a is not below 2^126, or that
 * holds an infinity or a NaN, is marked and decodes to NaN throughout: a value that blew up stays
 * visible in the gradient. The decoded value q 2^e has 7 significant bits and is exact in bf16.
 *
 * A checkpoint of [rows, cols] is one buffer of ss_act8_bytes(rows, cols) bytes, 16-byte aligned:
 * first rows * 32 * ceil(cols/32) bytes of values (sign in bit 7, magnitude in bits 0-6; columns
 * beyond cols are 0), then rows * ceil(cols/32) bytes of exponents (e + 127; 255 marks a group).
 */
#define SS_ACT8_GROUP 32

typedef enum {
    SS_ACT_GELU = 0, /* f(x) = x Phi(x), Phi the normal distribution function (no tanh form) */
    SS_ACT_SILU = 1  /* f(x) = x / (1 + exp(-x)) */
} ss_act;

/* Bytes of a checkpoint of [rows, cols]; -1 if a size is out of range. */
int64_t ss_act8_bytes(int64_t rows, int64_t cols);

/* x [rows, cols] of dtype dt -> checkpoint. */
int ss_act8_pack(const void* x, int64_t x_stride, ss_dtype dt, int64_t rows, int64_t cols, uint8_t* ckpt,
                 void* cuda_stream);

/* checkpoint -> out [rows, cols] of dtype dt (exact in both types). */
int ss_act8_unpack(const uint8_t* ckpt, int64_t rows, int64_t cols, void* out, int64_t out_stride, ss_dtype dt,
                   void* cuda_stream);

/*
 * Forward pass of an activation, with what its backward pass needs kept in 8 bits:
 *   y = f(x)        (up == NULL)      or      y = f(x) * up     (gated)
 * computed from the unrounded x and up.
 *   x, up    in   [rows, cols] of dt; up may be NULL
 *   y        out  [rows, cols] of dt; may be x or up in place
 *   ckpt_x   out  checkpoint of x; or NULL: nothing is kept of the inputs (no backward pass follows)
 *   ckpt_up  out  checkpoint of up; required if and only if up and ckpt_x are given
 *   ckpt_y   out  checkpoint of y as stored (after its rounding to dt), the input of the layer
 *                 that follows; or NULL
 */
int ss_act8_forward(const void* x, int64_t x_stride, const void* up, int64_t up_stride, ss_dtype dt, ss_act act,
                    int64_t rows, int64_t cols, void* y, int64_t y_stride, uint8_t* ckpt_x, uint8_t* ckpt_up,
                    uint8_t* ckpt_y, void* cuda_stream);

/*
 * Backward pass of ss_act8_forward from its checkpoints (x^, up^: the decoded values):
 *   dx = dy f'(x^)      or      dx = dy up^ f'(x^),  dup = dy f(x^)
 *   dy   in   [rows, cols] of dt
 *   dx   out  [rows, cols] of dt; may be dy in place
 *   dup  out  [rows, cols] of dt, required if and only if ckpt_up is given; may be dy in place
 */
int ss_act8_backward(const void* dy, int64_t dy_stride, const uint8_t* ckpt_x, const uint8_t* ckpt_up, ss_dtype dt,
                     ss_act act, int64_t rows, int64_t cols, void* dx, int64_t dx_stride, void* dup,
                     int64_t dup_stride, void* cuda_stream);

/*
 * Weight gradient of a linear layer y = x W^T whose input was kept in 8 bits:
 *   dW[n, k] = sum_t dy[t, n] x^[t, k]      (accumulate == 0)      or      dW += the same
 *   dy         in      [rows, n_out] of dt
 *   ckpt_x     in      checkpoint of x [rows, n_in]
 *   dw         out     [n_out, n_in] fp32, unit column stride, row stride dw_stride; in/out with
 *                      accumulate (a parameter's slice of a flat gradient buffer, say)
 *   workspace  scratch workspace_bytes >= ss_weight_grad8_workspace of the same arguments
 * At most 2^30 rows (a third of that for fp32) and 2^24 tiles of 256 x 256; more is SS_ERR_UNSUPPORTED.
 * rows == 0 leaves dW as it is with accumulate and zeroes it without. Too small a workspace is
 * SS_ERR_INVALID_ARG. Sums are added to dW by the memory, which may flush a subnormal sum to zero. A
 * wait inside the kernel that ran out (it is bounded) shows as NaN in the tiles concerned.
 */
int64_t ss_weight_grad8_workspace(const void* dy, int64_t dy_stride, ss_dtype dt, int64_t rows, int64_t n_out,
                                  int64_t n_in);
int ss_weight_grad8(const void* dy, int64_t dy_stride, ss_dtype dt, const uint8_t* ckpt_x, int64_t rows,
                    int64_t n_out, int64_t n_in, float* dw, int64_t dw_stride, int accumulate, void* workspace,
                    int64_t workspace_bytes, void* cuda_stream);

/* ------------------------------------------------------------------------------------------------
 * Losses over logits, with their gradient.
 *
 * Row t holds the logits z_t of one position and targets[t] the token that was taken there:
 *   logp_t = c z_t[targets[t]] - log sum_v exp(c z_t[v]),      c = inv_temperature > 0.
 * weights[t] says how much the position counts (a mask, a mask over a token count, ...). A
 * position whose weight is 0 or whose target is outside [0, vocab) (an ignore index, say) is left out: its
 * logits are not read, its logp is 0 and its row of dlogits is 0 whatever the logits hold.
 * Logits of -inf have probability 0; a row that holds +inf or NaN, or nothing but -inf, gives NaN
 * as the formulas do.
 *   logits       in   [rows, vocab] of dt
 *   targets      in   rows int64
 *   weights      in   rows fp32
 *   logp         out  rows fp32
 *   dlogits      out  [rows, vocab] of dt: the gradient of the loss times *grad_scale; or NULL
 *                     (loss only); may be logits in place
 *   grad_scale   in   one fp32 in device memory (the gradient that arrives at the loss), or NULL
 *                     for 1; it scales dlogits, not the loss
 *   workspace    scratch of ss_loss_workspace(rows, n_pairs) bytes (n_pairs = 0 for the policy loss)
 */
int64_t ss_loss_workspace(int64_t rows, int64_t n_pairs);

/*
 * Clipped policy loss with a KL term. With r_t = exp(logp_t - old_logp_t), u_t = exp(ref_logp_t - logp_t):
 *   pg_t = -min(r_t A_t, clip(r_t, 1 - clip_low, 1 + clip_high) A_t)
 *   kl_t = u_t - log u_t - 1
 *   loss = sum_t weights_t (pg_t + kl_coef kl_t)
 *   d loss / d logp_t = weights_t (-[not clipped] r_t A_t + kl_coef (1 - u_t))
 *   old_logp, advantages  in   rows fp32
 *   ref_logp              in   rows fp32, or NULL (then kl_coef must be 0 and kl_t is 0)
 *   totals                out  3 fp32: loss, sum_t weights_t kl_t, sum_t weights_t [clipped]
 * 0 <= clip_low <= 1, 0 <= clip_high, kl_coef finite; 0 leaves the KL term out of loss and gradient, be it infinite.
 */
int ss_policy_loss(const void* logits, int64_t logits_stride, ss_dtype dt, int64_t rows, int64_t vocab,
                   const int64_t* targets, const float* old_logp, const float* ref_logp, const float* advantages,
                   const float* weights, float inv_temperature, float clip_low, float clip_high, float kl_coef,
                   const float* grad_scale, float* totals, float* logp, void* dlogits, int64_t dlogits_stride,
                   void* workspace, int64_t workspace_bytes, void* cuda_stream);

/*
 * Preference loss over pairs of sequences packed one after another: sequence s covers rows
 * [seq_begin[s], seq_begin[s+1]); 2p is the preferred answer of pair p, 2p + 1 the other. A
 * sequence may be empty; rows before seq_begin[0] and from seq_begin[2 n_pairs] on belong to none.
 *   S_s = sum of weights_t logp_t over the sequence
 *   h_p = (S_2p - ref_2p) - (S_2p+1 - ref_2p+1),   m_p = beta h_p
 *   SS_PREF_SIGMOID  l_p = -(1 - label_smoothing) log sigma(m_p) - label_smoothing log sigma(-m_p)
 *   SS_PREF_HINGE    l_p = max(0, 1 - m_p)
 *   SS_PREF_SQUARED  l_p = (h_p - 1 / (2 beta))^2
 *   loss = scale * sum_p l_p
 *   seq_begin     in   2 n_pairs + 1 int64 in device memory, not decreasing, within [0, rows]
 *                      (values outside are clamped; nothing is read out of range)
 *   ref_seq_logp  in   2 n_pairs fp32: S_s under the reference model
 *   loss          out  1 fp32
 *   margins       out  n_pairs fp32: m_p
 *   seq_logp      out  2 n_pairs fp32: S_s
 * beta > 0, 0 <= label_smoothing <= 1/2 (0 unless SS_PREF_SIGMOID; 0 leaves the second term out, be it infinite).
 */
typedef enum { SS_PREF_SIGMOID = 0, SS_PREF_HINGE = 1, SS_PREF_SQUARED = 2 } ss_pref;

int ss_preference_loss(const void* logits, int64_t logits_stride, ss_dtype dt, int64_t rows, int64_t vocab,
                       const int64_t* targets, const float* weights, const int64_t* seq_begin, int64_t n_pairs,
                       const float* ref_seq_logp, float inv_temperature, ss_pref kind, float beta,
                       float label_smoothing, float scale, const float* grad_scale, float* loss, float* margins,
                       float* seq_logp, float* logp, void* dlogits, int64_t dlogits_stride, void* workspace,
                       int64_t workspace_bytes, void* cuda_stream);

/*
 * Softmax cross entropy at the head of a language model, from the hidden states and the head's weight:
 * the logits z = x w^T are formed in pieces and never kept as a whole. With lse_t = log sum_v exp(c z_t[v]):
 *   logp_t = c z_t[targets[t]] - lse_t
 *   loss = sum_t weights_t (-logp_t + z_coef lse_t^2)
 *   P_t[v] = d loss / d z_t[v] = c weights_t ((1 + 2 z_coef lse_t) exp(c z_t[v] - lse_t) - [v = targets[t]])
 *   dx = P w,  dw = P^T x,  both times *grad_scale
 * Positions are left out as in the losses over logits: their x is not read, their logp and dx are 0. A row of x, or a
 * w, that holds an infinity or a NaN gives what the formulas give, NaN for the most part.
 *   x        in      [rows, width] of dt
 *   w        in      [vocab, width] of dt
 *   totals   out     2 fp32: loss, sum_t weights_t lse_t^2
 *   logp     out     rows fp32
 *   dx       out     [rows, width] of dt, or NULL; may be x in place
 *   dw       out     [vocab, width] of dw_dt, or NULL; fp32, or for bf16 inputs bf16 as well. With accumulate
 *                    (fp32 only) it is added to
 *   workspace        scratch of ss_linear_cross_entropy_workspace of the same arguments. With a gradient 2 bytes a
 *                    logit (bf16) or 10 (fp32) of a piece: all rows, up to a multiple of 64, or as many as take
 *                    1 GiB, but 256 at least. And the rows that count; where w is fp32 or its rows do not start on 16 bytes, a
 *                    copy of it (6 or 2 bytes an element); a bf16 dw to which more than one piece adds has its sums there, 4 bytes
 *                    an element: 8192 x 4096 over 131072 takes 3.4 GB, more than its logits in bf16 (2.1 GB), with an fp32 dw 1.3 GB
 * targets, weights, inv_temperature, grad_scale as above. z_coef finite; 0 leaves its term out.
 * width, vocab >= 1 where there are rows. No rows: totals 0, dw 0 unless accumulate. More than 2^24 rows, 2^30 columns
 * or 2^24 tiles of 256 x 256 are SS_ERR_UNSUPPORTED.
 * bf16: products of bf16 with fp32 sums; exponentials are kept with 11 bits (fewer below 2^-62 of the largest of 128 neighbouring
 * columns), P is rounded to bf16. fp32: products of three bf16 terms, as precise as fp32
 * sums. Sums that are added by the memory may flush a subnormal to zero. A wait inside a kernel that ran out (it is bounded) shows as NaN.
 */
int64_t ss_linear_cross_entropy_workspace(const void* w, int64_t w_stride, ss_dtype dt, int64_t rows, int64_t width,
                                          int64_t vocab, int want_dx, int want_dw, ss_dtype dw_dt);
int ss_linear_cross_entropy(const void* x, int64_t x_stride, const void* w, int64_t w_stride, ss_dtype dt, int64_t rows,
                            int64_t width, int64_t vocab, const int64_t* targets, const float* weights,
                            float inv_temperature, float z_coef, const float* grad_scale, float* totals, float* logp,
                            void* dx, int64_t dx_stride, void* dw, int64_t dw_stride, ss_dtype dw_dt, int accumulate,
                            void* workspace, int64_t workspace_bytes, void* cuda_stream);

#ifdef __cplusplus
}
#endif

#endif /* SIGNSGD_TRAIN_H_ */
