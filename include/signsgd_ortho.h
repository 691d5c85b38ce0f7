/*
 * signsgd_ortho.h -- the orthogonal update: the momentum of a matrix, all singular values drawn
 * towards 1, as the step of its parameter. It stands beside the sign vote of signsgd.h, which takes
 * the sign of each coordinate where this takes the nearest thing to a sign that a matrix has. Same
 * library, same conventions as signsgd.h and signsgd_train.h (matrices, workspace, aliasing).
 *
 *   X_0 = u / |u|                        |u|: the root of the sum of all squares; 0 stays 0
 *   X_k+1 = a X_k + b S X_k + c S S X_k,   S = X_k X_k^T,   (a, b, c) = coefficients of step k
 *   O = X_steps
 *
 * An odd polynomial of the singular values, singular vectors untouched; rows and columns may be exchanged in the formula, and the
 * products are formed over the smaller side. With (3.4445, -4.7750, 2.0315) five times (the default of
 * the Python side) a singular value of X_0 from 0.01 on ends between 0.67 and 1.21.
 *
 * Numerics. |u| from squares that each thread sums in fp32, all threads' sums in fp64 (in fp64 throughout where those leave fp32's range); X in fp32. The products' operands are fp16 (11 significant bits), scaled by a power of
 * two so that their values lie well inside its range, with fp32 sums; the term a X takes X unrounded, so that directions with
 * small singular values are not lost in the rounding of large ones. Of a result O about 2e-3 (2-norm) is rounding with those coefficients; with others
 * a step adds 2^-11 (|b| s^3 + |c| s^5) or so to a direction of singular value s. Coefficients with which the operands could leave their range are refused
 * (SS_ERR_UNSUPPORTED), whatever the matrix: |a| at least (|b| + |c|) / 64; with m_0 = 1 and m_k+1 the largest |a s + b s^3 + c s^5| over 0 <= s <= m_k, m_k
 * at most 32 for each step's X, 1e30 for O, and |b s^2 + c s^4| at most 32768 over the same s. A matrix that
 * holds an infinity or a NaN gives NaN throughout; so does a wait inside a kernel that ran out (each is bounded).
 */
#ifndef SIGNSGD_ORTHO_H_
#define SIGNSGD_ORTHO_H_

#include <stdint.h>

#include "signsgd.h"

#ifdef __cplusplus
extern "C" {
#endif

#define SS_ORTHO_MAX_MATRICES 64
#define SS_ORTHO_MAX_STEPS 32

/* Scratch bytes for `count` matrices of [rows, cols]; -1 if a size is out of range. */
int64_t ss_orthogonal_workspace(int count, int64_t rows, int64_t cols);

/*
 * out_i = O(in_i) for `count` matrices of one shape. Array arguments are host arrays of `count` device pointers.
 *   in    in   [rows, cols] of in_dt, each with row stride in_stride
 *   out   out  [rows, cols] of out_dt, each with row stride out_stride; out_i may be in_i in place
 *   coefficients  in  3 * steps finite fp32 in host memory, in the range above
 * 1 <= steps <= SS_ORTHO_MAX_STEPS, 0 <= count <= SS_ORTHO_MAX_MATRICES.
 * Sides beyond 2^20 or more than 2^24 tiles of 256 x 256 are SS_ERR_UNSUPPORTED.
 */
int ss_orthogonalise(const void* const* in, int64_t in_stride, ss_dtype in_dt, void* const* out, int64_t out_stride,
                     ss_dtype out_dt, int count, int64_t rows, int64_t cols, const float* coefficients, int steps,
                     void* workspace, int64_t workspace_bytes, void* cuda_stream);

/*
 * One step of momentum and parameter around it:
 *   v' = (1 - beta) g + beta v          u = v', or (1 - beta) g + beta v' (nesterov)
 *   p' = p - lr (scale O(u) + weight_decay p)
 *   grads                  in      [rows, cols] of dt
 *   momenta, momenta_out   in/out  [rows, cols] fp32, row stride momentum_stride; momenta_out_i may be momenta_i
 *   params, params_out     in/out  [rows, cols] fp32, row stride param_stride; params_out_i may be params_i
 * 0 <= beta < 1; lr, scale, weight_decay finite.
 */
int ss_orthogonal_update(const void* const* grads, int64_t grad_stride, ss_dtype dt, const float* const* momenta,
                         float* const* momenta_out, int64_t momentum_stride, const float* const* params,
                         float* const* params_out, int64_t param_stride, int count, int64_t rows, int64_t cols,
                         float beta, int nesterov, const float* coefficients, int steps, float lr, float scale,
                         float weight_decay, void* workspace, int64_t workspace_bytes, void* cuda_stream);

#ifdef __cplusplus
}
#endif

#endif /* SIGNSGD_ORTHO_H_ */
