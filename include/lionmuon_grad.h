/*
 * lionmuon_grad.h -- operators that produce the gradients the step consumes
 * (MI355X, gfx950; same library as lionmuon.h, same status codes and
 * lionmuon_last_error).
 *
 * The step of lionmuon.h takes fp32 gradients of 2-D matrices and of 1-D
 * vectors. These operators are what a training program runs to get them:
 *
 *  - products grouped by expert and their two gradients. Rows of X are sorted
 *    by expert; expert e owns rows offsets[e] .. offsets[e + 1) and the matrix
 *    W_e (n x k, the layout of a parameter of the step):
 *        Y = X W_e^T,   dX = dY W_e,   dW_e = dY_e^T X_e  (fp32).
 *    One expert is an ordinary layer.
 *  - activation checkpoints in 8 bits: what the forward pass keeps of a tensor
 *    for the backward pass. dW reads X from one, the activation function's
 *    gradient its input, the norm's gradient the residual stream.
 *  - the root-mean-square norm with the residual's addition and an optional
 *    output as a checkpoint, and its gradients.
 *
 * Checkpoint format: rows x cols codes in e4m3 (OCP; NaN, no infinity), and
 * one byte e + 127 for each LM_CHECKPOINT_BLOCK columns of a row. A block's e
 * is the smallest integer >= -100 with max|x| <= 448 * 2^e over its finite
 * values; code = e4m3(x * 2^-e), to nearest, ties to even; NaN and infinities
 * become NaN. A code stands for code * 2^e, which bf16 holds exactly (where e is
 * 120, its largest, codes go to 240 only, so that what they stand for is finite). Each
 * value of magnitude above 2^-6 * 2^e is off by at most 2^-4 of itself, a
 * smaller one by 2^-10 * 2^e. Rows of codes start 16-byte aligned (codes pointer
 * and ld_codes multiples of 16, ld_codes >= cols); the bytes between cols and
 * the next multiple of 16 are written as 0.
 *
 * Conventions shared by these entry points:
 *  - Descriptors (lm_matrix, lm_stack, lm_checkpoint) live in HOST memory, the
 *    pointers that they hold are DEVICE pointers. At most 2^31 - 1 rows, which may
 *    be apart (ld >= cols, in elements, below 2^22); the elements of a row are
 *    contiguous. Addresses need the element's alignment only; products run
 *    fastest where rows start 16-byte aligned.
 *  - Every call is asynchronous on `stream` (0 = the null stream), allocates
 *    nothing, keeps nothing from call to call and may be captured in a
 *    graph. Calls may run at the same time on different streams if their
 *    outputs and workspaces are apart. `stream` and all memory belong to
 *    the current device.
 *  - Validation happens before anything is enqueued: an invalid call returns
 *    an error and modifies nothing.
 *  - Outputs must not overlap inputs or each other (checked), except where said.
 *  - Sums, norms and products accumulate in fp32. Results are the same, to the
 *    bit, on every run with the same arguments.
 *  - NaN and infinities propagate as in the formulas.
 */
#ifndef LIONMUON_GRAD_H
#define LIONMUON_GRAD_H

#include "lionmuon.h"

#ifdef __cplusplus
extern "C" {
#endif

#define LM_CHECKPOINT_BLOCK 128

enum { LM_F32 = 0, LM_BF16 = 1, LM_F16 = 2 };

/* rows x cols elements, row r at data + r * ld elements. */
typedef struct lm_matrix {
  void* data;
  int64_t rows, cols, ld;
  int32_t dtype;           /* LM_F32, LM_BF16 or LM_F16 */
  uint32_t reserved;       /* must be 0 */
} lm_matrix;

/* `count` matrices of one shape, matrix i at data + i * stride elements. */
typedef struct lm_stack {
  void* data;
  int64_t count, rows, cols, ld, stride;
  int32_t dtype;
  uint32_t reserved;       /* must be 0 */
} lm_stack;

/* 8-bit checkpoint of rows x cols values (format above). scales holds
 * ceil(cols / LM_CHECKPOINT_BLOCK) bytes a row, rows ld_scales bytes apart; where
 * ld_scales is a multiple of 4, all rows * ld_scales bytes can be read (the
 * weight gradient then copies scales four at a time, and is faster). */
typedef struct lm_checkpoint {
  void* codes;
  void* scales;
  int64_t rows, cols, ld_codes, ld_scales;
} lm_checkpoint;

/* ---- checkpoints ------------------------------------------------------- */

/* out = checkpoint of x (fp32, bf16 or fp16). */
lm_status lionmuon_checkpoint(const lm_matrix* x, const lm_checkpoint* out, hipStream_t stream);

/* out = the values of c, rounded to out's type (exact in fp32 and bf16). In
 * fp16 values beyond 65504 become infinite and those below 2^-14 lose bits. */
lm_status lionmuon_checkpoint_restore(const lm_checkpoint* c, const lm_matrix* out,
                                      hipStream_t stream);

/* ---- activation functions ---------------------------------------------- */

enum { LM_ACT_GELU = 0,     /* h = x/2 (1 + tanh(sqrt(2/pi) (x + 0.044715 x^3))) */
       LM_ACT_SWIGLU = 1 }; /* a = [g | u], h = g / (1 + exp(-g)) * u            */

/* h = act(a); kept (may be NULL) = checkpoint of a. a and h have one type; a
 * has h's columns (LM_ACT_GELU) or twice as many (LM_ACT_SWIGLU). */
lm_status lionmuon_activation(const lm_matrix* a, int32_t kind, const lm_matrix* h,
                              const lm_checkpoint* kept, hipStream_t stream);

/* da = dh * act'(a), a given as it is or (a == NULL) by its checkpoint; h (may
 * be NULL) = act(a) again from the same values, the input of the next layer's
 * weight gradient, which then need not be kept. dh, da, h (and a) have one type. */
lm_status lionmuon_activation_grad(const lm_matrix* dh, const lm_matrix* a,
                                   const lm_checkpoint* kept, int32_t kind, const lm_matrix* da,
                                   const lm_matrix* h, hipStream_t stream);

/* ---- root-mean-square norm --------------------------------------------- */

#define LM_RMSNORM_MAX_COLS 16384

/*
 * s = x + residual, rounded to the tensors' type (s = x if residual == NULL);
 * rstd = 1 / sqrt(mean(s^2) + eps) of each row; y = s * rstd * weight.
 * Outputs, each may be NULL: y; sum = s (needs residual; may be the residual
 * itself: same data and ld); rstd (fp32, one a row, contiguous); kept =
 * checkpoint of y, rounded from fp32 once. weight: cols fp32 values. All
 * matrices have one type. cols in [1, LM_RMSNORM_MAX_COLS], eps >= 0. The mean is
 * formed in fp32: where a row's sum of squares exceeds its range, rstd is 0.
 */
lm_status lionmuon_rmsnorm(const lm_matrix* x, const lm_matrix* residual, const float* weight,
                           double eps, const lm_matrix* y, const lm_matrix* sum, float* rstd,
                           const lm_checkpoint* kept, hipStream_t stream);

/*
 * Gradients of the norm. s: the normed stream as it is or (s == NULL) by its
 * checkpoint; rstd as lionmuon_rmsnorm wrote it. With xhat = s * rstd,
 *   dx = residual_grad + rstd * (weight*dy - xhat * mean(weight*dy*xhat))
 *   dweight = sum over rows of dy * xhat   (fp32; added to dweight if accumulate)
 * residual_grad (may be NULL): gradient that reaches s past the norm; dx may be
 * the same matrix. dx is the gradient of x and of the residual. dx and dweight
 * may each be NULL. Workspace: lionmuon_rmsnorm_workspace_bytes, 256-byte
 * aligned, not used by a concurrent call; none without dweight.
 */
lm_status lionmuon_rmsnorm_grad(const lm_matrix* dy, const lm_matrix* s,
                                const lm_checkpoint* kept, const float* weight,
                                const float* rstd, const lm_matrix* residual_grad,
                                const lm_matrix* dx, float* dweight, int32_t accumulate,
                                void* workspace, size_t workspace_bytes, hipStream_t stream);
lm_status lionmuon_rmsnorm_workspace_bytes(int64_t rows, int64_t cols, size_t* out_bytes);

/* ---- products grouped by expert ----------------------------------------- */

/*
 * offsets: device int32[count + 1], non-decreasing, in [0, rows of X]: expert e
 * owns rows offsets[e] .. offsets[e + 1) and may own none. Rows outside
 * offsets[0] .. offsets[count) belong to no expert: their inputs are not
 * used and their outputs left as they were. The host never reads offsets; offsets
 * that break the rule give unspecified values inside the outputs, nothing else.
 * X, dY, Y, dX and W: bf16 or fp16, one type. All columns counts >= 1. Fewer than
 * 2^30 rows, at most LM_GROUPED_MAX_EXPERTS experts (each workgroup goes through
 * the offsets, 64 at a time).
 */
#define LM_GROUPED_MAX_EXPERTS 65536

/* Y[r] = X[r] W_e^T for each row r of expert e: x T x k, w count x n x k, y T x n. */
lm_status lionmuon_grouped_product(const lm_matrix* x, const lm_stack* w, const int32_t* offsets,
                                   const lm_matrix* y, hipStream_t stream);

/* dX[r] = dY[r] W_e: dy T x n, w count x n x k, dx T x k. */
lm_status lionmuon_grouped_input_grad(const lm_matrix* dy, const lm_stack* w,
                                      const int32_t* offsets, const lm_matrix* dx,
                                      hipStream_t stream);

/*
 * dW_e = dY_e^T X_e, fp32 (dw: count x n x k), or dW_e += with accumulate; an
 * expert without rows gets 0 (keeps its values with accumulate). x: T x k as it
 * is or (x == NULL) by its checkpoint, then dy must be bf16, which holds a
 * checkpoint's values exactly. Workspace: lionmuon_grouped_workspace_bytes
 * (0: none), 256-byte aligned, not used by a concurrent call.
 */
lm_status lionmuon_grouped_weight_grad(const lm_matrix* dy, const lm_matrix* x,
                                       const lm_checkpoint* kept, const int32_t* offsets,
                                       const lm_stack* dw, int32_t accumulate, void* workspace,
                                       size_t workspace_bytes, hipStream_t stream);
lm_status lionmuon_grouped_workspace_bytes(int64_t rows, int64_t count, int64_t n, int64_t k,
                                           size_t* out_bytes);

#ifdef __cplusplus
}
#endif

#endif /* LIONMUON_GRAD_H */
