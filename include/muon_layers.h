/*
 * muon_layers.h -- C ABI of the MI355X (gfx950) layer operators that hold the
 * matrices the Muon step updates: a matrix product with a fused epilogue, the
 * same grouped by expert, and layer norm, each with its backward pass.  The
 * weight gradients come in the layout muon_step reads.
 *
 *   linear   z = x W + b,  y = act(z) + r      x rows x inner, W inner x outer
 *            dz = dy act'(z),  dx = dz W^T,  dW = x^T dz,  db = sum of dz's rows
 *   grouped  y_t = x_t W_e for offsets[e] <= t < offsets[e + 1]
 *            dx_t = dy_t W_e^T,  dW_e = sum over e's rows of x_t^T dy_t
 *   norm     mean, rstd = 1 / sqrt(var + eps) per row,
 *            y = (x - mean) rstd w + b;  dx, dw, db
 *
 * and those at a model's ends and on the way to its experts:
 *
 *   embedding              rows of a table by token, and the table's gradient
 *   sort_by_expert, dispatch, combine
 *                          a router's choices sorted, tokens to their experts and back
 *   linear_cross_entropy   softmax cross entropy of x W over a vocabulary
 *
 * Conventions of muon.h hold: every function returns a muon_status and
 * nothing aborts or throws; muon_layers_last_error() has the message of the
 * last failure on this thread; device buffers and the stream are the
 * caller's; a call checks its arguments, enqueues kernels on the stream and
 * returns (it never allocates, copies or waits), so it can be captured in a
 * HIP graph.  The current HIP device must be the buffers' and the stream's.
 *
 *  - A matrix is a pointer and a leading dimension in elements (row i starts
 *    at data + i * ld, ld >= its columns); rows need the alignment of their
 *    element type only; rows of whole, aligned 16-byte chunks are read where
 *    they lie, others copied first (MUON_LAYERS_UNALIGNED).
 *  - w_transposed != 0: W is kept as outer x inner (element (k, n) at
 *    w + n * ldw + k), and so is dW.
 *  - dtype is that of every matrix and of the bias: MUON_F32 or MUON_BF16.
 *    Sums are held in fp32; an output is rounded once.  In the bf16 backward
 *    pass dz is rounded to bf16 before the two products that read it.
 *  - Results do not depend on the run: no sum's order is left to timing.
 *  - NaN and infinities propagate within the rows and columns they belong to.
 *  - No output may overlap an input or another output, except that y may be
 *    the residual's own buffer (same ld).
 *  - rows is at most 2^30 and may be 0 (weight and bias gradients are then 0);
 *    inner, outer and cols are 1 to 2^24.
 *  - Workspaces are 256-byte aligned device memory of at least the bytes the
 *    workspace function names (which may be 0: NULL is then accepted), need
 *    no initialisation, and must not be shared by calls that may overlap.
 */
#ifndef MUON_LAYERS_MI355X_H
#define MUON_LAYERS_MI355X_H

#include "muon.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum muon_activation {
  MUON_ACT_NONE = 0,
  MUON_ACT_RELU = 1,      /* max(z, 0) */
  MUON_ACT_GELU = 2,      /* z Phi(z), Phi the normal distribution function */
  MUON_ACT_GELU_TANH = 3, /* z / 2 (1 + tanh(sqrt(2 / pi) (z + 0.044715 z^3))) */
  MUON_ACT_SILU = 4       /* z / (1 + exp(-z)) */
} muon_activation;

/* Most experts of one grouped call. */
#define MUON_GROUPED_MAX_EXPERTS 256

/* y = act(x W + bias) + residual.  bias (outer elements), residual and
 * preact may be NULL; preact, if given, gets z.  Errors: INVALID_ARG (NULL x,
 * w or y with rows > 0, a dimension or leading dimension out of range, an
 * unknown activation, a pointer not aligned to its element), UNSUPPORTED
 * (dtype; more output tiles than one grid holds), WORKSPACE_TOO_SMALL, DEVICE. */
MUON_API muon_status muon_linear_forward(const void* x, int64_t ldx, const void* w, int64_t ldw, int32_t w_transposed,
                                         const void* bias, const void* residual, int64_t ldr, void* y, int64_t ldy,
                                         void* preact, int64_t ldz, int64_t rows, int64_t inner, int64_t outer,
                                         int32_t dtype, int32_t activation, void* workspace, size_t workspace_bytes,
                                         void* hip_stream);

/* The gradients of muon_linear_forward's inputs for the output gradient dy
 * (the residual's is dy itself).  dx, dw and dbias may be NULL (not wanted);
 * dw is kept like w.  preact is the forward pass's z, read unless the
 * activation is MUON_ACT_NONE (then it may be NULL); w is read only for dx, x
 * only for dw. */
MUON_API muon_status muon_linear_backward(const void* dy, int64_t lddy, const void* x, int64_t ldx, const void* w,
                                          int64_t ldw, int32_t w_transposed, const void* preact, int64_t ldz, void* dx,
                                          int64_t lddx, void* dw, int64_t lddw, void* dbias, int64_t rows,
                                          int64_t inner, int64_t outer, int32_t dtype, int32_t activation,
                                          void* workspace, size_t workspace_bytes, void* hip_stream);

/* Flags of the workspace functions. */
#define MUON_LAYERS_BACKWARD 1   /* the backward pass's workspace, not the forward pass's */
#define MUON_LAYERS_UNALIGNED 2  /* room for copies of operands whose rows are not 16-byte aligned
                                    or not a multiple of 16 bytes long; without it the call still
                                    works, on a kernel that reads them as they lie and is many
                                    times slower on large products */

/* Workspace bytes of muon_linear_forward or muon_linear_backward (with any
 * choice of outputs). */
MUON_API muon_status muon_linear_workspace_bytes(int64_t rows, int64_t inner, int64_t outer, int32_t dtype,
                                                 int32_t activation, int32_t flags, size_t* bytes);

/* y_t = x_t W_e for the rows t of expert e.  w: a host array of `experts`
 * device pointers, all with leading dimension ldw; it is read during the call
 * only.  offsets: device, experts + 1 int32, non-decreasing: expert e owns the
 * rows offsets[e] .. offsets[e + 1] - 1 (none if equal).  Rows no expert owns
 * get 0.  The host never sees the offsets: they may come from the GPU's own
 * routing.  Values out of order or out of [0, rows] are clamped into order and
 * range, so that nothing outside the buffers is touched. */
MUON_API muon_status muon_grouped_linear_forward(const void* x, int64_t ldx, const void* const* w, int64_t ldw,
                                                 int32_t w_transposed, const int32_t* offsets, int32_t experts, void* y,
                                                 int64_t ldy, int64_t rows, int64_t inner, int64_t outer, int32_t dtype,
                                                 void* workspace, size_t workspace_bytes, void* hip_stream);

/* Gradients of the grouped product.  dx may be NULL; dw may be NULL, or a host
 * array of `experts` device pointers of which any may be NULL (that expert's
 * gradient is not wanted).  An expert without rows gets dW_e = 0; rows no
 * expert owns get dx = 0 and add to no gradient. */
MUON_API muon_status muon_grouped_linear_backward(const void* dy, int64_t lddy, const void* x, int64_t ldx,
                                                  const void* const* w, int64_t ldw, int32_t w_transposed,
                                                  const int32_t* offsets, int32_t experts, void* dx, int64_t lddx,
                                                  void* const* dw, int64_t lddw, int64_t rows, int64_t inner,
                                                  int64_t outer, int32_t dtype, void* workspace, size_t workspace_bytes,
                                                  void* hip_stream);

/* Workspace bytes of muon_grouped_linear_forward or _backward. */
MUON_API muon_status muon_grouped_linear_workspace_bytes(int64_t rows, int64_t inner, int64_t outer, int32_t experts,
                                                         int32_t dtype, int32_t flags, size_t* bytes);

/* Layer norm over the columns.  weight and bias (cols elements of
 * weight_dtype, MUON_F32 or dtype) may be NULL (1 and 0).  mean and rstd, rows
 * fp32 each, may be NULL.  eps >= 0, finite. */
MUON_API muon_status muon_layer_norm_forward(const void* x, int64_t ldx, const void* weight, const void* bias, void* y,
                                             int64_t ldy, float* mean, float* rstd, int64_t rows, int64_t cols,
                                             float eps, int32_t dtype, int32_t weight_dtype, void* hip_stream);

/* Its gradients, from the forward pass's mean and rstd.  dx, dweight and dbias
 * (weight_dtype) may be NULL. */
MUON_API muon_status muon_layer_norm_backward(const void* dy, int64_t lddy, const void* x, int64_t ldx,
                                              const void* weight, const float* mean, const float* rstd, void* dx,
                                              int64_t lddx, void* dweight, void* dbias, int64_t rows, int64_t cols,
                                              int32_t dtype, int32_t weight_dtype, void* workspace,
                                              size_t workspace_bytes, void* hip_stream);

/* Workspace bytes of muon_layer_norm_backward. */
MUON_API muon_status muon_layer_norm_workspace_bytes(int64_t rows, int64_t cols, size_t* bytes);

/* ------------------------------------------------- tokens and experts by number
 *
 * Numbers (tokens, targets, experts' indexes) are int32 or int64 (id_bytes 4 or
 * 8) on the GPU; the host never reads them.  One outside its range stands for
 * nobody: no table row, no target, no expert. */

/* y[i] = scale W[ids[i]] for a table W of vocab x cols; 0 for a number outside
 * [0, vocab). */
MUON_API muon_status muon_embedding_forward(const void* ids, int32_t id_bytes, const void* w, int64_t ldw, void* y,
                                            int64_t ldy, int64_t rows, int64_t vocab, int64_t cols, float scale,
                                            int32_t dtype, void* hip_stream);

/* dW[v] = scale times the sum of dy[i] over the i with ids[i] = v, all vocab rows
 * of it (0 where there is none).  The sums are taken in the order of i. */
MUON_API muon_status muon_embedding_backward(const void* dy, int64_t lddy, const void* ids, int32_t id_bytes, void* dw,
                                             int64_t lddw, int64_t rows, int64_t vocab, int64_t cols, float scale,
                                             int32_t dtype, void* workspace, size_t workspace_bytes,
                                             void* hip_stream);

/* Workspace bytes of muon_embedding_backward. */
MUON_API muon_status muon_embedding_workspace_bytes(int64_t rows, int64_t vocab, int64_t cols, size_t* bytes);

/* A router's choices ids[tokens][top] sorted by expert, in their own order within
 * each: offsets (experts + 1) as muon_grouped_linear_* take them; position
 * (tokens x top), each choice's row among the sorted, -1 if it names no expert;
 * source (tokens * top), each row's choice t * top + j; behind the last, ~ (t * top
 * + j) of the choices of no expert.
 * tokens * top is at most 2^30, top and experts at most MUON_GROUPED_MAX_EXPERTS. */
MUON_API muon_status muon_sort_by_expert(const void* ids, int32_t id_bytes, int64_t tokens, int32_t top,
                                         int32_t experts, int32_t* offsets, int32_t* position, int32_t* source,
                                         void* workspace, size_t workspace_bytes, void* hip_stream);

/* Workspace bytes of muon_sort_by_expert. */
MUON_API muon_status muon_sort_by_expert_workspace_bytes(int64_t tokens, int32_t top, size_t* bytes);

/* rows[position[t][j]] = x[t], and 0 in the rows r where source[r] is negative.
 * position and source are those of muon_sort_by_expert, here and below; a value
 * that it would not give stands for no row and no choice (a row that nothing names
 * is left as it is). */
MUON_API muon_status muon_dispatch_forward(const void* x, int64_t ldx, const int32_t* position, const int32_t* source,
                                           void* rows, int64_t ldr, int64_t tokens, int32_t top, int64_t cols,
                                           int32_t dtype, void* hip_stream);

/* dx[t] = the sum of drows[position[t][j]] over j. */
MUON_API muon_status muon_dispatch_backward(const void* drows, int64_t ldr, const int32_t* position, void* dx,
                                            int64_t ldx, int64_t tokens, int32_t top, int64_t cols, int32_t dtype,
                                            void* hip_stream);

/* y[t] = residual[t] + the sum of weights[t][j] rows[position[t][j]] over j.
 * weights: tokens x top of weight_dtype (MUON_F32 or dtype).  residual may be
 * NULL; y may be its buffer (same ld). */
MUON_API muon_status muon_combine_forward(const void* rows, int64_t ldr, const void* weights, int32_t weight_dtype,
                                          const int32_t* position, const void* residual, int64_t ldres, void* y,
                                          int64_t ldy, int64_t tokens, int32_t top, int64_t cols, int32_t dtype,
                                          void* hip_stream);

/* drows[r] = weights[s] dy[s / top] for s = source[r], 0 where it is negative;
 * dweights[s] = <dy[s / top], rows[r]>, 0 for a choice of no expert.  drows and
 * dweights may be NULL; rows is read only for dweights.  The residual's gradient is dy
 * itself. */
MUON_API muon_status muon_combine_backward(const void* dy, int64_t lddy, const void* rows, int64_t ldr,
                                           const void* weights, int32_t weight_dtype, const int32_t* source,
                                           void* drows, int64_t lddr, void* dweights, int64_t tokens, int32_t top,
                                           int64_t cols, int32_t dtype, void* hip_stream);

typedef enum muon_loss_reduction {
  MUON_LOSS_ROWS = 0,  /* a loss for every row */
  MUON_LOSS_SUM = 1,
  MUON_LOSS_MEAN = 2   /* over the rows with a target; 0 if there are none */
} muon_loss_reduction;

/* Softmax cross entropy of z = x W: lse[i] = log of the sum of exp(z[i][v]) over
 * v, loss[i] = lse[i] - z[i][targets[i]].  z exists a piece at a time, in the
 * workspace or not at all.  A row whose target is `ignore` or outside [0, outer)
 * has loss 0.  loss: rows fp32, or one (SUM, MEAN); lse: rows fp32, which the
 * backward pass reads.  inner is at most 2^20. */
MUON_API muon_status muon_linear_cross_entropy_forward(const void* x, int64_t ldx, const void* w, int64_t ldw,
                                                       int32_t w_transposed, const void* targets,
                                                       int32_t target_bytes, int64_t ignore, int32_t reduction,
                                                       float* loss, float* lse, int64_t rows, int64_t inner,
                                                       int64_t outer, int32_t dtype, void* workspace,
                                                       size_t workspace_bytes, void* hip_stream);

/* Its gradients for dloss (rows fp32, or one): z is computed again piece by piece.
 * dz is rounded to dtype before the products that read it.  dx and dw may be NULL;
 * dw is kept like w.  Rows without a target have dx = 0 and add nothing to dw,
 * whatever they hold. */
MUON_API muon_status muon_linear_cross_entropy_backward(const float* dloss, const void* x, int64_t ldx, const void* w,
                                                        int64_t ldw, int32_t w_transposed, const void* targets,
                                                        int32_t target_bytes, int64_t ignore, int32_t reduction,
                                                        const float* lse, void* dx, int64_t lddx, void* dw,
                                                        int64_t lddw, int64_t rows, int64_t inner, int64_t outer,
                                                        int32_t dtype, void* workspace, size_t workspace_bytes,
                                                        void* hip_stream);

/* Workspace bytes of either pass (flags: MUON_LAYERS_BACKWARD,
 * MUON_LAYERS_UNALIGNED -- which these passes need where rows of x or w are not
 * whole, aligned 16-byte chunks, or lie 2^23 bytes or more apart). */
MUON_API muon_status muon_linear_cross_entropy_workspace_bytes(int64_t rows, int64_t inner, int64_t outer,
                                                               int32_t dtype, int32_t flags, size_t* bytes);

/* Thread-local description of the last failure of a function of this header
 * on this thread ("" if none). */
MUON_API const char* muon_layers_last_error(void);

#ifdef __cplusplus
}
#endif

#endif /* MUON_LAYERS_MI355X_H */
