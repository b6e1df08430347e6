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

/* Thread-local description of the last failure of a function of this header
 * on this thread ("" if none). */
MUON_API const char* muon_layers_last_error(void);

#ifdef __cplusplus
}
#endif

#endif /* MUON_LAYERS_MI355X_H */
