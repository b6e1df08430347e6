/*
 * muon_adamw.h -- C ABI of the AdamW step for the parameters that the Muon step
 * leaves out (embedding tables, norms, biases): many tensors in one call, with
 * states in 32 bits or in 8.
 *
 *   m = beta1 m + (1 - beta1) g          v = beta2 v + (1 - beta2) g^2
 *   w = w (1 - lr decay) - lr / (1 - beta1^k) m / (sqrt(v / (1 - beta2^k)) + eps)
 *
 * k is the tensor's step, counted from 1; everything is computed in fp32 (under
 * the root, v counts as 2^-126 at least), the parameter rounded once (to nearest).
 *
 * States in 8 bits.  A code of 8 bits stands for the upper 12 bits of an fp32
 * number (sign, exponent, 3 bits of fraction) relative to a base that 256
 * consecutive elements share: code c > 0 for the number whose bits are
 * (c + base) << 20, code 0 for 0; exp_avg has 7 such bits and a sign in the
 * eighth, 16 powers of two, exp_avg_sq all 8, 32 powers of two -- the square of
 * the same range.  The base follows the block's largest number.  Averages move by
 * less than a code's step (a thousandth where beta2 is 0.999, against an eighth),
 * so they are rounded up or down at random, with the probability that keeps the
 * mean: 16 bits of a hash of seed, step, tensor and element decide.  A number too
 * small for code 1 becomes 0; an exp_avg_sq that is not 0 becomes code 1 at least, so
 * that no element divides by less than it should.  The parameter's step uses the
 * new averages before they are rounded.  A gradient that is not finite makes its
 * block's base that of infinity: the block's other averages are lost with it.
 *
 * Conventions of muon.h hold: every function returns a muon_status and nothing
 * aborts or throws; muon_adamw_last_error() has the message of the last failure on
 * this thread; buffers and the stream are the caller's; a call checks its
 * arguments, enqueues kernels on the stream and returns (it never allocates,
 * copies or waits), so it can be captured in a HIP graph, whose replays then take
 * the captured lr and step.  The current HIP device must be the buffers' and the
 * stream's.  Results do not depend on timing.
 */
#ifndef MUON_ADAMW_MI355X_H
#define MUON_ADAMW_MI355X_H

#include "muon.h"

#ifdef __cplusplus
extern "C" {
#endif

#define MUON_ADAMW_BLOCK 256   /* elements of an 8-bit state that share a base */

typedef struct muon_adamw_tensor {
  void* param;         /* n elements of param_dtype */
  const void* grad;    /* n elements of grad_dtype; NULL: the tensor is skipped */
  void* exp_avg;       /* n fp32, or n codes */
  void* exp_avg_sq;    /* n fp32, or n codes */
  int16_t* bases;      /* 8 bits: the bases of exp_avg and exp_avg_sq, a pair for each block */
  int64_t n;           /* elements, 0 to 2^35 */
  int64_t step;        /* from 1 on */
  int32_t param_dtype; /* MUON_F32 or MUON_BF16 */
  int32_t grad_dtype;
} muon_adamw_tensor;

typedef struct muon_adamw_opts {
  double lr, beta1, beta2, eps, weight_decay;
  int32_t state_bits;  /* 32 or 8 */
  uint32_t seed;       /* 8 bits: of the rounding */
} muon_adamw_opts;

/* Steps count tensors (a host array, read during the call only).  Tensors must
 * not overlap.  Errors: INVALID_ARG (a NULL or misaligned pointer, a size, step or
 * option out of range), UNSUPPORTED (dtype, state_bits), DEVICE. */
MUON_API muon_status muon_adamw_step(const muon_adamw_tensor* tensors, int32_t count, const muon_adamw_opts* opts,
                                     void* hip_stream);

/* The numbers that an 8-bit state's codes stand for, as bf16 (which holds them exactly).  Either
 * output may be NULL. */
MUON_API muon_status muon_adamw_state_values(const void* exp_avg, const void* exp_avg_sq, const int16_t* bases,
                                             int64_t n, void* exp_avg_out, void* exp_avg_sq_out, void* hip_stream);

/* Thread-local description of the last failure of a function of this header
 * on this thread ("" if none). */
MUON_API const char* muon_adamw_last_error(void);

#ifdef __cplusplus
}
#endif

#endif /* MUON_ADAMW_MI355X_H */
