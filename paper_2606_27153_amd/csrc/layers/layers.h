// Shared declarations of the layer operators: the description of one matrix
// product (plain, grouped by rows, or grouped along the summed dimension), the
// kernels' launchers, and the host-side choice of kernel.
#ifndef MUON_LAYERS_H
#define MUON_LAYERS_H

#include <hip/hip_runtime.h>

#include <cstddef>
#include <cstdint>

#include "muon_layers.h"

namespace muon {
namespace layers {

// C[m][n] = sum_k A[m][k] B[k][n].  An operand is kept with the summed
// dimension along its rows' memory ("row": A as a[m * lda + k], B as
// b[n * ldb + k]) or across it ("tr": A as a[k * lda + m], B as
// b[k * ldb + n]).  The layers need three of the four combinations:
enum Form {
  FORM_RT = 0,  // A row, B tr:  x W, and dz W^T of a transposed W
  FORM_RR = 1,  // A row, B row: dz W^T, and x W of a transposed W
  FORM_TT = 2   // A tr, B tr:   x^T dz (or dz^T x, when W is transposed)
};

constexpr int kCUs = 256;   // of an MI355X

enum Group {
  GROUP_NONE = 0,
  GROUP_ROWS = 1,  // row ranges of A and C belong to experts; B is the expert's
  GROUP_SUM = 2    // ranges of the summed rows of A and B belong to experts; C is the expert's
};

struct Product {
  const void* a;
  const void* b;          // GROUP_ROWS: unused (Table)
  void* c;                // GROUP_SUM: unused (Table)
  const void* bias;       // N elements or NULL
  const void* res;        // M x N or NULL
  void* z;                // M x N or NULL: the sum with the bias, before the activation
  const int32_t* offsets; // grouped: experts + 1
  float* part;            // split sums: `splits` fp32 partial results of M x N each
  int64_t lda, ldb, ldc, ldr, ldz;
  int32_t M, N, K;        // GROUP_ROWS: M = all rows; GROUP_SUM: K = all rows
  int32_t experts;
  int32_t act;
  int32_t splits;         // ranges the summed dimension is cut into (1: none)
};

// Pointers of the experts' matrices (grouped products), passed by value.
struct Table {
  const void* p[MUON_GROUPED_MAX_EXPERTS];
};

// An operand's copy: rows x cols of leading dimension ld_src to rows of ld_dst
// elements (a multiple of 16 bytes), zeros after the last column.  dst NULL: none.
struct PackOne {
  const void* src;
  void* dst;
  int64_t rows, cols, ld_src, ld_dst;
};
struct PackArgs {
  PackOne a, b;
  int32_t experts;   // > 0: b is copied from every pointer of the table, one after the other
};

struct NormArgs {
  const void* x;
  const void* dy;
  const void* weight;
  const void* bias;
  void* y;
  void* dx;
  float* mean;
  float* rstd;
  float* part;            // backward: per-block partial sums of dweight and dbias
  void* dweight;
  void* dbias;
  int64_t ldx, ldy, lddy, lddx;
  int32_t rows, cols;
  int32_t wf32;           // weight, bias and their gradients are fp32
  float eps;
};

struct ActGradArgs {
  const void* dy;
  const void* z;          // NULL: no activation
  void* dz;               // NULL: only the column sums are wanted
  void* dbias;            // NULL: no column sums
  float* part;            // chunks x N fp32
  int64_t lddy, ldz, lddz;
  int32_t rows, N, act;
};

// Launchers: enqueue and return hipGetLastError's answer.
hipError_t launch_simple(bool bf16, int form, int group, const Product& p, const Table* t, hipStream_t st);

// Matrix-core kernels on tiles of 256 x 256 and 128 x 256 (bf16 only), 128 x 128
// and 64 x 64;
// the operands must suit them (tile_fits in layers_api.cpp).
hipError_t launch_tile256_bf16(int form, int group, const Product& p, const Table* t, hipStream_t st);
hipError_t launch_tile128x256_bf16(int form, int group, const Product& p, const Table* t, hipStream_t st);
hipError_t launch_tile128_bf16(int form, int group, const Product& p, const Table* t, hipStream_t st);
hipError_t launch_tile128_f32(int form, int group, const Product& p, const Table* t, hipStream_t st);
hipError_t launch_tile64_bf16(int form, int group, const Product& p, const Table* t, hipStream_t st);
hipError_t launch_tile64_f32(int form, int group, const Product& p, const Table* t, hipStream_t st);

// Few rows: tiles of 16 mt rows (mt 1, 2 or 4), forms RT and RR, any alignment,
// at least 16 bytes of columns.
hipError_t launch_skinny(bool bf16, int form, int group, int mt, const Product& p, const Table* t, hipStream_t st);
// Adds p.splits partial results and applies the epilogue.
hipError_t launch_reduce(bool bf16, const Product& p, hipStream_t st);

hipError_t launch_pack(bool bf16, const PackArgs& a, const Table& t, hipStream_t st);

hipError_t launch_act_grad(bool bf16, const ActGradArgs& a, hipStream_t st);
int act_grad_chunks(int64_t rows, int64_t N);   // rows of `part`

hipError_t launch_norm_forward(bool bf16, const NormArgs& a, hipStream_t st);
hipError_t launch_norm_backward(bool bf16, const NormArgs& a, hipStream_t st);
int norm_blocks(int64_t rows, int64_t cols);    // blocks that hold partial sums

}  // namespace layers
}  // namespace muon

#endif  // MUON_LAYERS_H
