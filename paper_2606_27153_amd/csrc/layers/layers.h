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
constexpr int64_t kMaxGrid = int64_t(1) << 24;   // blocks of 256 threads that one grid holds

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
  int32_t raw;            // != 0: C is left in `part` as it is summed, also where splits is 1
                          // (not by the simple kernel)
  int32_t add;            // raw: added to what `part` holds
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

// Tokens to their experts and back (routing.hip).
struct RouteArgs {
  const void* x;          // dispatch: tokens x cols
  void* rows;             // tokens * top x cols: dispatch writes them, the others read them
  const void* weights;    // tokens x top, or NULL (1)
  const void* res;        // tokens x cols or NULL
  void* y;                // tokens x cols
  const void* dy;
  void* drows;            // or NULL
  void* dweights;         // or NULL
  const int32_t* position;
  const int32_t* source;
  int64_t ldx, ldr, ldres, ldy, lddy, lddr;
  int32_t tokens, top, cols;
  int32_t wf32;           // weights and their gradients are fp32
};
enum RoutePass { ROUTE_DISPATCH, ROUTE_GATHER, ROUTE_COMBINE_GRAD };

struct EmbeddingArgs {
  const void* ids;
  const void* w;
  void* y;
  const void* dy;
  void* dw;
  const int32_t* keys;    // backward: the tokens sorted, and where each was
  const int32_t* index;
  int32_t* starts;        // vocab + 1: where each token's places begin
  float* part;            // sums of groups of places inside one token's run
  int64_t ldw, ldy, lddy, lddw;
  int32_t rows, cols, vocab, id_bytes;
  float scale;
};

// Softmax cross entropy over the columns of z = x W, of which a piece at a time
// exists (loss.hip).
struct LossArgs {
  const void* targets;
  const float* dloss;     // a number for every row (each), or one
  const float* alpha;     // factor of all gradients, or NULL (1)
  float2* part;           // strips x rows: the largest logit and the sum of exponentials relative to it
  float* logit;           // the target's
  float* loss;            // of every row
  float* lse;
  float* total;           // of all rows
  const float* raw;       // splits x rows x cols: a piece of z, to be added up
  void* dz;               // rows x lddz: the gradient of a piece of z
  int64_t ignore, lddz;
  int32_t rows, vocab, target_bytes, each, mean;
  int32_t first, cols;    // the piece
  int32_t splits, strip, strips;
};
constexpr int kRawStrip = 2048;   // columns of a strip of `raw`
// What the tile kernels make of the loss's products: part and logit, or dz, of a
// piece of z; x^T dz times alpha.
enum LossStep { LOSS_STRIPS, LOSS_GRAD, LOSS_WEIGHT };

// Launchers: enqueue and return hipGetLastError's answer.
size_t expert_sort_bytes(int64_t n);
hipError_t launch_expert_sort(const void* ids, int id_bytes, int64_t n, int experts, int32_t* offsets,
                              int32_t* position, int32_t* source, int32_t* counts, hipStream_t st);
hipError_t launch_route(bool bf16, int pass, const RouteArgs& a, hipStream_t st);

size_t embedding_bytes(int64_t rows, int64_t vocab, int64_t cols);
hipError_t launch_embedding_forward(bool bf16, const EmbeddingArgs& a, hipStream_t st);
hipError_t launch_embedding_backward(bool bf16, EmbeddingArgs a, void* workspace, hipStream_t st);

hipError_t launch_loss_mean(const LossArgs& a, float* alpha, hipStream_t st);   // dloss over the rows with a target
hipError_t launch_loss_strips(const LossArgs& a, hipStream_t st);   // raw -> part and logit
hipError_t launch_loss_finish(const LossArgs& a, hipStream_t st);   // part -> lse and loss
hipError_t launch_loss_total(const LossArgs& a, hipStream_t st);    // loss -> total
hipError_t launch_loss_grad(bool bf16, const LossArgs& a, hipStream_t st);   // raw -> dz
// y (rows of ldy): x, with zeros in rows without a target and behind the columns
hipError_t launch_loss_rows(bool bf16, const LossArgs& a, const void* x, int64_t ldx, void* y, int64_t ldy,
                            int64_t cols, hipStream_t st);
// The weight's gradient (a piece: a.cols columns; x_down: kept as [inner, cols], else
// [cols, inner]) of at most outer_rows rows, from x as it lies and dz (which sizes take
// it: outer_product_wins).
constexpr int outer_rows(bool bf16) { return bf16 ? 16 : 32; }
hipError_t launch_loss_outer(bool bf16, bool x_down, const LossArgs& a, const void* x, int64_t ldx, int64_t inner,
                             void* out, int64_t ldo, hipStream_t st);
// y: alpha times the sum of `splits` partial results of a.rows x cols, 0 in rows without a target
hipError_t launch_loss_sum(bool bf16, const LossArgs& a, const float* part, int splits, void* y, int64_t ldy,
                           int64_t cols, hipStream_t st);

hipError_t launch_simple(bool bf16, int form, int group, const Product& p, const Table* t, hipStream_t st);

// Matrix-core kernels on tiles of 256 x 256 and 128 x 256 (bf16 only), 128 x 128
// and 64 x 64; the operands must suit them (tile_fits in host.h).
hipError_t launch_tile256_bf16(int form, int group, const Product& p, const Table* t, hipStream_t st);
hipError_t launch_tile128x256_bf16(int form, int group, const Product& p, const Table* t, hipStream_t st);
hipError_t launch_tile128_bf16(int form, int group, const Product& p, const Table* t, hipStream_t st);
hipError_t launch_tile128_f32(int form, int group, const Product& p, const Table* t, hipStream_t st);
hipError_t launch_tile64_bf16(int form, int group, const Product& p, const Table* t, hipStream_t st);
hipError_t launch_tile64_f32(int form, int group, const Product& p, const Table* t, hipStream_t st);

hipError_t launch_loss256_bf16(int step, int form, const Product& p, const LossArgs& a, hipStream_t st);
hipError_t launch_loss128x256_bf16(int step, int form, const Product& p, const LossArgs& a, hipStream_t st);
hipError_t launch_loss128_bf16(int step, int form, const Product& p, const LossArgs& a, hipStream_t st);
hipError_t launch_loss64_bf16(int step, int form, const Product& p, const LossArgs& a, hipStream_t st);
hipError_t launch_loss128_f32(int step, int form, const Product& p, const LossArgs& a, hipStream_t st);
hipError_t launch_loss64_f32(int step, int form, const Product& p, const LossArgs& a, hipStream_t st);

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
