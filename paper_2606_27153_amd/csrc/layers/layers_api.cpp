// C ABI of the layer operators: argument checks, workspace layout, choice of
// kernels and their launch order.
#include <cmath>
#include <cstdarg>
#include <cstdio>

#include "layers.h"

namespace {

using namespace muon::layers;

thread_local char g_error[256];

muon_status fail(muon_status s, const char* fmt, ...) {
  va_list ap;
  va_start(ap, fmt);
  std::vsnprintf(g_error, sizeof(g_error), fmt, ap);
  va_end(ap);
  return s;
}

muon_status done(hipError_t e, const char* what) {
  if (e != hipSuccess) return fail(MUON_ERR_DEVICE, "%s: %s", what, hipGetErrorString(e));
  g_error[0] = 0;
  return MUON_OK;
}

constexpr int64_t kMaxDim = int64_t(1) << 30;
constexpr int64_t kMaxLd = int64_t(1) << 40;

bool known_dtype(int32_t d) { return d == MUON_F32 || d == MUON_BF16; }
size_t size_of(int32_t dtype) { return dtype == MUON_BF16 ? 2 : 4; }
size_t padded(size_t v) { return (v + 255) / 256 * 256; }

muon_status check_sizes(int64_t rows, int64_t inner, int64_t outer, int32_t dtype) {
  if (rows < 0 || rows > kMaxDim) return fail(MUON_ERR_INVALID_ARG, "rows %lld out of [0, 2^30]", (long long)rows);
  if (inner < 1 || inner > kMaxDim)
    return fail(MUON_ERR_INVALID_ARG, "inner %lld out of [1, 2^30]", (long long)inner);
  if (outer < 1 || outer > kMaxDim)
    return fail(MUON_ERR_INVALID_ARG, "outer %lld out of [1, 2^30]", (long long)outer);
  if (!known_dtype(dtype)) return fail(MUON_ERR_UNSUPPORTED, "dtype %d: MUON_F32 or MUON_BF16", dtype);
  return MUON_OK;
}

muon_status check_activation(int32_t a) {
  if (a < MUON_ACT_NONE || a > MUON_ACT_SILU) return fail(MUON_ERR_INVALID_ARG, "unknown activation %d", a);
  return MUON_OK;
}

// A matrix operand: a pointer aligned to its element and a leading dimension of
// at least its columns.
muon_status check_matrix(const char* name, const void* p, int64_t ld, int64_t cols, size_t esize) {
  if (!p) return fail(MUON_ERR_INVALID_ARG, "%s is NULL", name);
  if (reinterpret_cast<uintptr_t>(p) % esize) return fail(MUON_ERR_INVALID_ARG, "%s is not aligned to its element", name);
  if (ld < cols || ld > kMaxLd)
    return fail(MUON_ERR_INVALID_ARG, "%s has leading dimension %lld, needs at least %lld", name, (long long)ld,
                (long long)cols);
  return MUON_OK;
}

muon_status check_vector(const char* name, const void* p, size_t esize) {
  if (reinterpret_cast<uintptr_t>(p) % esize) return fail(MUON_ERR_INVALID_ARG, "%s is not aligned to its element", name);
  return MUON_OK;
}

muon_status check_workspace(const void* ws, size_t have, size_t need) {
  if (!need) return MUON_OK;
  if (!ws) return fail(MUON_ERR_INVALID_ARG, "workspace is NULL, %zu bytes are needed", need);
  if (reinterpret_cast<uintptr_t>(ws) % 256) return fail(MUON_ERR_INVALID_ARG, "workspace must be 256-byte aligned");
  if (have < need) return fail(MUON_ERR_WORKSPACE_TOO_SMALL, "workspace has %zu bytes, %zu are needed", have, need);
  return MUON_OK;
}

#define TRY(call)                              \
  do {                                         \
    const muon_status try_st = (call);         \
    if (try_st != MUON_OK) return try_st;      \
  } while (0)

bool aligned16(const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }

// Whether the tile kernels can fetch the operands: 16-byte chunks that lie on
// 16-byte addresses and do not straddle the end of a row, and 32-bit byte
// offsets within a tile of 256 rows.
bool tile_fits(bool bf16, int form, int group, const Product& p, const Table* t) {
  const int64_t epc = bf16 ? 8 : 4, es = bf16 ? 2 : 4;
  const bool atr = form == FORM_TT, btr = form != FORM_RR;
  if (p.lda % epc || p.ldb % epc) return false;
  if (p.lda * es * 256 >= (int64_t(1) << 31) || p.ldb * es * 256 >= (int64_t(1) << 31)) return false;
  if ((atr ? p.M : p.K) % epc || (btr ? p.N : p.K) % epc) return false;
  if (!aligned16(p.a)) return false;
  if (group == GROUP_ROWS) {
    for (int32_t e = 0; e < p.experts; ++e)
      if (!aligned16(t->p[e])) return false;
    return true;
  }
  return aligned16(p.b);
}

// One matrix product: the kernel that suits it.
hipError_t product(bool bf16, int form, int group, Product p, const Table* t, hipStream_t st) {
  p.splits = 1;
  if (!tile_fits(bf16, form, group, p, t)) return launch_simple(bf16, form, group, p, t, st);
  if (!bf16) return launch_tile128_f32(form, group, p, t, st);
  const int64_t big = ((p.M + 255) / 256) * ((p.N + 255) / 256) * int64_t(group == GROUP_SUM ? p.experts : 1);
  return big >= 256 ? launch_tile256_bf16(form, group, p, t, st) : launch_tile128_bf16(form, group, p, t, st);
}

// Workspace of muon_linear_backward: dz and the partial column sums.
struct BackwardLayout {
  size_t dz = 0, part = 0, total = 0;
};
BackwardLayout backward_layout(int64_t rows, int64_t outer, int32_t dtype, int32_t act) {
  BackwardLayout l;
  if (act != MUON_ACT_NONE) l.part = padded(size_t(rows) * size_t(outer) * size_of(dtype));
  l.total = l.part + padded(size_t(act_grad_chunks(rows, outer)) * size_t(outer) * 4);
  return l;
}

muon_status fill_table(const char* name, const void* const* p, int32_t n, bool may_be_null, size_t esize, Table& t) {
  if (!p) return fail(MUON_ERR_INVALID_ARG, "%s is NULL", name);
  for (int32_t i = 0; i < n; ++i) {
    if (!p[i] && !may_be_null) return fail(MUON_ERR_INVALID_ARG, "%s[%d] is NULL", name, i);
    if (reinterpret_cast<uintptr_t>(p[i]) % esize)
      return fail(MUON_ERR_INVALID_ARG, "%s[%d] is not aligned to its element", name, i);
    t.p[i] = p[i];
  }
  for (int32_t i = n; i < MUON_GROUPED_MAX_EXPERTS; ++i) t.p[i] = nullptr;
  return MUON_OK;
}

muon_status check_experts(int32_t experts, const int32_t* offsets) {
  if (experts < 1 || experts > MUON_GROUPED_MAX_EXPERTS)
    return fail(MUON_ERR_INVALID_ARG, "experts %d out of [1, %d]", experts, MUON_GROUPED_MAX_EXPERTS);
  if (!offsets || reinterpret_cast<uintptr_t>(offsets) % 4)
    return fail(MUON_ERR_INVALID_ARG, "offsets is NULL or not 4-byte aligned");
  return MUON_OK;
}

}  // namespace

extern "C" {

MUON_API const char* muon_layers_last_error(void) { return g_error; }

MUON_API muon_status muon_linear_workspace_bytes(int64_t rows, int64_t inner, int64_t outer, int32_t dtype,
                                                 int32_t activation, int32_t backward, size_t* bytes) {
  if (!bytes) return fail(MUON_ERR_INVALID_ARG, "bytes is NULL");
  TRY(check_sizes(rows, inner, outer, dtype));
  TRY(check_activation(activation));
  *bytes = backward ? backward_layout(rows, outer, dtype, activation).total : 0;
  return done(hipSuccess, "");
}

MUON_API muon_status muon_linear_forward(const void* x, int64_t ldx, const void* w, int64_t ldw, int32_t w_transposed,
                                         const void* bias, const void* residual, int64_t ldr, void* y, int64_t ldy,
                                         void* preact, int64_t ldz, int64_t rows, int64_t inner, int64_t outer,
                                         int32_t dtype, int32_t activation, void* workspace, size_t workspace_bytes,
                                         void* hip_stream) {
  TRY(check_sizes(rows, inner, outer, dtype));
  TRY(check_activation(activation));
  if (rows == 0) return done(hipSuccess, "");
  const size_t es = size_of(dtype);
  TRY(check_matrix("x", x, ldx, inner, es));
  TRY(check_matrix("w", w, ldw, w_transposed ? inner : outer, es));
  TRY(check_matrix("y", y, ldy, outer, es));
  if (residual) TRY(check_matrix("residual", residual, ldr, outer, es));
  if (preact) TRY(check_matrix("preact", preact, ldz, outer, es));
  TRY(check_vector("bias", bias, es));
  size_t need = 0;
  TRY(muon_linear_workspace_bytes(rows, inner, outer, dtype, activation, 0, &need));
  TRY(check_workspace(workspace, workspace_bytes, need));
  Product p{};
  p.a = x; p.lda = ldx;
  p.b = w; p.ldb = ldw;
  p.c = y; p.ldc = ldy;
  p.bias = bias;
  p.res = residual; p.ldr = ldr;
  p.z = preact; p.ldz = ldz;
  p.M = int32_t(rows); p.N = int32_t(outer); p.K = int32_t(inner);
  p.act = activation;
  return done(product(dtype == MUON_BF16, w_transposed ? FORM_RR : FORM_RT, GROUP_NONE, p, nullptr,
                      hipStream_t(hip_stream)),
              "linear forward");
}

MUON_API muon_status muon_linear_backward(const void* dy, int64_t lddy, const void* x, int64_t ldx, const void* w,
                                          int64_t ldw, int32_t w_transposed, const void* preact, int64_t ldz, void* dx,
                                          int64_t lddx, void* dw, int64_t lddw, void* dbias, int64_t rows,
                                          int64_t inner, int64_t outer, int32_t dtype, int32_t activation,
                                          void* workspace, size_t workspace_bytes, void* hip_stream) {
  TRY(check_sizes(rows, inner, outer, dtype));
  TRY(check_activation(activation));
  const size_t es = size_of(dtype);
  const bool bf16 = dtype == MUON_BF16, act = activation != MUON_ACT_NONE;
  if (rows) {
    TRY(check_matrix("dy", dy, lddy, outer, es));
    if (dw) TRY(check_matrix("x", x, ldx, inner, es));
    if (dx) TRY(check_matrix("w", w, ldw, w_transposed ? inner : outer, es));
    if (act) TRY(check_matrix("preact", preact, ldz, outer, es));
    if (dx) TRY(check_matrix("dx", dx, lddx, inner, es));
  }
  if (dw) TRY(check_matrix("dw", dw, lddw, w_transposed ? inner : outer, es));
  TRY(check_vector("dbias", dbias, es));
  const BackwardLayout l = backward_layout(rows, outer, dtype, activation);
  TRY(check_workspace(workspace, workspace_bytes, l.total));
  const hipStream_t st = hipStream_t(hip_stream);
  char* ws = static_cast<char*>(workspace);
  const void* dz = dy;
  int64_t lddz = lddy;
  if ((act && rows) || dbias) {
    ActGradArgs a{};
    a.dy = dy; a.lddy = lddy;
    a.z = act ? preact : nullptr; a.ldz = ldz;
    a.dz = act ? ws + l.dz : nullptr; a.lddz = outer;
    a.dbias = dbias;
    a.part = reinterpret_cast<float*>(ws + l.part);
    a.rows = int32_t(rows); a.N = int32_t(outer); a.act = activation;
    TRY(done(launch_act_grad(bf16, a, st), "activation gradient"));
    if (act) {
      dz = ws + l.dz;
      lddz = outer;
    }
  }
  if (dx && rows) {
    Product p{};
    p.a = dz; p.lda = lddz;
    p.b = w; p.ldb = ldw;
    p.c = dx; p.ldc = lddx;
    p.M = int32_t(rows); p.N = int32_t(inner); p.K = int32_t(outer);
    TRY(done(product(bf16, w_transposed ? FORM_RT : FORM_RR, GROUP_NONE, p, nullptr, st), "linear input gradient"));
  }
  if (dw) {
    Product p{};
    p.c = dw; p.ldc = lddw;
    p.K = int32_t(rows);
    // dW = x^T dz, or dW^T = dz^T x for a transposed weight
    p.a = w_transposed ? dz : x; p.lda = w_transposed ? lddz : ldx;
    p.b = w_transposed ? x : dz; p.ldb = w_transposed ? ldx : lddz;
    p.M = int32_t(w_transposed ? outer : inner); p.N = int32_t(w_transposed ? inner : outer);
    TRY(done(product(bf16, FORM_TT, GROUP_NONE, p, nullptr, st), "linear weight gradient"));
  }
  return done(hipSuccess, "");
}

MUON_API muon_status muon_grouped_linear_workspace_bytes(int64_t rows, int64_t inner, int64_t outer, int32_t experts,
                                                         int32_t dtype, int32_t backward, size_t* bytes) {
  if (!bytes) return fail(MUON_ERR_INVALID_ARG, "bytes is NULL");
  TRY(check_sizes(rows, inner, outer, dtype));
  if (experts < 1 || experts > MUON_GROUPED_MAX_EXPERTS)
    return fail(MUON_ERR_INVALID_ARG, "experts %d out of [1, %d]", experts, MUON_GROUPED_MAX_EXPERTS);
  (void)backward;
  *bytes = 0;
  return done(hipSuccess, "");
}

MUON_API muon_status muon_grouped_linear_forward(const void* x, int64_t ldx, const void* const* w, int64_t ldw,
                                                 int32_t w_transposed, const int32_t* offsets, int32_t experts, void* y,
                                                 int64_t ldy, int64_t rows, int64_t inner, int64_t outer, int32_t dtype,
                                                 void* workspace, size_t workspace_bytes, void* hip_stream) {
  TRY(check_sizes(rows, inner, outer, dtype));
  TRY(check_experts(experts, offsets));
  if (rows == 0) return done(hipSuccess, "");
  const size_t es = size_of(dtype);
  TRY(check_matrix("x", x, ldx, inner, es));
  TRY(check_matrix("y", y, ldy, outer, es));
  Table t;
  TRY(fill_table("w", w, experts, false, es, t));
  TRY(check_matrix("w", w[0], ldw, w_transposed ? inner : outer, es));
  size_t need = 0;
  TRY(muon_grouped_linear_workspace_bytes(rows, inner, outer, experts, dtype, 0, &need));
  TRY(check_workspace(workspace, workspace_bytes, need));
  Product p{};
  p.a = x; p.lda = ldx;
  p.ldb = ldw;
  p.c = y; p.ldc = ldy;
  p.offsets = offsets;
  p.experts = experts;
  p.M = int32_t(rows); p.N = int32_t(outer); p.K = int32_t(inner);
  return done(product(dtype == MUON_BF16, w_transposed ? FORM_RR : FORM_RT, GROUP_ROWS, p, &t,
                      hipStream_t(hip_stream)),
              "grouped linear forward");
}

MUON_API muon_status muon_grouped_linear_backward(const void* dy, int64_t lddy, const void* x, int64_t ldx,
                                                  const void* const* w, int64_t ldw, int32_t w_transposed,
                                                  const int32_t* offsets, int32_t experts, void* dx, int64_t lddx,
                                                  void* const* dw, int64_t lddw, int64_t rows, int64_t inner,
                                                  int64_t outer, int32_t dtype, void* workspace, size_t workspace_bytes,
                                                  void* hip_stream) {
  TRY(check_sizes(rows, inner, outer, dtype));
  TRY(check_experts(experts, offsets));
  const size_t es = size_of(dtype);
  const bool bf16 = dtype == MUON_BF16;
  Table tw, td;
  if (rows) TRY(check_matrix("dy", dy, lddy, outer, es));
  if (rows && dx) {
    TRY(fill_table("w", w, experts, false, es, tw));
    TRY(check_matrix("w", w[0], ldw, w_transposed ? inner : outer, es));
    TRY(check_matrix("dx", dx, lddx, inner, es));
  }
  if (dw) {
    if (rows) TRY(check_matrix("x", x, ldx, inner, es));
    TRY(fill_table("dw", dw, experts, true, es, td));
    if (lddw < (w_transposed ? inner : outer) || lddw > kMaxLd)
      return fail(MUON_ERR_INVALID_ARG, "dw has leading dimension %lld, needs at least %lld", (long long)lddw,
                  (long long)(w_transposed ? inner : outer));
  }
  size_t need = 0;
  TRY(muon_grouped_linear_workspace_bytes(rows, inner, outer, experts, dtype, 1, &need));
  TRY(check_workspace(workspace, workspace_bytes, need));
  const hipStream_t st = hipStream_t(hip_stream);
  Product p{};
  p.offsets = offsets;
  p.experts = experts;
  if (dx && rows) {
    p.a = dy; p.lda = lddy;
    p.ldb = ldw;
    p.c = dx; p.ldc = lddx;
    p.M = int32_t(rows); p.N = int32_t(inner); p.K = int32_t(outer);
    TRY(done(product(bf16, w_transposed ? FORM_RT : FORM_RR, GROUP_ROWS, p, &tw, st), "grouped input gradient"));
  }
  if (dw) {
    p.c = nullptr; p.ldc = lddw;
    p.K = int32_t(rows);
    p.a = w_transposed ? dy : x; p.lda = w_transposed ? lddy : ldx;
    p.b = w_transposed ? x : dy; p.ldb = w_transposed ? ldx : lddy;
    p.M = int32_t(w_transposed ? outer : inner); p.N = int32_t(w_transposed ? inner : outer);
    TRY(done(product(bf16, FORM_TT, GROUP_SUM, p, &td, st), "grouped weight gradients"));
  }
  return done(hipSuccess, "");
}

MUON_API muon_status muon_layer_norm_forward(const void* x, int64_t ldx, const void* weight, const void* bias, void* y,
                                             int64_t ldy, float* mean, float* rstd, int64_t rows, int64_t cols,
                                             float eps, int32_t dtype, int32_t weight_dtype, void* hip_stream) {
  TRY(check_sizes(rows, cols, cols, dtype));
  if (weight_dtype != MUON_F32 && weight_dtype != dtype)
    return fail(MUON_ERR_UNSUPPORTED, "weight_dtype %d: MUON_F32 or the dtype of x", weight_dtype);
  if (!std::isfinite(eps) || eps < 0.f) return fail(MUON_ERR_INVALID_ARG, "eps must be finite and >= 0");
  if (rows == 0) return done(hipSuccess, "");
  const size_t es = size_of(dtype), ws = size_of(weight_dtype);
  TRY(check_matrix("x", x, ldx, cols, es));
  TRY(check_matrix("y", y, ldy, cols, es));
  TRY(check_vector("weight", weight, ws));
  TRY(check_vector("bias", bias, ws));
  TRY(check_vector("mean", mean, 4));
  TRY(check_vector("rstd", rstd, 4));
  NormArgs a{};
  a.x = x; a.ldx = ldx;
  a.y = y; a.ldy = ldy;
  a.weight = weight; a.bias = bias;
  a.mean = mean; a.rstd = rstd;
  a.rows = int32_t(rows); a.cols = int32_t(cols);
  a.wf32 = weight_dtype == MUON_F32;
  a.eps = eps;
  return done(launch_norm_forward(dtype == MUON_BF16, a, hipStream_t(hip_stream)), "layer norm forward");
}

MUON_API muon_status muon_layer_norm_workspace_bytes(int64_t rows, int64_t cols, size_t* bytes) {
  if (!bytes) return fail(MUON_ERR_INVALID_ARG, "bytes is NULL");
  TRY(check_sizes(rows, cols, cols, MUON_F32));
  *bytes = padded(size_t(norm_blocks(rows, cols)) * 2 * size_t(cols) * 4);
  return done(hipSuccess, "");
}

MUON_API muon_status muon_layer_norm_backward(const void* dy, int64_t lddy, const void* x, int64_t ldx,
                                              const void* weight, const float* mean, const float* rstd, void* dx,
                                              int64_t lddx, void* dweight, void* dbias, int64_t rows, int64_t cols,
                                              int32_t dtype, int32_t weight_dtype, void* workspace,
                                              size_t workspace_bytes, void* hip_stream) {
  TRY(check_sizes(rows, cols, cols, dtype));
  if (weight_dtype != MUON_F32 && weight_dtype != dtype)
    return fail(MUON_ERR_UNSUPPORTED, "weight_dtype %d: MUON_F32 or the dtype of x", weight_dtype);
  const size_t es = size_of(dtype), wsz = size_of(weight_dtype);
  if (rows) {
    TRY(check_matrix("dy", dy, lddy, cols, es));
    TRY(check_matrix("x", x, ldx, cols, es));
    if (!mean || !rstd) return fail(MUON_ERR_INVALID_ARG, "mean or rstd is NULL");
    TRY(check_vector("mean", mean, 4));
    TRY(check_vector("rstd", rstd, 4));
    if (dx) TRY(check_matrix("dx", dx, lddx, cols, es));
  }
  TRY(check_vector("weight", weight, wsz));
  TRY(check_vector("dweight", dweight, wsz));
  TRY(check_vector("dbias", dbias, wsz));
  size_t need = 0;
  if (dweight || dbias) TRY(muon_layer_norm_workspace_bytes(rows, cols, &need));
  TRY(check_workspace(workspace, workspace_bytes, need));
  NormArgs a{};
  a.dy = dy; a.lddy = lddy;
  a.x = x; a.ldx = ldx;
  a.weight = weight;
  a.mean = const_cast<float*>(mean); a.rstd = const_cast<float*>(rstd);
  a.dx = dx; a.lddx = lddx;
  a.dweight = dweight; a.dbias = dbias;
  a.part = static_cast<float*>(workspace);
  a.rows = int32_t(rows); a.cols = int32_t(cols);
  a.wf32 = weight_dtype == MUON_F32;
  return done(launch_norm_backward(dtype == MUON_BF16, a, hipStream_t(hip_stream)), "layer norm backward");
}

}  // extern "C"
