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
  if (e == hipErrorInvalidConfiguration) return fail(MUON_ERR_UNSUPPORTED, "%s: more tiles than one grid holds", what);
  if (e != hipSuccess) return fail(MUON_ERR_DEVICE, "%s: %s", what, hipGetErrorString(e));
  g_error[0] = 0;
  return MUON_OK;
}

constexpr int64_t kMaxRows = int64_t(1) << 30, kMaxDim = int64_t(1) << 24;
constexpr int64_t kMaxLd = int64_t(1) << 40;

bool known_dtype(int32_t d) { return d == MUON_F32 || d == MUON_BF16; }
size_t size_of(int32_t dtype) { return dtype == MUON_BF16 ? 2 : 4; }
size_t padded(size_t v) { return (v + 255) / 256 * 256; }

muon_status check_sizes(int64_t rows, int64_t inner, int64_t outer, int32_t dtype) {
  if (rows < 0 || rows > kMaxRows) return fail(MUON_ERR_INVALID_ARG, "rows %lld out of [0, 2^30]", (long long)rows);
  if (inner < 1 || inner > kMaxDim)
    return fail(MUON_ERR_INVALID_ARG, "inner %lld out of [1, 2^24]", (long long)inner);
  if (outer < 1 || outer > kMaxDim)
    return fail(MUON_ERR_INVALID_ARG, "outer %lld out of [1, 2^24]", (long long)outer);
  if (!known_dtype(dtype)) return fail(MUON_ERR_UNSUPPORTED, "dtype %d: MUON_F32 or MUON_BF16", dtype);
  return MUON_OK;
}

muon_status check_activation(int32_t a) {
  if (a < MUON_ACT_NONE || a > MUON_ACT_SILU) return fail(MUON_ERR_INVALID_ARG, "unknown activation %d", a);
  return MUON_OK;
}

muon_status check_flags(int32_t f) {
  if (f & ~(MUON_LAYERS_BACKWARD | MUON_LAYERS_UNALIGNED)) return fail(MUON_ERR_INVALID_ARG, "unknown flags %d", f);
  return MUON_OK;
}

// A matrix operand: a pointer aligned to its element and a leading dimension of
// at least its columns.
muon_status check_matrix(const char* name, const void* p, int64_t ld, int64_t cols, size_t esize) {
  if (!p) return fail(MUON_ERR_INVALID_ARG, "%s is NULL", name);
  if (reinterpret_cast<uintptr_t>(p) % esize)
    return fail(MUON_ERR_INVALID_ARG, "%s is not aligned to its element", name);
  if (ld < cols || ld > kMaxLd)
    return fail(MUON_ERR_INVALID_ARG, "%s has leading dimension %lld, needs at least %lld", name, (long long)ld,
                (long long)cols);
  return MUON_OK;
}

muon_status check_vector(const char* name, const void* p, size_t esize) {
  if (reinterpret_cast<uintptr_t>(p) % esize)
    return fail(MUON_ERR_INVALID_ARG, "%s is not aligned to its element", name);
  return MUON_OK;
}

muon_status check_workspace(const void* ws, size_t have, size_t need) {
  // (more than the need may be used: for copies)
  if (have && reinterpret_cast<uintptr_t>(ws) % 256)
    return fail(MUON_ERR_INVALID_ARG, "workspace must be 256-byte aligned");
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

// Whether the tile kernels can fetch an operand of rows of `cols` elements:
// 16-byte chunks that lie on 16-byte addresses and do not straddle the end of a
// row, and 32-bit byte offsets within a tile of 256 rows.
bool rows_fit(const void* ptr, int64_t ld, int64_t cols, int64_t epc) {
  return aligned16(ptr) && ld % epc == 0 && cols % epc == 0 && ld * 16 / epc * 256 < (int64_t(1) << 31);
}
struct Fits {
  bool a, b;
};
Fits tile_fits(bool bf16, int form, int group, const Product& p, const Table* t) {
  const int64_t epc = bf16 ? 8 : 4;
  Fits f;
  f.a = rows_fit(p.a, p.lda, form == FORM_TT ? p.M : p.K, epc);
  const int64_t cols = form == FORM_RR ? p.K : p.N;
  f.b = group != GROUP_ROWS && rows_fit(p.b, p.ldb, cols, epc);
  if (group == GROUP_ROWS) {
    f.b = true;
    for (int32_t e = 0; e < p.experts && f.b; ++e) f.b = rows_fit(t->p[e], p.ldb, cols, epc);
  }
  return f;
}

// Shapes of the operands' copies (pack.hip): rows of whole chunks.
PackOne copy_shape(int64_t rows, int64_t cols, int64_t epc) {
  PackOne o{};
  o.rows = rows;
  o.cols = cols;
  o.ld_dst = (cols + epc - 1) / epc * epc;
  return o;
}
PackOne copy_of_a(int form, int64_t M, int64_t K, int64_t epc) {
  return form == FORM_TT ? copy_shape(K, M, epc) : copy_shape(M, K, epc);
}
PackOne copy_of_b(int form, int64_t N, int64_t K, int64_t epc) {
  return form == FORM_RR ? copy_shape(N, K, epc) : copy_shape(K, N, epc);
}
size_t copy_bytes(const PackOne& o, int64_t epc, int64_t copies) {
  return padded(size_t(o.rows) * size_t(o.ld_dst) * size_t(16 / epc) * size_t(copies));
}

// Which kernel runs a product, and into how many ranges it cuts the summed
// dimension (each range leaves an fp32 partial result; not where experts own
// ranges of it).
struct Choice {
  enum Kernel { SIMPLE, SKINNY, TILE64, TILE128, TILE128X256, TILE256 } kernel = SIMPLE;
  int mt = 0;       // SKINNY: 16-row tiles per block
  int splits = 1;
};

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// The tile kernels, and the measured times their expected run time is made of:
// us a slab (64 K in bf16, 32 in fp32) with the chip full and with one block on a
// CU, us for everything else of a tile (its first loads and its epilogue; act:
// more for an activation), and blocks per CU.  Where two blocks share a CU, `full`
// is for the two.  They are for ranking kernels; the sums come within 13% of what
// is measured (bf16, 5832 x 1152 x 4304: x W with an activation 76 us for 77, dz W^T 64
// for 70 to 74, x^T dz 79 for 82 to 84).
struct TileKind {
  Choice::Kernel kernel;
  int tm, tn;
  double full, alone, rest, act;
  int per_cu;
};
constexpr TileKind kBf16Tiles[] = {{Choice::TILE256, 256, 256, 1.55, 1.1, 7, 5, 1},
                                   {Choice::TILE128X256, 128, 256, 0.9, 0.66, 5, 3, 1},
                                   {Choice::TILE128, 128, 128, 0.95, 0.53, 5, 3.5, 2},
                                   {Choice::TILE64, 64, 64, 0.4, 0.29, 3, 1, 2}};
constexpr TileKind kF32Tiles[] = {{Choice::TILE128, 128, 128, 4.0, 2.05, 4.5, 0, 2},
                                  {Choice::TILE64, 64, 64, 1.08, 0.57, 3.5, 0, 2}};

double tile_us(const TileKind& k, double blocks, double slabs, bool act) {
  const double rest = k.rest + (act ? k.act : 0), cus = kCUs;
  if (k.per_cu == 1) {
    const double rounds = std::floor(blocks / cus), left = blocks - rounds * cus;
    return rounds * (slabs * k.full + rest) +
           (left > 0 ? slabs * (k.alone + (k.full - k.alone) * left / cus) + rest : 0);
  }
  if (blocks <= cus) return slabs * k.alone + rest;
  return (blocks <= 2 * cus ? 1 : blocks / (2 * cus)) * (slabs * k.full + rest);
}

// Partial results are written and read once in fp32 (4 bytes a pass at about
// 4 TB/s); the kernel that adds them costs a launch.
double reduce_us(int64_t M, int64_t N, int splits) {
  return splits > 1 ? 3.0 + double(splits) * M * N * 8 / 4e6 : 0.0;
}

Choice choose(bool bf16, int form, int group, int64_t M, int64_t N, int64_t K, int64_t experts,
              bool act) {
  Choice c;
  const int64_t epc = bf16 ? 8 : 4;
  // Few rows: the weight's bytes are all that counts, which the skinny kernel
  // streams without LDS.  From 65 rows on (17 per expert) the tile kernels win.
  const double per_expert = group == GROUP_ROWS ? double(M) / experts : double(M);
  if (form != FORM_TT && N >= epc && per_expert <= (group == GROUP_ROWS ? 16 : 64)) {
    c.kernel = Choice::SKINNY;
    c.mt = group == GROUP_ROWS || M <= 16 ? 1 : M <= 32 ? 2 : 4;
    // 512 blocks keep enough loads in flight: two per CU (of the bf16 kernel for 33 to
    // 64 rows, which takes 268 registers, one at a time); at least 4 K steps per wave.
    // Of experts, as many as rows or half of them are taken to be met.
    const int64_t met = group == GROUP_NONE ? 1 : M < (experts + 1) / 2 ? M : (experts + 1) / 2;
    const int64_t blocks = ceil_div(N, 16 * epc) * met, steps = ceil_div(K, 4 * epc);
    int64_t s = 512 / blocks;
    s = s < steps / 16 ? s : steps / 16;
    c.splits = int(s < 1 ? 1 : s);
    return c;
  }
  const int64_t bk = bf16 ? 64 : 32;
  double best = 0;
  const TileKind* kinds = bf16 ? kBf16Tiles : kF32Tiles;
  for (int i = 0; i < (bf16 ? 4 : 2); ++i) {
    const TileKind& k = kinds[i];
    const int64_t nt = ceil_div(N, k.tn);
    double blocks = double(ceil_div(M, k.tm) * nt), slabs = double(ceil_div(K, bk));
    // experts: half a tile of rows (half a slab) is lost on each
    if (group == GROUP_ROWS) blocks = (double(M) / k.tm + 0.5 * (experts < M ? experts : M)) * nt;
    if (group == GROUP_SUM) {
      blocks *= experts;
      slabs = double(K) / experts / bk + 0.5;
    }
    for (int s = 1; s <= 16; ++s) {
      if (s > 1 && (group == GROUP_SUM || slabs < 4 * s)) break;
      const double us = tile_us(k, blocks * s, std::ceil(slabs / s), act) + reduce_us(M, N, s);
      if (best == 0 || us < best) {
        best = us;
        c.kernel = k.kernel;
        c.splits = s;
      }
    }
  }
  return c;
}

size_t part_bytes(const Choice& c, int64_t M, int64_t N) {
  return c.splits > 1 ? padded(size_t(c.splits) * size_t(M) * size_t(N) * 4) : 0;
}

// Scratch memory of a product, and what it can use: partial results, and copies
// of operands the tile kernels cannot fetch.
struct Scratch {
  char* p;
  size_t bytes;
};

// One matrix product: the kernel that suits it.  Operands off 16-byte rows are
// copied first if the scratch memory holds the copies; else the simple kernel
// takes them as they lie.
hipError_t product(bool bf16, int form, int group, Product p, const Table* t, Scratch ws, hipStream_t st) {
  const int64_t epc = bf16 ? 8 : 4;
  Choice c = choose(bf16, form, group, p.M, p.N, p.K, p.experts, p.act != MUON_ACT_NONE);
  hipError_t e = hipSuccess;
  Table copies;
  if (c.kernel != Choice::SKINNY) {
    const Fits f = tile_fits(bf16, form, group, p, t);
    if (!f.a || !f.b) {
      PackArgs k{};
      const int64_t n = group == GROUP_ROWS ? p.experts : 1;
      size_t used = part_bytes(c, p.M, p.N);
      if (!f.a) {
        k.a = copy_of_a(form, p.M, p.K, epc);
        k.a.src = p.a;
        k.a.ld_src = p.lda;
        k.a.dst = ws.p + used;
        used += copy_bytes(k.a, epc, 1);
      }
      if (!f.b) {
        k.b = copy_of_b(form, p.N, p.K, epc);
        k.b.src = p.b;
        k.b.ld_src = p.ldb;
        k.b.dst = ws.p + used;
        k.experts = group == GROUP_ROWS ? p.experts : 0;
        used += copy_bytes(k.b, epc, n);
      }
      // (the tile kernels' 32-bit offsets hold for the copies too)
      const int64_t longest = k.a.ld_dst > k.b.ld_dst ? k.a.ld_dst : k.b.ld_dst;
      const bool near = longest * 16 / epc * 256 < (int64_t(1) << 31);
      if (ws.p && used <= ws.bytes && near && p.K > 0) {
        static const Table none{};
        e = launch_pack(bf16, k, group == GROUP_ROWS ? *t : none, st);
        if (e != hipSuccess) return e;
        if (!f.a) {
          p.a = k.a.dst;
          p.lda = k.a.ld_dst;
        }
        if (!f.b) {
          p.b = k.b.dst;
          p.ldb = k.b.ld_dst;
          if (group == GROUP_ROWS) {
            const size_t step = size_t(k.b.rows) * size_t(k.b.ld_dst) * size_t(16 / epc);
            for (int32_t i = 0; i < p.experts; ++i) copies.p[i] = static_cast<char*>(k.b.dst) + i * step;
            t = &copies;
          }
        }
      } else {
        c = Choice{};
      }
    }
  }
  p.splits = c.splits;
  p.part = reinterpret_cast<float*>(ws.p);
  switch (c.kernel) {
    case Choice::SIMPLE: e = launch_simple(bf16, form, group, p, t, st); break;
    case Choice::SKINNY: e = launch_skinny(bf16, form, group, c.mt, p, t, st); break;
    case Choice::TILE64:
      e = bf16 ? launch_tile64_bf16(form, group, p, t, st) : launch_tile64_f32(form, group, p, t, st);
      break;
    case Choice::TILE128:
      e = bf16 ? launch_tile128_bf16(form, group, p, t, st) : launch_tile128_f32(form, group, p, t, st);
      break;
    case Choice::TILE128X256: e = launch_tile128x256_bf16(form, group, p, t, st); break;
    case Choice::TILE256: e = launch_tile256_bf16(form, group, p, t, st); break;
  }
  return e == hipSuccess && c.splits > 1 ? launch_reduce(bf16, p, st) : e;
}
// What product() can use.  copies: for operands at any alignment.
size_t product_bytes(bool bf16, int form, int group, int64_t M, int64_t N, int64_t K, int64_t experts, bool act,
                     bool copies) {
  if (M == 0 || K == 0) return 0;
  const int64_t epc = bf16 ? 8 : 4;
  const Choice c = choose(bf16, form, group, M, N, K, experts, act);
  size_t b = part_bytes(c, M, N);
  if (copies && c.kernel != Choice::SKINNY)
    b += copy_bytes(copy_of_a(form, M, K, epc), epc, 1) +
         copy_bytes(copy_of_b(form, N, K, epc), epc, group == GROUP_ROWS ? experts : 1);
  return b;
}
// Most of a layer's products, in either layout of the weight.
size_t forward_bytes(int group, int64_t rows, int64_t inner, int64_t outer, int64_t experts, int32_t dtype,
                     bool act, bool copies) {
  const bool bf16 = dtype == MUON_BF16;
  const size_t a = product_bytes(bf16, FORM_RT, group, rows, outer, inner, experts, act, copies);
  const size_t b = product_bytes(bf16, FORM_RR, group, rows, outer, inner, experts, act, copies);
  return a > b ? a : b;
}
size_t gradient_bytes(int group, int64_t rows, int64_t inner, int64_t outer, int64_t experts, int32_t dtype,
                      bool copies) {
  const bool bf16 = dtype == MUON_BF16;
  const int sums = group == GROUP_ROWS ? GROUP_SUM : GROUP_NONE;
  const size_t dx = forward_bytes(group, rows, outer, inner, experts, dtype, false, copies);
  const size_t d1 = product_bytes(bf16, FORM_TT, sums, inner, outer, rows, experts, false, copies);
  const size_t d2 = product_bytes(bf16, FORM_TT, sums, outer, inner, rows, experts, false, copies);
  const size_t dw = d1 > d2 ? d1 : d2;
  return dx > dw ? dx : dw;
}

// Workspace of muon_linear_backward: dz, the partial column sums and the two
// products' scratch memory (one after the other, in one place).
struct BackwardLayout {
  size_t dz = 0, sums = 0, scratch = 0, total = 0;
};
BackwardLayout backward_layout(int64_t rows, int64_t inner, int64_t outer, int32_t dtype, int32_t act, bool copies) {
  BackwardLayout l;
  if (act != MUON_ACT_NONE) l.sums = padded(size_t(rows) * size_t(outer) * size_of(dtype));
  l.scratch = l.sums + padded(size_t(act_grad_chunks(rows, outer)) * size_t(outer) * 4);
  l.total = l.scratch + gradient_bytes(GROUP_NONE, rows, inner, outer, 0, dtype, copies);
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
                                                 int32_t activation, int32_t flags, size_t* bytes) {
  if (!bytes) return fail(MUON_ERR_INVALID_ARG, "bytes is NULL");
  TRY(check_sizes(rows, inner, outer, dtype));
  TRY(check_activation(activation));
  TRY(check_flags(flags));
  const bool copies = flags & MUON_LAYERS_UNALIGNED, act = activation != MUON_ACT_NONE;
  *bytes = flags & MUON_LAYERS_BACKWARD ? backward_layout(rows, inner, outer, dtype, activation, copies).total
                                        : forward_bytes(GROUP_NONE, rows, inner, outer, 0, dtype, act, copies);
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
  const bool act = activation != MUON_ACT_NONE;
  TRY(check_workspace(workspace, workspace_bytes, forward_bytes(GROUP_NONE, rows, inner, outer, 0, dtype, act, false)));
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
                      Scratch{static_cast<char*>(workspace), workspace_bytes}, hipStream_t(hip_stream)),
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
  const BackwardLayout l = backward_layout(rows, inner, outer, dtype, activation, false);
  TRY(check_workspace(workspace, workspace_bytes, l.total));
  const hipStream_t st = hipStream_t(hip_stream);
  char* ws = static_cast<char*>(workspace);
  const Scratch scratch{ws ? ws + l.scratch : nullptr, workspace_bytes > l.scratch ? workspace_bytes - l.scratch : 0};
  const void* dz = dy;
  int64_t lddz = lddy;
  if ((act && rows) || dbias) {
    ActGradArgs a{};
    a.dy = dy; a.lddy = lddy;
    a.z = act ? preact : nullptr; a.ldz = ldz;
    a.dz = act ? ws + l.dz : nullptr; a.lddz = outer;
    a.dbias = dbias;
    a.part = reinterpret_cast<float*>(ws + l.sums);
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
    TRY(done(product(bf16, w_transposed ? FORM_RT : FORM_RR, GROUP_NONE, p, nullptr, scratch, st),
             "linear input gradient"));
  }
  if (dw) {
    Product p{};
    p.c = dw; p.ldc = lddw;
    p.K = int32_t(rows);
    // dW = x^T dz, or dW^T = dz^T x for a transposed weight
    p.a = w_transposed ? dz : x; p.lda = w_transposed ? lddz : ldx;
    p.b = w_transposed ? x : dz; p.ldb = w_transposed ? ldx : lddz;
    p.M = int32_t(w_transposed ? outer : inner); p.N = int32_t(w_transposed ? inner : outer);
    TRY(done(product(bf16, FORM_TT, GROUP_NONE, p, nullptr, scratch, st), "linear weight gradient"));
  }
  return done(hipSuccess, "");
}

MUON_API muon_status muon_grouped_linear_workspace_bytes(int64_t rows, int64_t inner, int64_t outer, int32_t experts,
                                                         int32_t dtype, int32_t flags, size_t* bytes) {
  if (!bytes) return fail(MUON_ERR_INVALID_ARG, "bytes is NULL");
  TRY(check_sizes(rows, inner, outer, dtype));
  if (experts < 1 || experts > MUON_GROUPED_MAX_EXPERTS)
    return fail(MUON_ERR_INVALID_ARG, "experts %d out of [1, %d]", experts, MUON_GROUPED_MAX_EXPERTS);
  TRY(check_flags(flags));
  const bool copies = flags & MUON_LAYERS_UNALIGNED;
  *bytes = flags & MUON_LAYERS_BACKWARD ? gradient_bytes(GROUP_ROWS, rows, inner, outer, experts, dtype, copies)
                                        : forward_bytes(GROUP_ROWS, rows, inner, outer, experts, dtype, false, copies);
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
                      Scratch{static_cast<char*>(workspace), workspace_bytes}, hipStream_t(hip_stream)),
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
  TRY(muon_grouped_linear_workspace_bytes(rows, inner, outer, experts, dtype, MUON_LAYERS_BACKWARD, &need));
  TRY(check_workspace(workspace, workspace_bytes, need));
  const hipStream_t st = hipStream_t(hip_stream);
  const Scratch scratch{static_cast<char*>(workspace), workspace_bytes};
  Product p{};
  p.offsets = offsets;
  p.experts = experts;
  if (dx && rows) {
    p.a = dy; p.lda = lddy;
    p.ldb = ldw;
    p.c = dx; p.ldc = lddx;
    p.M = int32_t(rows); p.N = int32_t(inner); p.K = int32_t(outer);
    TRY(done(product(bf16, w_transposed ? FORM_RT : FORM_RR, GROUP_ROWS, p, &tw, scratch, st),
             "grouped input gradient"));
  }
  if (dw) {
    p.c = nullptr; p.ldc = lddw;
    p.K = int32_t(rows);
    p.a = w_transposed ? dy : x; p.lda = w_transposed ? lddy : ldx;
    p.b = w_transposed ? x : dy; p.ldb = w_transposed ? ldx : lddy;
    p.M = int32_t(w_transposed ? outer : inner); p.N = int32_t(w_transposed ? inner : outer);
    TRY(done(product(bf16, FORM_TT, GROUP_SUM, p, &td, scratch, st), "grouped weight gradients"));
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
