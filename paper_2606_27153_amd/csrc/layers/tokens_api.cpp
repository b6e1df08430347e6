// C ABI of the operators that take token or expert numbers: lookup in a table and
// its gradient, the way to the experts and back, and the loss over a vocabulary.
// Argument checks, workspace layouts and launch order.
#include "host.h"

namespace {

using namespace muon::layers;

constexpr int64_t kMaxInner = int64_t(1) << 20;   // of the loss: 256 rows of it within 32-bit offsets

muon_status check_count(const char* name, int64_t v, int64_t lo, int64_t hi) {
  if (v < lo || v > hi)
    return fail(MUON_ERR_INVALID_ARG, "%s %lld out of [%lld, %lld]", name, (long long)v, (long long)lo, (long long)hi);
  return MUON_OK;
}

muon_status check_ids(const char* name, const void* ids, int32_t bytes, int64_t n) {
  if (bytes != 4 && bytes != 8) return fail(MUON_ERR_UNSUPPORTED, "%s of %d bytes: 4 or 8", name, bytes);
  if (n && !ids) return fail(MUON_ERR_INVALID_ARG, "%s is NULL", name);
  if (reinterpret_cast<uintptr_t>(ids) % size_t(bytes))
    return fail(MUON_ERR_INVALID_ARG, "%s is not aligned to its element", name);
  return MUON_OK;
}

muon_status check_dtype(int32_t dtype) {
  return known_dtype(dtype) ? MUON_OK : fail(MUON_ERR_UNSUPPORTED, "dtype %d: MUON_F32 or MUON_BF16", dtype);
}

muon_status check_needed(const char* name, const void* p, size_t esize) {
  if (!p) return fail(MUON_ERR_INVALID_ARG, "%s is NULL", name);
  return check_vector(name, p, esize);
}

// ----------------------------------------------------------------- routing

muon_status check_choices(int64_t tokens, int64_t top) {
  TRY(check_count("tokens", tokens, 0, kMaxRows));
  TRY(check_count("top", top, 1, MUON_GROUPED_MAX_EXPERTS));
  if (tokens * top > kMaxRows) return fail(MUON_ERR_INVALID_ARG, "tokens * top is over 2^30");
  return MUON_OK;
}

muon_status check_route(int64_t tokens, int64_t top, int64_t cols, int32_t dtype) {
  TRY(check_choices(tokens, top));
  TRY(check_count("cols", cols, 1, kMaxDim));
  return check_dtype(dtype);
}

muon_status check_weights(const void* w, int32_t weight_dtype, int32_t dtype) {
  if (weight_dtype != MUON_F32 && weight_dtype != dtype)
    return fail(MUON_ERR_UNSUPPORTED, "weight_dtype %d: MUON_F32 or the dtype of the rows", weight_dtype);
  return check_needed("weights", w, size_of(weight_dtype));
}

RouteArgs route_args(int64_t tokens, int64_t top, int64_t cols, const int32_t* position = nullptr) {
  RouteArgs a{};
  a.tokens = int32_t(tokens);
  a.top = int32_t(top);
  a.cols = int32_t(cols);
  a.position = position;
  return a;
}

// -------------------------------------------------------------------- loss

// Rows at a time, fewer in a forward pass over a very large vocabulary: its strips'
// sums take 8 bytes a row and strip, 1 GB in all.
constexpr int64_t kLossRows = 32768;
constexpr int64_t kLossSums = int64_t(1) << 27;
// Columns of a piece: as many as one grid has tiles for; where the weight has to
// be copied, fewer, so that the copy stays small; of a gradient piece, 2^29 elements at most
// (and 2048 columns at least).
constexpr int64_t kPiece = int64_t(1) << 18, kCopyPiece = int64_t(1) << 15;
constexpr int64_t kGradPiece = int64_t(1) << 29;

int64_t even_piece(int64_t outer, int64_t most) {
  const int64_t pieces = ceil_div(outer, most);
  int64_t p = ceil_div(ceil_div(outer, pieces), 256) * 256;
  // of many pieces the last can be short: not below the 16 bytes of columns that the kernel of
  // few rows needs (their pieces are never smaller than these: two steps down are enough for
  // all of the 2^24 columns)
  while (most >= kCopyPiece && p > 256 && p < outer && outer % p && outer % p < 8) p -= 256;
  return p < outer ? p : outer;
}
size_t larger(size_t a, size_t b) { return a > b ? a : b; }

struct LossLayout {
  int64_t rows = 0;    // at a time
  int64_t piece = 0;   // columns at a time
  Choice z, x, w;      // the kernels of x W, dz W^T and x^T dz (a last piece has fewer columns, and the same ones)
  size_t logit = 0, loss = 0, alpha = 0, part = 0, raw = 0, dz = 0, dx = 0, wcopy = 0, xcopy = 0, scratch = 0, total = 0;
  void take(size_t& p, size_t bytes) {
    p = total;
    total += padded(bytes);
  }
};

// The kernel of a piece of x W: few rows leave it in memory (`raw`), tiles do not.
// The latter take over from 33 rows on (128000 x 4096 in bf16, 40 rows: 223 us for 294), and
// at once where a bf16 weight is kept by its columns, of which a wave of the other
// kernel reads 64 bytes at a time (one row: 182 us for 270; in fp32, 32000 x 2048, 92 for 69).
Choice choose_logits(bool bf16, bool w_transposed, int64_t rows, int64_t piece, int64_t inner) {
  const Choice c = choose(bf16, FORM_RT, GROUP_NONE, rows, piece, inner, 0, false);
  return c.kernel == Choice::SKINNY && rows <= 32 && !(w_transposed && bf16) ? c : choose_tile(bf16, GROUP_NONE, rows, piece, inner, 0, true, 1);
}
// Columns of its strips: a wave has half of a tile's.
int64_t strip_columns(const Choice& c) {
  switch (c.kernel) {
    case Choice::TILE256:
    case Choice::TILE128X256: return 128;
    case Choice::TILE128: return 64;
    case Choice::TILE64: return 32;
    default: return kRawStrip;
  }
}
// Whether the weight's gradient [down, across], as it is kept, is made by the outer product of
// few rows.  Its stores are streamed at the memory's rate, but a thread walks down 32 rows of it with
// a multiply-add for each element and row of x (4, 8, 16 or 32 of these): time that small gradients,
// whose blocks do not fill the CUs, cannot hide.  The tile kernels, one launch more, leave up
// to about 150 MB in the caches, and store beyond that at half the memory's rate.  us of a backward
// pass without dx, outer product and tile:
//   up to 4 rows (fp32 8): 16384 x 200 in bf16 17 and 21, 65536 x 2048 101 and 159
//   up to 8 (fp32 16), where a row has at most 128 lanes of 16 bytes: 32000 x 256 in bf16 20 and 20, in fp32
//     25 and 30; wider, of 12 MB 25 and 23, 21 MB 32 and 31, 33 MB 29 and 29 (fp32 29 and 29),
//     90 MB 45 and 52, 268 MB 104 and 160
//   up to 16 (fp32 32): in bf16 of 16 MB 32 and 20, 66 MB 48 and 37, 134 MB 80 and 63, 151 MB 88 and 91 or,
//     tied, 102 and 80, 185 MB 101 and 118 or 108 and 108, 268 MB 134 and 175; in fp32 of 33 MB 40 and 33,
//     66 MB 47 and 48 or, tied, 55 and 49, 131 MB 78 and 82 or 82 and 83, 180 MB 97 and 122
bool outer_product_wins(bool bf16, bool w_transposed, int64_t rows, int64_t inner, int64_t outer) {
  constexpr int64_t kWide = int64_t(24) << 20;
  if (!rows || rows > outer_rows(bf16)) return false;
  const int64_t es = bf16 ? 2 : 4, bytes = inner * outer * es, across = w_transposed ? inner : outer;
  if (rows <= 8 / (bf16 ? 2 : 1)) return true;
  if (rows <= 16 / (bf16 ? 2 : 1)) return bytes >= kWide || across * es <= 128 * 16;
  return bytes >= int64_t(bf16 ? 160 : 96) << 20;
}
size_t raw_bytes(const LossLayout& l) {
  return l.z.kernel == Choice::SKINNY ? size_t(l.z.splits) * size_t(l.rows) * size_t(l.piece) * 4 : 0;
}

hipError_t launch_loss_tile(const Choice& c, int step, bool bf16, int form, const Product& p, const LossArgs& a,
                            hipStream_t st) {
  switch (c.kernel) {
    case Choice::TILE64:
      return bf16 ? launch_loss64_bf16(step, form, p, a, st) : launch_loss64_f32(step, form, p, a, st);
    case Choice::TILE128:
      return bf16 ? launch_loss128_bf16(step, form, p, a, st) : launch_loss128_f32(step, form, p, a, st);
    case Choice::TILE128X256: return launch_loss128x256_bf16(step, form, p, a, st);
    case Choice::TILE256: return launch_loss256_bf16(step, form, p, a, st);
    default: return hipErrorInvalidValue;
  }
}

// A product of the loss by the kernel chosen for it, whose operands it can fetch.
hipError_t loss_product(const Choice& c, int step, bool bf16, int form, Product p, const LossArgs& a, char* part,
                        hipStream_t st) {
  p.splits = c.splits;
  p.part = reinterpret_cast<float*>(part);
  const hipError_t e = launch_loss_tile(c, step, bf16, form, p, a, st);
  return e == hipSuccess && c.splits > 1 ? launch_reduce(bf16, p, st) : e;
}
// A product left in fp32 at `sums`, as c.splits partial results, or added to what is there.
hipError_t product_sums(const Choice& c, bool bf16, int form, Product p, float* sums, hipStream_t st) {
  p.splits = c.splits;
  p.raw = 1;
  p.part = sums;
  return launch_choice(bf16, form, GROUP_NONE, c, p, nullptr, st);
}

// Copies of x (once; in the backward pass always, without what rows of no target hold) and of
// a piece of the weight, as it is kept, for all the products that read them: rows of
// whole chunks, zeros after the last column.
PackOne copy_of_w(int64_t piece, int64_t inner, bool w_transposed, int64_t epc) {
  return w_transposed ? copy_shape(piece, inner, epc) : copy_shape(inner, piece, epc);
}
void take_copies(LossLayout& l, int64_t rows, int64_t inner, bool w_transposed, bool bf16, bool unaligned,
                 bool backward) {
  const int64_t epc = bf16 ? 8 : 4;
  l.take(l.xcopy, unaligned || backward ? copy_bytes(copy_shape(rows, inner, epc), epc, 1) : 0);
  l.take(l.wcopy, unaligned ? copy_bytes(copy_of_w(l.piece, inner, w_transposed, epc), epc, 1) : 0);
}

LossLayout forward_layout(int64_t rows, int64_t inner, int64_t outer, bool w_transposed, bool bf16, bool unaligned) {
  LossLayout l;
  l.piece = even_piece(outer, unaligned ? kCopyPiece : kPiece);
  // as many rows as the strips of the kernel chosen for them allow: 256 at least (2^24
  // columns by 32)
  for (int64_t strip = 128;;) {
    const int64_t sums = kLossSums / ceil_div(outer, strip), most = sums < kLossRows ? sums : kLossRows;
    l.rows = rows < most ? rows : most;
    l.z = choose_logits(bf16, w_transposed, l.rows, l.piece, inner);
    if (strip_columns(l.z) >= strip) break;
    strip = strip_columns(l.z);
  }
  l.take(l.logit, size_t(rows) * 4);
  l.take(l.loss, size_t(rows) * 4);
  l.take(l.part, size_t(ceil_div(outer, l.piece)) * size_t(ceil_div(l.piece, strip_columns(l.z))) * size_t(l.rows) * 8);
  l.take(l.raw, raw_bytes(l));
  if (l.z.kernel != Choice::SKINNY) take_copies(l, rows, inner, w_transposed, bf16, unaligned, false);
  return l;
}

LossLayout backward_layout(int64_t rows, int64_t inner, int64_t outer, bool w_transposed, bool bf16, bool unaligned) {
  LossLayout l;
  const int64_t cap = unaligned ? kCopyPiece : kPiece;
  int64_t most = kGradPiece / (rows > 0 ? rows : 1) / 256 * 256;
  most = most < 2048 ? 2048 : most > cap ? cap : most;
  l.rows = rows < kLossRows ? rows : kLossRows;
  l.piece = even_piece(outer, most);
  l.z = choose_logits(bf16, w_transposed, l.rows, l.piece, inner);
  l.x = choose(bf16, FORM_RT, GROUP_NONE, rows, inner, l.piece, 0, false);
  const int64_t wm = w_transposed ? l.piece : inner, wn = w_transposed ? inner : l.piece;
  l.w = choose(bf16, FORM_TT, GROUP_NONE, wm, wn, rows, 0, false);
  l.take(l.alpha, 4);
  l.take(l.dz, size_t(rows) * size_t(ceil_div(l.piece, 8) * 8) * (bf16 ? 2 : 4));
  l.take(l.raw, raw_bytes(l));
  l.take(l.dx, size_t(l.x.splits) * size_t(rows) * size_t(inner) * 4);
  take_copies(l, rows, inner, w_transposed, bf16, unaligned, true);
  l.take(l.scratch, part_bytes(l.w, wm, wn));
  return l;
}

muon_status check_loss(int64_t rows, int64_t inner, int64_t outer, int32_t dtype, int32_t reduction) {
  TRY(check_sizes(rows, inner, outer, dtype));
  if (inner > kMaxInner) return fail(MUON_ERR_UNSUPPORTED, "inner %lld: at most 2^20", (long long)inner);
  if (reduction < MUON_LOSS_ROWS || reduction > MUON_LOSS_MEAN)
    return fail(MUON_ERR_INVALID_ARG, "unknown reduction %d", reduction);
  return MUON_OK;
}

// x or a piece of the weight as a product's operand: where it lies, or its copy.
struct Operand {
  const void* p;
  int64_t ld;
};
bool x_fits(const Operand& x, int64_t inner, bool bf16) { return rows_fit(x.p, x.ld, inner, bf16 ? 8 : 4); }
bool w_fits(const Operand& w, int64_t inner, int64_t outer, bool w_transposed, bool bf16) {
  return rows_fit(w.p, w.ld, w_transposed ? inner : outer, bf16 ? 8 : 4);
}
// Columns first .. of a weight.
Operand columns(const Operand& w, bool w_transposed, int64_t first, size_t es) {
  return Operand{static_cast<const char*>(w.p) + size_t(w_transposed ? first * w.ld : first) * es, w.ld};
}
hipError_t copy_operand(bool bf16, Operand& o, PackOne shape, void* to, hipStream_t st) {
  PackArgs k{};
  k.a = shape;
  k.a.src = o.p;
  k.a.ld_src = o.ld;
  k.a.dst = to;
  static const Table none{};
  o = Operand{to, shape.ld_dst};
  return launch_pack(bf16, k, none, st);
}

}  // namespace

extern "C" {

MUON_API muon_status muon_sort_by_expert_workspace_bytes(int64_t tokens, int32_t top, size_t* bytes) {
  if (!bytes) return fail(MUON_ERR_INVALID_ARG, "bytes is NULL");
  TRY(check_choices(tokens, top));
  *bytes = padded(expert_sort_bytes(tokens * top));
  return done(hipSuccess, "");
}

MUON_API muon_status muon_sort_by_expert(const void* ids, int32_t id_bytes, int64_t tokens, int32_t top,
                                         int32_t experts, int32_t* offsets, int32_t* position, int32_t* source,
                                         void* workspace, size_t workspace_bytes, void* hip_stream) {
  TRY(check_choices(tokens, top));
  TRY(check_count("experts", experts, 1, MUON_GROUPED_MAX_EXPERTS));
  const int64_t n = tokens * top;
  TRY(check_ids("ids", ids, id_bytes, n));
  TRY(check_needed("offsets", offsets, 4));
  if (n) {
    TRY(check_needed("position", position, 4));
    TRY(check_needed("source", source, 4));
  }
  size_t need = 0;
  TRY(muon_sort_by_expert_workspace_bytes(tokens, top, &need));
  TRY(check_workspace(workspace, workspace_bytes, need));
  return done(launch_expert_sort(ids, id_bytes, n, experts, offsets, position, source,
                                 static_cast<int32_t*>(workspace), hipStream_t(hip_stream)),
              "sort by expert");
}

MUON_API muon_status muon_dispatch_forward(const void* x, int64_t ldx, const int32_t* position, const int32_t* source,
                                           void* rows, int64_t ldr, int64_t tokens, int32_t top, int64_t cols,
                                           int32_t dtype, void* hip_stream) {
  TRY(check_route(tokens, top, cols, dtype));
  if (!tokens) return done(hipSuccess, "");
  const size_t es = size_of(dtype);
  TRY(check_matrix("x", x, ldx, cols, es));
  TRY(check_matrix("rows", rows, ldr, cols, es));
  TRY(check_needed("position", position, 4));
  TRY(check_needed("source", source, 4));
  RouteArgs a = route_args(tokens, top, cols, position);
  a.source = source;
  a.x = x; a.ldx = ldx;
  a.rows = rows; a.ldr = ldr;
  return done(launch_route(dtype == MUON_BF16, ROUTE_DISPATCH, a, hipStream_t(hip_stream)), "dispatch");
}

MUON_API muon_status muon_dispatch_backward(const void* drows, int64_t ldr, const int32_t* position, void* dx,
                                            int64_t ldx, int64_t tokens, int32_t top, int64_t cols, int32_t dtype,
                                            void* hip_stream) {
  TRY(check_route(tokens, top, cols, dtype));
  if (!tokens) return done(hipSuccess, "");
  const size_t es = size_of(dtype);
  TRY(check_matrix("drows", drows, ldr, cols, es));
  TRY(check_matrix("dx", dx, ldx, cols, es));
  TRY(check_needed("position", position, 4));
  RouteArgs a = route_args(tokens, top, cols, position);
  a.rows = const_cast<void*>(drows); a.ldr = ldr;
  a.y = dx; a.ldy = ldx;
  return done(launch_route(dtype == MUON_BF16, ROUTE_GATHER, a, hipStream_t(hip_stream)), "dispatch backward");
}

MUON_API muon_status muon_combine_forward(const void* rows, int64_t ldr, const void* weights, int32_t weight_dtype,
                                          const int32_t* position, const void* residual, int64_t ldres, void* y,
                                          int64_t ldy, int64_t tokens, int32_t top, int64_t cols, int32_t dtype,
                                          void* hip_stream) {
  TRY(check_route(tokens, top, cols, dtype));
  if (!tokens) return done(hipSuccess, "");
  const size_t es = size_of(dtype);
  TRY(check_matrix("rows", rows, ldr, cols, es));
  TRY(check_weights(weights, weight_dtype, dtype));
  TRY(check_needed("position", position, 4));
  if (residual) TRY(check_matrix("residual", residual, ldres, cols, es));
  TRY(check_matrix("y", y, ldy, cols, es));
  RouteArgs a = route_args(tokens, top, cols, position);
  a.rows = const_cast<void*>(rows); a.ldr = ldr;
  a.weights = weights; a.wf32 = weight_dtype == MUON_F32;
  a.res = residual; a.ldres = ldres;
  a.y = y; a.ldy = ldy;
  return done(launch_route(dtype == MUON_BF16, ROUTE_GATHER, a, hipStream_t(hip_stream)), "combine");
}

MUON_API muon_status muon_combine_backward(const void* dy, int64_t lddy, const void* rows, int64_t ldr,
                                           const void* weights, int32_t weight_dtype, const int32_t* source,
                                           void* drows, int64_t lddr, void* dweights, int64_t tokens, int32_t top,
                                           int64_t cols, int32_t dtype, void* hip_stream) {
  TRY(check_route(tokens, top, cols, dtype));
  if (!tokens) return done(hipSuccess, "");
  const size_t es = size_of(dtype);
  TRY(check_matrix("dy", dy, lddy, cols, es));
  if (dweights) TRY(check_matrix("rows", rows, ldr, cols, es));
  TRY(check_weights(weights, weight_dtype, dtype));
  TRY(check_needed("source", source, 4));
  if (drows) TRY(check_matrix("drows", drows, lddr, cols, es));
  TRY(check_vector("dweights", dweights, size_of(weight_dtype)));
  RouteArgs a = route_args(tokens, top, cols);
  a.source = source;
  a.dy = dy; a.lddy = lddy;
  a.rows = const_cast<void*>(rows); a.ldr = ldr;
  a.weights = weights; a.wf32 = weight_dtype == MUON_F32;
  a.drows = drows; a.lddr = lddr;
  a.dweights = dweights;
  return done(launch_route(dtype == MUON_BF16, ROUTE_COMBINE_GRAD, a, hipStream_t(hip_stream)), "combine backward");
}

MUON_API muon_status muon_embedding_forward(const void* ids, int32_t id_bytes, const void* w, int64_t ldw, void* y,
                                            int64_t ldy, int64_t rows, int64_t vocab, int64_t cols, float scale,
                                            int32_t dtype, void* hip_stream) {
  TRY(check_count("rows", rows, 0, kMaxRows));
  TRY(check_count("vocab", vocab, 1, kMaxDim));
  TRY(check_count("cols", cols, 1, kMaxDim));
  TRY(check_dtype(dtype));
  if (!std::isfinite(scale)) return fail(MUON_ERR_INVALID_ARG, "scale must be finite");
  TRY(check_ids("ids", ids, id_bytes, rows));
  if (!rows) return done(hipSuccess, "");
  const size_t es = size_of(dtype);
  TRY(check_matrix("w", w, ldw, cols, es));
  TRY(check_matrix("y", y, ldy, cols, es));
  EmbeddingArgs a{};
  a.ids = ids; a.id_bytes = id_bytes;
  a.w = w; a.ldw = ldw;
  a.y = y; a.ldy = ldy;
  a.rows = int32_t(rows); a.cols = int32_t(cols); a.vocab = int32_t(vocab);
  a.scale = scale;
  return done(launch_embedding_forward(dtype == MUON_BF16, a, hipStream_t(hip_stream)), "embedding");
}

MUON_API muon_status muon_embedding_workspace_bytes(int64_t rows, int64_t vocab, int64_t cols,
                                                    size_t* bytes) {
  if (!bytes) return fail(MUON_ERR_INVALID_ARG, "bytes is NULL");
  TRY(check_count("rows", rows, 0, kMaxRows));
  TRY(check_count("vocab", vocab, 1, kMaxDim));
  TRY(check_count("cols", cols, 1, kMaxDim));
  *bytes = embedding_bytes(rows, vocab, cols);
  return done(hipSuccess, "");
}

MUON_API muon_status muon_embedding_backward(const void* dy, int64_t lddy, const void* ids, int32_t id_bytes, void* dw,
                                             int64_t lddw, int64_t rows, int64_t vocab, int64_t cols, float scale,
                                             int32_t dtype, void* workspace, size_t workspace_bytes,
                                             void* hip_stream) {
  TRY(check_count("rows", rows, 0, kMaxRows));
  TRY(check_count("vocab", vocab, 1, kMaxDim));
  TRY(check_count("cols", cols, 1, kMaxDim));
  TRY(check_dtype(dtype));
  if (!std::isfinite(scale)) return fail(MUON_ERR_INVALID_ARG, "scale must be finite");
  TRY(check_ids("ids", ids, id_bytes, rows));
  const size_t es = size_of(dtype);
  if (rows) TRY(check_matrix("dy", dy, lddy, cols, es));
  TRY(check_matrix("dw", dw, lddw, cols, es));
  TRY(check_workspace(workspace, workspace_bytes, embedding_bytes(rows, vocab, cols)));
  EmbeddingArgs a{};
  a.ids = ids; a.id_bytes = id_bytes;
  a.dy = dy; a.lddy = lddy;
  a.dw = dw; a.lddw = lddw;
  a.rows = int32_t(rows); a.cols = int32_t(cols); a.vocab = int32_t(vocab);
  a.scale = scale;
  return done(launch_embedding_backward(dtype == MUON_BF16, a, workspace, hipStream_t(hip_stream)),
              "embedding backward");
}

MUON_API muon_status muon_linear_cross_entropy_workspace_bytes(int64_t rows, int64_t inner, int64_t outer,
                                                               int32_t dtype, int32_t flags, size_t* bytes) {
  if (!bytes) return fail(MUON_ERR_INVALID_ARG, "bytes is NULL");
  TRY(check_loss(rows, inner, outer, dtype, MUON_LOSS_ROWS));
  TRY(check_flags(flags));
  size_t most = 0;
  for (bool transposed : {false, true})
    for (bool unaligned : {false, true}) {
      if (unaligned && !(flags & MUON_LAYERS_UNALIGNED)) continue;
      const auto layout = flags & MUON_LAYERS_BACKWARD ? backward_layout : forward_layout;
      most = larger(most, layout(rows, inner, outer, transposed, dtype == MUON_BF16, unaligned).total);
    }
  *bytes = most;
  return done(hipSuccess, "");
}

MUON_API muon_status muon_linear_cross_entropy_forward(const void* x, int64_t ldx, const void* w, int64_t ldw,
                                                       int32_t w_transposed, const void* targets,
                                                       int32_t target_bytes, int64_t ignore, int32_t reduction,
                                                       float* loss, float* lse, int64_t rows, int64_t inner,
                                                       int64_t outer, int32_t dtype, void* workspace,
                                                       size_t workspace_bytes, void* hip_stream) {
  TRY(check_loss(rows, inner, outer, dtype, reduction));
  TRY(check_ids("targets", targets, target_bytes, rows));
  const size_t es = size_of(dtype);
  const bool bf16 = dtype == MUON_BF16, each = reduction == MUON_LOSS_ROWS;
  if (rows || !each) TRY(check_needed("loss", loss, 4));
  Operand xo{x, ldx};
  const Operand wo{w, ldw};
  bool xf = true, wf = true;
  if (rows) {
    TRY(check_needed("lse", lse, 4));
    TRY(check_matrix("x", x, ldx, inner, es));
    TRY(check_matrix("w", w, ldw, w_transposed ? inner : outer, es));
    xf = x_fits(xo, inner, bf16);
    wf = w_fits(wo, inner, outer, w_transposed, bf16);
  }
  const LossLayout l = forward_layout(rows, inner, outer, w_transposed, bf16, !(xf && wf));
  TRY(check_workspace(workspace, workspace_bytes, l.total));
  const hipStream_t st = hipStream_t(hip_stream);
  char* ws = static_cast<char*>(workspace);
  const int64_t epc = bf16 ? 8 : 4;
  const bool few = l.z.kernel == Choice::SKINNY;
  if (!xf && !few) TRY(done(copy_operand(bf16, xo, copy_shape(rows, inner, epc), ws + l.xcopy, st), "copy of x"));
  LossArgs a{};
  a.targets = targets; a.target_bytes = target_bytes; a.ignore = ignore;
  a.rows = int32_t(rows); a.vocab = int32_t(outer);
  a.logit = reinterpret_cast<float*>(ws + l.logit);
  a.loss = each ? loss : reinterpret_cast<float*>(ws + l.loss);
  a.lse = lse;
  float* const raw = reinterpret_cast<float*>(ws + l.raw);
  const int form = w_transposed ? FORM_RR : FORM_RT;
  for (int64_t r = 0; r < rows; r += l.rows) {
    LossArgs b = a;
    b.targets = static_cast<const char*>(targets) + r * target_bytes;
    b.logit = a.logit + r;
    b.loss = a.loss + r;
    b.lse = a.lse + r;
    b.rows = int32_t(rows - r < l.rows ? rows - r : l.rows);
    b.part = reinterpret_cast<float2*>(ws + l.part);
    b.raw = raw;
    b.splits = l.z.splits;
    for (int64_t c = 0; c < outer; c += l.piece) {
      const int64_t cols = outer - c < l.piece ? outer - c : l.piece;
      Operand wc = columns(wo, w_transposed, c, es);
      if (!wf && !few)
        TRY(done(copy_operand(bf16, wc, copy_of_w(cols, inner, w_transposed, epc), ws + l.wcopy, st), "copy of w"));
      Product p{};
      p.M = b.rows; p.N = int32_t(cols); p.K = int32_t(inner);
      p.a = static_cast<const char*>(xo.p) + size_t(r * xo.ld) * es; p.lda = xo.ld;
      p.b = wc.p; p.ldb = wc.ld;
      b.first = int32_t(c);
      b.cols = p.N;
      if (few) {
        TRY(done(product_sums(l.z, bf16, form, p, raw, st), "logits"));
        TRY(done(launch_loss_strips(b, st), "loss strips"));
      } else {
        TRY(done(loss_product(l.z, LOSS_STRIPS, bf16, form, p, b, nullptr, st), "loss strips"));
      }
      b.strip += int32_t(ceil_div(cols, strip_columns(l.z)));
    }
    b.strips = b.strip;
    TRY(done(launch_loss_finish(b, st), "loss"));
  }
  if (!each) {
    a.total = loss;
    a.mean = reduction == MUON_LOSS_MEAN;
    TRY(done(launch_loss_total(a, st), "loss"));
  }
  return done(hipSuccess, "");
}

MUON_API muon_status muon_linear_cross_entropy_backward(const float* dloss, const void* x, int64_t ldx, const void* w,
                                                        int64_t ldw, int32_t w_transposed, const void* targets,
                                                        int32_t target_bytes, int64_t ignore, int32_t reduction,
                                                        const float* lse, void* dx, int64_t lddx, void* dw,
                                                        int64_t lddw, int64_t rows, int64_t inner, int64_t outer,
                                                        int32_t dtype, void* workspace, size_t workspace_bytes,
                                                        void* hip_stream) {
  TRY(check_loss(rows, inner, outer, dtype, reduction));
  TRY(check_ids("targets", targets, target_bytes, rows));
  const size_t es = size_of(dtype);
  const bool bf16 = dtype == MUON_BF16;
  Operand xo{x, ldx};
  const Operand wo{w, ldw};
  bool xf = true, wf = true;
  if (rows) {
    TRY(check_needed("dloss", dloss, 4));
    TRY(check_needed("lse", lse, 4));
    TRY(check_matrix("x", x, ldx, inner, es));
    TRY(check_matrix("w", w, ldw, w_transposed ? inner : outer, es));
    if (dx) TRY(check_matrix("dx", dx, lddx, inner, es));
    xf = x_fits(xo, inner, bf16);
    wf = w_fits(wo, inner, outer, w_transposed, bf16);
  }
  if (dw) TRY(check_matrix("dw", dw, lddw, w_transposed ? inner : outer, es));
  const LossLayout l = backward_layout(rows, inner, outer, w_transposed, bf16, !(xf && wf));
  TRY(check_workspace(workspace, workspace_bytes, l.total));
  const hipStream_t st = hipStream_t(hip_stream);
  char* ws = static_cast<char*>(workspace);
  const int64_t epc = bf16 ? 8 : 4;
  const bool few = l.z.kernel == Choice::SKINNY;
  LossArgs a{};
  a.targets = targets; a.target_bytes = target_bytes; a.ignore = ignore;
  a.rows = int32_t(rows); a.vocab = int32_t(outer);
  a.dloss = dloss;
  a.each = reduction == MUON_LOSS_ROWS;
  a.lse = const_cast<float*>(lse);
  if (!rows && !dw) return done(hipSuccess, "");
  // (which reads x as it lies)
  const bool outer_product = outer_product_wins(bf16, w_transposed, rows, inner, outer);
  if (rows && ((dw && !outer_product) || (!xf && !few))) {
    const int64_t ld = copy_shape(rows, inner, epc).ld_dst;
    TRY(done(launch_loss_rows(bf16, a, xo.p, xo.ld, ws + l.xcopy, ld, inner, st), "copy of x"));
    xo = Operand{ws + l.xcopy, ld};
  }
  if (reduction == MUON_LOSS_SUM) a.alpha = dloss;
  if (reduction == MUON_LOSS_MEAN && rows) {
    float* const alpha = reinterpret_cast<float*>(ws + l.alpha);
    TRY(done(launch_loss_mean(a, alpha, st), "loss mean"));
    a.alpha = alpha;
  }
  const int64_t lddz = ceil_div(l.piece, 8) * 8;
  float* const raw = reinterpret_cast<float*>(ws + l.raw);
  float* const sums = reinterpret_cast<float*>(ws + l.dx);
  for (int64_t c = 0; c < outer; c += l.piece) {
    const int64_t cols = outer - c < l.piece ? outer - c : l.piece;
    Operand wc = columns(wo, w_transposed, c, es);
    if (!wf && !(few && l.x.kernel == Choice::SKINNY))
      TRY(done(copy_operand(bf16, wc, copy_of_w(cols, inner, w_transposed, epc), ws + l.wcopy, st), "copy of w"));
    for (int64_t r = 0; r < rows; r += l.rows) {
      LossArgs b = a;
      b.rows = int32_t(rows - r < l.rows ? rows - r : l.rows);
      b.targets = static_cast<const char*>(targets) + r * target_bytes;
      b.dloss = a.each ? dloss + r : dloss;
      b.lse = a.lse + r;
      b.raw = raw;
      b.splits = l.z.splits;
      b.dz = ws + l.dz + size_t(r * lddz) * es;
      b.lddz = lddz;
      b.first = int32_t(c);
      b.cols = int32_t(cols);
      Product p{};
      p.M = b.rows; p.N = b.cols; p.K = int32_t(inner);
      p.a = static_cast<const char*>(xo.p) + size_t(r * xo.ld) * es; p.lda = xo.ld;
      p.b = wc.p; p.ldb = wc.ld;
      p.c = b.dz; p.ldc = lddz;
      const int form = w_transposed ? FORM_RR : FORM_RT;
      if (few) {
        TRY(done(product_sums(l.z, bf16, form, p, raw, st), "logits"));
        TRY(done(launch_loss_grad(bf16, b, st), "loss gradient"));
      } else {
        TRY(done(loss_product(l.z, LOSS_GRAD, bf16, form, p, b, nullptr, st), "loss gradient"));
      }
    }
    if (dx && rows) {
      Product p{};
      p.M = int32_t(rows); p.N = int32_t(inner); p.K = int32_t(cols);
      p.a = ws + l.dz; p.lda = lddz;
      p.b = wc.p; p.ldb = wc.ld;
      p.add = c > 0;
      TRY(done(product_sums(l.x, bf16, w_transposed ? FORM_RT : FORM_RR, p, sums, st), "loss input gradient"));
    }
    if (dw && outer_product) {
      LossArgs b = a;
      b.dz = ws + l.dz;
      b.lddz = lddz;
      b.cols = int32_t(cols);
      TRY(done(launch_loss_outer(bf16, !w_transposed, b, xo.p, xo.ld, inner,
                                 const_cast<void*>(columns(Operand{dw, lddw}, w_transposed, c, es).p), lddw, st),
               "loss weight gradient"));
    } else if (dw) {
      Product p{};
      p.K = int32_t(rows);
      p.c = const_cast<void*>(columns(Operand{dw, lddw}, w_transposed, c, es).p); p.ldc = lddw;
      if (w_transposed) {
        p.a = ws + l.dz; p.lda = lddz;
        p.b = xo.p; p.ldb = xo.ld;
        p.M = int32_t(cols); p.N = int32_t(inner);
      } else {
        p.a = xo.p; p.lda = xo.ld;
        p.b = ws + l.dz; p.ldb = lddz;
        p.M = int32_t(inner); p.N = int32_t(cols);
      }
      TRY(done(loss_product(l.w, LOSS_WEIGHT, bf16, FORM_TT, p, a, ws + l.scratch, st), "loss weight gradient"));
    }
  }
  if (dx && rows)
    TRY(done(launch_loss_sum(bf16, a, sums, l.x.splits, dx, lddx, inner, st), "loss input gradient"));
  return done(hipSuccess, "");
}

}  // extern "C"
