// Host side that the layer operators share: argument checks, the choice of a
// matrix product's kernel, and its launch.
#ifndef MUON_LAYERS_HOST_H
#define MUON_LAYERS_HOST_H

#include <cmath>
#include <cstdarg>
#include <cstdio>

#include "layers.h"

namespace muon {
namespace layers {

inline thread_local char g_error[256];   // one for the library

inline muon_status fail(muon_status s, const char* fmt, ...) {
  va_list ap;
  va_start(ap, fmt);
  std::vsnprintf(g_error, sizeof(g_error), fmt, ap);
  va_end(ap);
  return s;
}

inline muon_status done(hipError_t e, const char* what) {
  if (e == hipErrorInvalidConfiguration) return fail(MUON_ERR_UNSUPPORTED, "%s: more tiles than one grid holds", what);
  if (e != hipSuccess) return fail(MUON_ERR_DEVICE, "%s: %s", what, hipGetErrorString(e));
  g_error[0] = 0;
  return MUON_OK;
}

inline constexpr int64_t kMaxRows = int64_t(1) << 30, kMaxDim = int64_t(1) << 24;
inline constexpr int64_t kMaxLd = int64_t(1) << 40;

inline bool known_dtype(int32_t d) { return d == MUON_F32 || d == MUON_BF16; }
inline size_t size_of(int32_t dtype) { return dtype == MUON_BF16 ? 2 : 4; }
inline size_t padded(size_t v) { return (v + 255) / 256 * 256; }

inline muon_status check_sizes(int64_t rows, int64_t inner, int64_t outer, int32_t dtype) {
  if (rows < 0 || rows > kMaxRows) return fail(MUON_ERR_INVALID_ARG, "rows %lld out of [0, 2^30]", (long long)rows);
  if (inner < 1 || inner > kMaxDim)
    return fail(MUON_ERR_INVALID_ARG, "inner %lld out of [1, 2^24]", (long long)inner);
  if (outer < 1 || outer > kMaxDim)
    return fail(MUON_ERR_INVALID_ARG, "outer %lld out of [1, 2^24]", (long long)outer);
  if (!known_dtype(dtype)) return fail(MUON_ERR_UNSUPPORTED, "dtype %d: MUON_F32 or MUON_BF16", dtype);
  return MUON_OK;
}

inline muon_status check_activation(int32_t a) {
  if (a < MUON_ACT_NONE || a > MUON_ACT_SILU) return fail(MUON_ERR_INVALID_ARG, "unknown activation %d", a);
  return MUON_OK;
}

inline muon_status check_flags(int32_t f) {
  if (f & ~(MUON_LAYERS_BACKWARD | MUON_LAYERS_UNALIGNED)) return fail(MUON_ERR_INVALID_ARG, "unknown flags %d", f);
  return MUON_OK;
}

// A matrix operand: a pointer aligned to its element and a leading dimension of
// at least its columns.
inline muon_status check_matrix(const char* name, const void* p, int64_t ld, int64_t cols, size_t esize) {
  if (!p) return fail(MUON_ERR_INVALID_ARG, "%s is NULL", name);
  if (reinterpret_cast<uintptr_t>(p) % esize)
    return fail(MUON_ERR_INVALID_ARG, "%s is not aligned to its element", name);
  if (ld < cols || ld > kMaxLd)
    return fail(MUON_ERR_INVALID_ARG, "%s has leading dimension %lld, needs at least %lld", name, (long long)ld,
                (long long)cols);
  return MUON_OK;
}

inline muon_status check_vector(const char* name, const void* p, size_t esize) {
  if (reinterpret_cast<uintptr_t>(p) % esize)
    return fail(MUON_ERR_INVALID_ARG, "%s is not aligned to its element", name);
  return MUON_OK;
}

inline muon_status check_workspace(const void* ws, size_t have, size_t need) {
  // (more than the need may be used: for copies)
  if (have && reinterpret_cast<uintptr_t>(ws) % 256)
    return fail(MUON_ERR_INVALID_ARG, "workspace must be 256-byte aligned");
  if (!need) return MUON_OK;
  if (!ws) return fail(MUON_ERR_INVALID_ARG, "workspace is NULL, %zu bytes are needed", need);
  if (reinterpret_cast<uintptr_t>(ws) % 256) return fail(MUON_ERR_INVALID_ARG, "workspace must be 256-byte aligned");
  if (have < need) return fail(MUON_ERR_WORKSPACE_TOO_SMALL, "workspace has %zu bytes, %zu are needed", have, need);
  return MUON_OK;
}

inline muon_status check_experts(int32_t experts, const int32_t* offsets) {
  if (experts < 1 || experts > MUON_GROUPED_MAX_EXPERTS)
    return fail(MUON_ERR_INVALID_ARG, "experts %d out of [1, %d]", experts, MUON_GROUPED_MAX_EXPERTS);
  if (!offsets || reinterpret_cast<uintptr_t>(offsets) % 4)
    return fail(MUON_ERR_INVALID_ARG, "offsets is NULL or not 4-byte aligned");
  return MUON_OK;
}

#define TRY(call)                              \
  do {                                         \
    const muon_status try_st = (call);         \
    if (try_st != MUON_OK) return try_st;      \
  } while (0)

inline bool aligned16(const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }

// Whether the tile kernels can fetch an operand of rows of `cols` elements:
// 16-byte chunks that lie on 16-byte addresses and do not straddle the end of a
// row, and 32-bit byte offsets within a tile of 256 rows.
inline bool rows_fit(const void* ptr, int64_t ld, int64_t cols, int64_t epc) {
  return aligned16(ptr) && ld % epc == 0 && cols % epc == 0 && ld * 16 / epc * 256 < (int64_t(1) << 31);
}
struct Fits {
  bool a, b;
};
inline Fits tile_fits(bool bf16, int form, int group, const Product& p, const Table* t) {
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
inline PackOne copy_shape(int64_t rows, int64_t cols, int64_t epc) {
  PackOne o{};
  o.rows = rows;
  o.cols = cols;
  o.ld_dst = (cols + epc - 1) / epc * epc;
  return o;
}
inline PackOne copy_of_a(int form, int64_t M, int64_t K, int64_t epc) {
  return form == FORM_TT ? copy_shape(K, M, epc) : copy_shape(M, K, epc);
}
inline PackOne copy_of_b(int form, int64_t N, int64_t K, int64_t epc) {
  return form == FORM_RR ? copy_shape(N, K, epc) : copy_shape(K, N, epc);
}
inline size_t copy_bytes(const PackOne& o, int64_t epc, int64_t copies) {
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

inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

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
inline constexpr TileKind kBf16Tiles[] = {{Choice::TILE256, 256, 256, 1.55, 1.1, 7, 5, 1},
                                          {Choice::TILE128X256, 128, 256, 0.9, 0.66, 5, 3, 1},
                                          {Choice::TILE128, 128, 128, 0.95, 0.53, 5, 3.5, 2},
                                          {Choice::TILE64, 64, 64, 0.4, 0.29, 3, 1, 2}};
inline constexpr TileKind kF32Tiles[] = {{Choice::TILE128, 128, 128, 4.0, 2.05, 4.5, 0, 2},
                                         {Choice::TILE64, 64, 64, 1.08, 0.57, 3.5, 0, 2}};

inline double tile_us(const TileKind& k, double blocks, double slabs, bool act) {
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
inline double reduce_us(int64_t M, int64_t N, int splits) {
  return splits > 1 ? 3.0 + double(splits) * M * N * 8 / 4e6 : 0.0;
}

// The tile kernel whose expected time is least, with the sum cut into `most` ranges at most.
inline Choice choose_tile(bool bf16, int group, int64_t M, int64_t N, int64_t K, int64_t experts, bool act,
                          int most = 16) {
  const int64_t bk = bf16 ? 64 : 32;
  Choice c;
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
    for (int s = 1; s <= most; ++s) {
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

inline Choice choose(bool bf16, int form, int group, int64_t M, int64_t N, int64_t K, int64_t experts,
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
  return choose_tile(bf16, group, M, N, K, experts, act);
}

inline size_t part_bytes(const Choice& c, int64_t M, int64_t N) {
  return c.splits > 1 ? padded(size_t(c.splits) * size_t(M) * size_t(N) * 4) : 0;
}

// Scratch memory of a product, and what it can use: partial results, and copies
// of operands the tile kernels cannot fetch.
struct Scratch {
  char* p;
  size_t bytes;
};

// Makes the operands of a product such that its kernel can fetch them: those off
// 16-byte rows are copied if the scratch memory (after the partial results) holds
// the copies; else the simple kernel takes them as they lie.  `copies`: room for the
// table of copied experts.
inline hipError_t fit_operands(bool bf16, int form, int group, Product& p, const Table*& t, Table& copies, Choice& c,
                               Scratch ws, hipStream_t st) {
  if (c.kernel == Choice::SKINNY) return hipSuccess;
  const int64_t epc = bf16 ? 8 : 4;
  const Fits f = tile_fits(bf16, form, group, p, t);
  if (f.a && f.b) return hipSuccess;
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
    const hipError_t e = launch_pack(bf16, k, group == GROUP_ROWS ? *t : none, st);
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
  return hipSuccess;
}

// The chosen kernel of a plain product or of one grouped by expert.
inline hipError_t launch_choice(bool bf16, int form, int group, const Choice& c, const Product& p, const Table* t,
                                hipStream_t st) {
  switch (c.kernel) {
    case Choice::SIMPLE: return launch_simple(bf16, form, group, p, t, st);
    case Choice::SKINNY: return launch_skinny(bf16, form, group, c.mt, p, t, st);
    case Choice::TILE64:
      return bf16 ? launch_tile64_bf16(form, group, p, t, st) : launch_tile64_f32(form, group, p, t, st);
    case Choice::TILE128:
      return bf16 ? launch_tile128_bf16(form, group, p, t, st) : launch_tile128_f32(form, group, p, t, st);
    case Choice::TILE128X256: return launch_tile128x256_bf16(form, group, p, t, st);
    case Choice::TILE256: return launch_tile256_bf16(form, group, p, t, st);
  }
  return hipErrorInvalidValue;
}

// One matrix product: the kernel that suits it.
inline hipError_t product(bool bf16, int form, int group, Product p, const Table* t, Scratch ws, hipStream_t st) {
  Choice c = choose(bf16, form, group, p.M, p.N, p.K, p.experts, p.act != MUON_ACT_NONE);
  Table copies;
  hipError_t e = fit_operands(bf16, form, group, p, t, copies, c, ws, st);
  if (e != hipSuccess) return e;
  p.splits = c.splits;
  p.part = reinterpret_cast<float*>(ws.p);
  e = launch_choice(bf16, form, group, c, p, t, st);
  return e == hipSuccess && c.splits > 1 ? launch_reduce(bf16, p, st) : e;
}

}  // namespace layers
}  // namespace muon

#endif  // MUON_LAYERS_HOST_H
