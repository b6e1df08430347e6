// Host check of the loss's two passes: tokens_api.cpp with launchers that note
// what they are asked to run instead of running it, and hold what it would read and
// write of the workspace against the workspace's size.
//
// Reads lines "bf16 transposed rows inner outer off reduction" (off: elements by
// which x and w are off 16-byte addresses) and prints, for each, the products of both
// passes as "step/kernel/dtype/form/split" words, or FAILED and the reason.  The
// workspaces have the size the library asks for.
#include "../paper_2606_27153_amd/csrc/layers/tokens_api.cpp"

#include <iostream>
#include <map>
#include <string>
#include <vector>

namespace {
std::string g_words, g_failed;
uintptr_t g_ws, g_end;
// what each buffer of the workspace spans; two of different names must not overlap
std::map<std::string, std::pair<uintptr_t, uintptr_t>> g_spans;

bool in_workspace(const void* p) {
  const uintptr_t a = reinterpret_cast<uintptr_t>(p);
  return a >= g_ws && a < g_ws + (uintptr_t(1) << 44);   // (operands and results lie elsewhere)
}
void span(const std::string& name, const void* p, size_t bytes) {
  const uintptr_t a = reinterpret_cast<uintptr_t>(p), b = a + bytes;
  if (!bytes) return;
  if (a < g_ws || b > g_end) g_failed += " " + name + " is out of the workspace;";
  auto at = g_spans.emplace(name, std::make_pair(a, b)).first;
  at->second.first = std::min(at->second.first, a);
  at->second.second = std::max(at->second.second, b);
  for (const auto& o : g_spans)
    if (o.first != name && at->second.first < o.second.second && o.second.first < at->second.second)
      g_failed += " " + name + " overlaps " + o.first + ";";
}
void maybe(const std::string& name, const void* p, size_t bytes) {
  if (in_workspace(p)) span(name, p, bytes);
}
size_t block(int64_t rows, int64_t ld, int64_t cols, size_t es) { return rows ? ((rows - 1) * ld + cols) * es : 0; }

const char* const kForms[] = {"RT", "RR", "TT"};
std::string word(const std::string& step, const std::string& kernel, bool bf16, int form, int splits) {
  return " " + step + "/" + kernel + (bf16 ? "/bf16/" : "/f32/") + kForms[form] + (splits > 1 ? "/1" : "/0");
}
// what the tile kernels fetch: whole chunks of aligned rows, to the end of the last chunk
void operands(bool bf16, int form, const Product& p, const std::string& a, const std::string& b) {
  const int64_t epc = bf16 ? 8 : 4;
  const size_t es = bf16 ? 2 : 4;
  const int64_t ar = form == FORM_TT ? p.K : p.M, ac = form == FORM_TT ? p.M : p.K;
  const int64_t br = form == FORM_RR ? p.N : p.K, bc = form == FORM_RR ? p.K : p.N;
  auto one = [&](const std::string& name, const void* q, int64_t ld, int64_t rows, int64_t cols) {
    if (!rows) return;
    const int64_t whole = (cols + epc - 1) / epc * epc;
    if (reinterpret_cast<uintptr_t>(q) % 16 || ld % epc) g_failed += " " + name + " is off 16-byte rows;";
    if (whole != cols && !in_workspace(q)) g_failed += " " + name + " is read past its rows' ends;";
    if (ld < whole) g_failed += " " + name + "'s rows overlap;";
    if (ld * int64_t(es) * 256 >= (int64_t(1) << 31)) g_failed += " " + name + " is out of 32-bit offsets;";
    maybe(name, q, block(rows, ld, whole, es));
  };
  one(a, p.a, p.lda, ar, ac);
  one(b, p.b, p.ldb, br, bc);
}
hipError_t raw(const std::string& kernel, bool tile, bool bf16, int form, const Product& p) {
  const bool logits = g_words.rfind("dz") == std::string::npos || !in_workspace(p.a) || g_spans.count("dz") == 0 ||
                      reinterpret_cast<uintptr_t>(p.a) < g_spans["dz"].first ||
                      reinterpret_cast<uintptr_t>(p.a) >= g_spans["dz"].second;
  g_words += word(logits ? "logits" : "dx", kernel, bf16, form, p.splits);
  if (!p.raw) g_failed += " a product that should stay in fp32;";
  if (tile) operands(bf16, form, p, logits ? "xcopy" : "dz", "wcopy");
  span(logits ? "raw" : "sums", p.part, size_t(p.splits) * p.M * p.N * 4);
  return hipSuccess;
}
hipError_t step(const std::string& kernel, int wave_cols, bool bf16, int s, int form, const Product& p,
                const LossArgs& a) {
  static const char* const names[] = {"strips", "dz", "weight"};
  g_words += word(names[s], kernel, bf16, form, p.splits);
  if (s == LOSS_WEIGHT) {
    const bool t = in_workspace(p.a) && g_spans.count("dz") && reinterpret_cast<uintptr_t>(p.a) >= g_spans["dz"].first &&
                   reinterpret_cast<uintptr_t>(p.a) < g_spans["dz"].second;
    operands(bf16, form, p, t ? "dz" : "xcopy", t ? "xcopy" : "dz");
    if (p.splits > 1) span("weight part", p.part, size_t(p.splits) * p.M * p.N * 4);
    return hipSuccess;
  }
  operands(bf16, form, p, "xcopy", "wcopy");
  if (s == LOSS_STRIPS) {
    const int64_t strips = (p.N + wave_cols - 1) / wave_cols;
    span("part", a.part + int64_t(a.strip) * a.rows, size_t(strips) * a.rows * 8);
    span("logit", a.logit, size_t(a.rows) * 4);
  } else {
    if (a.lddz % 8 || reinterpret_cast<uintptr_t>(p.c) % 16) g_failed += " dz is off 16-byte rows;";
    span("dz", p.c, block(p.M, p.ldc, (p.N + 7) / 8 * 8, bf16 ? 2 : 4));
  }
  return hipSuccess;
}
}  // namespace

const char* hipGetErrorString(hipError_t) { return "error"; }

namespace muon {
namespace layers {

size_t expert_sort_bytes(int64_t) { return 0; }
hipError_t launch_expert_sort(const void*, int, int64_t, int, int32_t*, int32_t*, int32_t*, int32_t*, hipStream_t) {
  return hipSuccess;
}
hipError_t launch_route(bool, int, const RouteArgs&, hipStream_t) { return hipSuccess; }
size_t embedding_bytes(int64_t, int64_t, int64_t) { return 0; }
hipError_t launch_embedding_forward(bool, const EmbeddingArgs&, hipStream_t) { return hipSuccess; }
hipError_t launch_embedding_backward(bool, EmbeddingArgs, void*, hipStream_t) { return hipSuccess; }

hipError_t launch_loss_mean(const LossArgs&, float* alpha, hipStream_t) {
  span("alpha", alpha, 4);
  return hipSuccess;
}
hipError_t launch_loss_strips(const LossArgs& a, hipStream_t) {
  span("raw", a.raw, size_t(a.splits) * a.rows * a.cols * 4);
  span("part", a.part + int64_t(a.strip) * a.rows, size_t((a.cols + kRawStrip - 1) / kRawStrip) * a.rows * 8);
  span("logit", a.logit, size_t(a.rows) * 4);
  return hipSuccess;
}
hipError_t launch_loss_finish(const LossArgs& a, hipStream_t) {
  span("part", a.part, size_t(a.strips) * a.rows * 8);
  maybe("loss", a.loss, size_t(a.rows) * 4);
  return hipSuccess;
}
hipError_t launch_loss_total(const LossArgs& a, hipStream_t) {
  span("loss", a.loss, size_t(a.rows) * 4);
  return hipSuccess;
}
hipError_t launch_loss_grad(bool bf16, const LossArgs& a, hipStream_t) {
  span("raw", a.raw, size_t(a.splits) * a.rows * a.cols * 4);
  span("dz", a.dz, block(a.rows, a.lddz, (a.cols + 7) / 8 * 8, bf16 ? 2 : 4));
  g_words += std::string(" dz/rows/") + (bf16 ? "bf16" : "f32");
  return hipSuccess;
}
hipError_t launch_loss_rows(bool bf16, const LossArgs& a, const void*, int64_t, void* y, int64_t ldy, int64_t cols,
                            hipStream_t) {
  if (ldy < cols) g_failed += " xcopy's rows overlap;";
  span("xcopy", y, size_t(a.rows) * ldy * (bf16 ? 2 : 4));
  return hipSuccess;
}
hipError_t launch_loss_outer(bool bf16, bool x_down, const LossArgs& a, const void*, int64_t ldx, int64_t inner, void*,
                             int64_t ldo, hipStream_t) {
  span("dz", a.dz, block(a.rows, a.lddz, a.cols, bf16 ? 2 : 4));
  if (a.rows > outer_rows(bf16)) g_failed += " too many rows;";
  if (ldx < inner || ldo < (x_down ? a.cols : inner)) g_failed += " rows overlap;";
  g_words += std::string(" weight/outer/") + (bf16 ? "bf16" : "f32");
  return hipSuccess;
}
hipError_t launch_loss_sum(bool, const LossArgs& a, const float* part, int splits, void*, int64_t, int64_t cols,
                           hipStream_t) {
  span("sums", part, size_t(splits) * a.rows * cols * 4);
  return hipSuccess;
}
hipError_t launch_simple(bool, int, int, const Product&, const Table*, hipStream_t) { return hipErrorInvalidValue; }
hipError_t launch_reduce(bool, const Product& p, hipStream_t) {
  span("weight part", p.part, size_t(p.splits) * p.M * p.N * 4);
  return hipSuccess;
}
hipError_t launch_pack(bool bf16, const PackArgs& a, const Table&, hipStream_t) {
  const bool x = reinterpret_cast<uintptr_t>(a.a.src) < (uintptr_t(1) << 41);
  span(x ? "xcopy" : "wcopy", a.a.dst, size_t(a.a.rows) * a.a.ld_dst * (bf16 ? 2 : 4));
  return hipSuccess;
}
hipError_t launch_skinny(bool bf16, int form, int, int mt, const Product& p, const Table*, hipStream_t) {
  if (p.N < (bf16 ? 8 : 4)) g_failed += " too few columns;";
  return raw("skinny" + std::to_string(16 * mt), false, bf16, form, p);
}
#define TILE(name, kernel, bf16)                                                                   \
  hipError_t launch_tile##name(int form, int, const Product& p, const Table*, hipStream_t) {        \
    return raw(kernel, true, bf16, form, p);                                                       \
  }
TILE(256_bf16, "tile256", true)
TILE(128x256_bf16, "tile128x256", true)
TILE(128_bf16, "tile128", true)
TILE(128_f32, "tile128", false)
TILE(64_bf16, "tile64", true)
TILE(64_f32, "tile64", false)
#define LOSS(name, kernel, bf16, cols)                                                             \
  hipError_t launch_loss##name(int s, int form, const Product& p, const LossArgs& a, hipStream_t) { \
    return step(kernel, cols, bf16, s, form, p, a);                                                \
  }
LOSS(256_bf16, "tile256", true, 128)
LOSS(128x256_bf16, "tile128x256", true, 128)
LOSS(128_bf16, "tile128", true, 64)
LOSS(128_f32, "tile128", false, 64)
LOSS(64_bf16, "tile64", true, 32)
LOSS(64_f32, "tile64", false, 32)

}  // namespace layers
}  // namespace muon

int main() {
  int32_t bf16, t, off, reduction;
  int64_t rows, inner, outer;
  while (std::cin >> bf16 >> t >> rows >> inner >> outer >> off >> reduction) {
    const int32_t dt = bf16 ? MUON_BF16 : MUON_F32;
    const size_t es = bf16 ? 2 : 4;
    // addresses that are checked, never read: x, the weight, results, the workspace, far apart
    void* const x = reinterpret_cast<void*>((uintptr_t(1) << 40) + off * es);
    void* const w = reinterpret_cast<void*>((uintptr_t(1) << 41) + off * es);
    void* const out = reinterpret_cast<void*>(uintptr_t(1) << 42);
    g_ws = uintptr_t(1) << 45;
    const int64_t ldw = t ? inner : outer;
    const bool far = std::max(inner, ldw) * int64_t(es) >= (int64_t(1) << 23);
    const int flag = far || (inner * es | outer * es | off * es) % 16 ? MUON_LAYERS_UNALIGNED : 0;
    g_words.clear();
    g_failed.clear();
    for (int back = 0; back < 2 && g_failed.empty(); ++back) {
      size_t bytes = 0;
      g_spans.clear();
      muon_status s = muon_linear_cross_entropy_workspace_bytes(rows, inner, outer, dt, flag | back, &bytes);
      g_end = g_ws + bytes;
      void* const ws = reinterpret_cast<void*>(g_ws);
      if (s == MUON_OK && !back)
        s = muon_linear_cross_entropy_forward(x, inner, w, ldw, t, out, 8, -100, reduction, static_cast<float*>(out),
                                              static_cast<float*>(out), rows, inner, outer, dt, ws, bytes, nullptr);
      if (s == MUON_OK && back)
        s = muon_linear_cross_entropy_backward(static_cast<float*>(out), x, inner, w, ldw, t, out, 8, -100, reduction,
                                               static_cast<float*>(out), out, inner, out, ldw, rows, inner, outer, dt,
                                               ws, bytes, nullptr);
      if (s != MUON_OK) g_failed += std::string(" ") + muon::layers::g_error;
    }
    std::cout << (g_failed.empty() ? g_words : "FAILED" + g_failed) << "\n";
  }
}
