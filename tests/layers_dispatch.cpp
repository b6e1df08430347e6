// Host check of the layer operators' choice of kernel: layers_api.cpp with
// launchers that note what they are asked to run instead of running it.
//
// Reads lines "op bf16 transposed rows inner outer experts act" (op l: both
// passes of the linear operator, op g: of the grouped one; experts is 0 for l)
// and prints, for each, the launches of the two passes:
// "kernel/dtype/form/group/split" words, the split being 1 if the summed
// dimension is cut.  Workspaces have the size the library asks for, with room
// for copies; operands are aligned.
#include "../paper_2606_27153_amd/csrc/layers/layers_api.cpp"

#include <iostream>
#include <string>
#include <vector>

namespace {
std::string g_words;

hipError_t note(const std::string& kernel, bool bf16, int form, int group, const muon::layers::Product& p) {
  static const char* const forms[] = {"RT", "RR", "TT"};
  static const char* const groups[] = {"plain", "rows", "sum"};
  g_words += " " + kernel + (bf16 ? "/bf16/" : "/f32/") + forms[form] + "/" + groups[group] +
             (p.splits > 1 ? "/1" : "/0");
  return hipSuccess;
}
}  // namespace

const char* hipGetErrorString(hipError_t) { return "error"; }

namespace muon {
namespace layers {

hipError_t launch_simple(bool bf16, int form, int group, const Product& p, const Table*, hipStream_t) {
  return note("simple", bf16, form, group, p);
}
hipError_t launch_tile256_bf16(int form, int group, const Product& p, const Table*, hipStream_t) {
  return note("tile256", true, form, group, p);
}
hipError_t launch_tile128x256_bf16(int form, int group, const Product& p, const Table*, hipStream_t) {
  return note("tile128x256", true, form, group, p);
}
hipError_t launch_tile128_bf16(int form, int group, const Product& p, const Table*, hipStream_t) {
  return note("tile128", true, form, group, p);
}
hipError_t launch_tile128_f32(int form, int group, const Product& p, const Table*, hipStream_t) {
  return note("tile128", false, form, group, p);
}
hipError_t launch_tile64_bf16(int form, int group, const Product& p, const Table*, hipStream_t) {
  return note("tile64", true, form, group, p);
}
hipError_t launch_tile64_f32(int form, int group, const Product& p, const Table*, hipStream_t) {
  return note("tile64", false, form, group, p);
}
hipError_t launch_skinny(bool bf16, int form, int group, int mt, const Product& p, const Table*, hipStream_t) {
  return note("skinny" + std::to_string(16 * mt), bf16, form, group, p);
}
hipError_t launch_reduce(bool, const Product&, hipStream_t) { return hipSuccess; }
hipError_t launch_pack(bool, const PackArgs&, const Table&, hipStream_t) { return hipSuccess; }
hipError_t launch_act_grad(bool, const ActGradArgs&, hipStream_t) { return hipSuccess; }
int act_grad_chunks(int64_t, int64_t) { return 1; }
hipError_t launch_norm_forward(bool, const NormArgs&, hipStream_t) { return hipSuccess; }
hipError_t launch_norm_backward(bool, const NormArgs&, hipStream_t) { return hipSuccess; }
int norm_blocks(int64_t, int64_t) { return 1; }

}  // namespace layers
}  // namespace muon

int main() {
  void* const at = reinterpret_cast<void*>(uintptr_t(1) << 20);   // addresses that are checked, never read
  void* const ws = reinterpret_cast<void*>(uintptr_t(1) << 24);
  const int32_t* const off = static_cast<const int32_t*>(at);
  const std::vector<void*> table(MUON_GROUPED_MAX_EXPERTS, at);
  std::string op;
  int32_t bf16, t, experts, act;
  int64_t rows, inner, outer;
  while (std::cin >> op >> bf16 >> t >> rows >> inner >> outer >> experts >> act) {
    const int32_t dt = bf16 ? MUON_BF16 : MUON_F32;
    const int64_t ldw = t ? inner : outer;
    size_t f = 0, b = 0;
    muon_status s[4] = {};
    g_words.clear();
    if (op == "l") {
      s[0] = muon_linear_workspace_bytes(rows, inner, outer, dt, act, MUON_LAYERS_UNALIGNED, &f);
      s[1] = muon_linear_workspace_bytes(rows, inner, outer, dt, act, MUON_LAYERS_UNALIGNED | MUON_LAYERS_BACKWARD, &b);
      s[2] = muon_linear_forward(at, inner, at, ldw, t, nullptr, nullptr, 0, at, outer, nullptr, 0, rows, inner, outer,
                                 dt, act, ws, f, nullptr);
      s[3] = muon_linear_backward(at, outer, at, inner, at, ldw, t, at, outer, at, inner, at, ldw, at, rows, inner,
                                  outer, dt, act, ws, b, nullptr);
    } else {
      s[0] = muon_grouped_linear_workspace_bytes(rows, inner, outer, experts, dt, MUON_LAYERS_UNALIGNED, &f);
      s[1] = muon_grouped_linear_workspace_bytes(rows, inner, outer, experts, dt,
                                                 MUON_LAYERS_UNALIGNED | MUON_LAYERS_BACKWARD, &b);
      s[2] = muon_grouped_linear_forward(at, inner, table.data(), ldw, t, off, experts, at, outer, rows, inner, outer,
                                         dt, ws, f, nullptr);
      s[3] = muon_grouped_linear_backward(at, outer, at, inner, table.data(), ldw, t, off, experts, at, inner,
                                          table.data(), ldw, rows, inner, outer, dt, ws, b, nullptr);
    }
    for (const muon_status v : s)
      if (v != MUON_OK) {
        std::cout << "FAILED " << muon_layers_last_error() << "\n";
        return 1;
      }
    std::cout << g_words << "\n";
  }
  return 0;
}
