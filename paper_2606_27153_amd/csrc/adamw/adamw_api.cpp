// C ABI of the AdamW step: argument checks, and tensors gathered into launches.
#include <cmath>
#include <cstdarg>
#include <cstdio>

#include "adamw.h"

namespace {

using namespace muon::adamw;

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

#define TRY(call)                         \
  do {                                    \
    const muon_status try_st = (call);    \
    if (try_st != MUON_OK) return try_st; \
  } while (0)

constexpr int64_t kMaxElements = int64_t(1) << 35;
constexpr int64_t kMaxBlocks = (int64_t(1) << 24) - 1;   // of 256 threads that one grid holds

muon_status check_pointer(const char* name, int32_t i, const void* p, size_t align) {
  if (!p) return fail(MUON_ERR_INVALID_ARG, "tensor %d: %s is NULL", i, name);
  if (reinterpret_cast<uintptr_t>(p) % align)
    return fail(MUON_ERR_INVALID_ARG, "tensor %d: %s is not aligned to its element", i, name);
  return MUON_OK;
}

size_t size_of(int32_t dtype) { return dtype == MUON_BF16 ? 2 : 4; }
bool known(int32_t dtype) { return dtype == MUON_F32 || dtype == MUON_BF16; }

muon_status check_tensor(const muon_adamw_tensor& t, int32_t i, int32_t bits) {
  if (t.n < 0 || t.n > kMaxElements)
    return fail(MUON_ERR_INVALID_ARG, "tensor %d: n %lld out of [0, 2^35]", i, (long long)t.n);
  if (!known(t.param_dtype) || !known(t.grad_dtype))
    return fail(MUON_ERR_UNSUPPORTED, "tensor %d: dtypes %d and %d: MUON_F32 or MUON_BF16", i, t.param_dtype,
                t.grad_dtype);
  if (!t.grad || !t.n) return MUON_OK;
  if (t.step < 1) return fail(MUON_ERR_INVALID_ARG, "tensor %d: step %lld, counted from 1", i, (long long)t.step);
  TRY(check_pointer("param", i, t.param, size_of(t.param_dtype)));
  TRY(check_pointer("grad", i, t.grad, size_of(t.grad_dtype)));
  TRY(check_pointer("exp_avg", i, t.exp_avg, bits / 8));
  TRY(check_pointer("exp_avg_sq", i, t.exp_avg_sq, bits / 8));
  return bits == 8 ? check_pointer("bases", i, t.bases, 2) : MUON_OK;
}

muon_status check_opts(const muon_adamw_opts* o) {
  if (!o) return fail(MUON_ERR_INVALID_ARG, "opts is NULL");
  if (o->state_bits != 32 && o->state_bits != 8)
    return fail(MUON_ERR_UNSUPPORTED, "state_bits %d: 32 or 8", o->state_bits);
  const struct {
    const char* name;
    double v, most;
  } ranges[] = {{"lr", o->lr, 3e38}, {"beta1", o->beta1, 1}, {"beta2", o->beta2, 1}, {"eps", o->eps, 3e38}};
  for (const auto& r : ranges)
    if (!(r.v >= 0 && r.v <= r.most) || ((r.v == 1) && r.most == 1))
      return fail(MUON_ERR_INVALID_ARG, "%s %g out of range", r.name, r.v);
  if (!(o->weight_decay >= 0 && std::isfinite(o->lr * o->weight_decay)))
    return fail(MUON_ERR_INVALID_ARG, "weight_decay %g out of range", o->weight_decay);
  return MUON_OK;
}

}  // namespace

extern "C" {

MUON_API const char* muon_adamw_last_error(void) { return g_error; }

MUON_API muon_status muon_adamw_step(const muon_adamw_tensor* tensors, int32_t count, const muon_adamw_opts* opts,
                                     void* hip_stream) {
  TRY(check_opts(opts));
  if (count < 0) return fail(MUON_ERR_INVALID_ARG, "count %d is negative", count);
  if (count && !tensors) return fail(MUON_ERR_INVALID_ARG, "tensors is NULL");
  for (int32_t i = 0; i < count; ++i) TRY(check_tensor(tensors[i], i, opts->state_bits));
  Args a;
  a.keep = float(1 - opts->lr * opts->weight_decay);
  a.b1 = float(opts->beta1);
  a.c1 = float(1 - opts->beta1);
  a.b2 = float(opts->beta2);
  a.c2 = float(1 - opts->beta2);
  a.eps = float(opts->eps);
  // the tensors of each pair of types, in order, as many to a launch as fit
  for (int pair = 0; pair < 4; ++pair) {
    const bool pb = pair & 1, gb = pair & 2;
    int64_t blocks = 0;
    a.count = 0;
    auto flush = [&]() {
      const hipError_t e =
          a.count ? launch_step(pb, gb, opts->state_bits, a, blocks, hipStream_t(hip_stream)) : hipSuccess;
      a.count = 0;
      blocks = 0;
      return done(e, "adamw step");
    };
    for (int32_t i = 0; i < count; ++i) {
      const muon_adamw_tensor& t = tensors[i];
      if ((t.param_dtype == MUON_BF16) != pb || (t.grad_dtype == MUON_BF16) != gb || !t.grad || !t.n) continue;
      const int64_t need = (t.n + kChunk - 1) / kChunk;
      if (a.count == kTensors || blocks + need > kMaxBlocks) TRY(flush());
      Tensor& to = a.t[a.count++];
      to.p = t.param;
      to.g = t.grad;
      to.m = t.exp_avg;
      to.v = t.exp_avg_sq;
      to.bases = t.bases;
      to.n = t.n;
      to.first = int32_t(blocks);
      to.key = mix(mix(opts->seed + uint32_t(t.step) * 0x9E3779B9u) + uint32_t(i));
      to.step = float(opts->lr / (1 - std::pow(opts->beta1, double(t.step))));
      to.scale = float(1 / std::sqrt(1 - std::pow(opts->beta2, double(t.step))));
      blocks += need;
    }
    TRY(flush());
  }
  return done(hipSuccess, "");
}

MUON_API muon_status muon_adamw_state_values(const void* exp_avg, const void* exp_avg_sq, const int16_t* bases,
                                             int64_t n, void* exp_avg_out, void* exp_avg_sq_out, void* hip_stream) {
  if (n < 0 || n > kMaxElements) return fail(MUON_ERR_INVALID_ARG, "n %lld out of [0, 2^35]", (long long)n);
  if (!n || (!exp_avg_out && !exp_avg_sq_out)) return done(hipSuccess, "");
  TRY(check_pointer("bases", 0, bases, 2));
  if (exp_avg_out) {
    TRY(check_pointer("exp_avg", 0, exp_avg, 1));
    TRY(check_pointer("exp_avg_out", 0, exp_avg_out, 2));
  }
  if (exp_avg_sq_out) {
    TRY(check_pointer("exp_avg_sq", 0, exp_avg_sq, 1));
    TRY(check_pointer("exp_avg_sq_out", 0, exp_avg_sq_out, 2));
  }
  return done(launch_values(static_cast<const uint8_t*>(exp_avg), static_cast<const uint8_t*>(exp_avg_sq), bases, n,
                            exp_avg_out, exp_avg_sq_out, hipStream_t(hip_stream)),
              "adamw state values");
}

}  // extern "C"
