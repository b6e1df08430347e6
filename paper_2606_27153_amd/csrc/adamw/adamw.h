// Shared declarations of the AdamW step.
#ifndef MUON_ADAMW_H
#define MUON_ADAMW_H

#include <hip/hip_runtime.h>

#include <cstddef>
#include <cstdint>

#include "muon_adamw.h"

namespace muon {
namespace adamw {

constexpr int kBlock = MUON_ADAMW_BLOCK;
constexpr int kChunk = 4096;     // elements of a workgroup
constexpr int kTensors = 56;     // of a launch: its arguments stay under 4 KB

struct Tensor {
  void* p;
  const void* g;
  void* m;
  void* v;
  int16_t* bases;
  int64_t n;
  uint32_t key;       // of the rounding
  int32_t first;      // its first workgroup
  float step;         // lr / (1 - beta1^k)
  float scale;        // 1 / sqrt(1 - beta2^k)
};

struct Args {
  float keep;             // 1 - lr decay
  float b1, c1, b2, c2;   // c = 1 - b
  float eps;
  int32_t count;
  Tensor t[kTensors];
};
static_assert(sizeof(Args) <= 4096, "kernel arguments");

// Integer hash of 32 bits: two rounds of a multiplication by an odd constant
// (fractional bits of sqrt 2 and sqrt 3) between shifts that bring the upper bits
// down.  Flipping one bit of x flips each bit of the result with a probability of 0.5 +- 0.004.
__host__ __device__ inline uint32_t mix(uint32_t x) {
  x ^= x >> 16;
  x *= 0x6A09E667u;
  x ^= x >> 15;
  x *= 0xBB67AE85u;
  return x ^ (x >> 16);
}

hipError_t launch_step(bool param_bf16, bool grad_bf16, int bits, const Args& a, int64_t blocks, hipStream_t st);
hipError_t launch_values(const uint8_t* m, const uint8_t* v, const int16_t* bases, int64_t n, void* mo, void* vo,
                         hipStream_t st);

}  // namespace adamw
}  // namespace muon

#endif  // MUON_ADAMW_H
