// Copies of operands that the tile kernels cannot fetch -- rows off 16-byte
// addresses, or that end inside a 16-byte chunk -- to rows of whole chunks, the
// last one filled with zeros.
//
// One launch copies both operands of a product (and every expert's).  A thread
// moves a chunk: 16 bytes from any alignment, or element by element at a row's
// end.  Memory bound: 16384 x 4001 (the weight 4001 x 4096 lies on whole chunks)
// 52 us, 5.0 TB/s, ahead of a product of 430 to 490 us.
#include "device.h"

namespace muon {
namespace layers {
namespace {

template <typename E>
struct __attribute__((packed, aligned(sizeof(E)))) Chunk {
  E v[16 / sizeof(E)];
};

template <typename E>
__global__ __launch_bounds__(256) void pack_kernel(PackArgs a, Table t) {
  constexpr int V = 16 / int(sizeof(E));
  // blockIdx.y: A, then B (every expert's)
  const bool first = a.a.src && blockIdx.y == 0;
  const PackOne o = first ? a.a : a.b;
  const int e = int(blockIdx.y) - (a.a.src ? 1 : 0);
  const E* src = static_cast<const E*>(first || !a.experts ? o.src : t.p[e]);
  E* dst = static_cast<E*>(o.dst) + (first ? 0 : int64_t(e) * o.rows * o.ld_dst);
  const int64_t cpr = o.ld_dst / V, n = o.rows * cpr;
  for (int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x; i < n; i += int64_t(gridDim.x) * 256) {
    const int64_t r = i / cpr, c = i % cpr * V;
    const E* p = src + r * o.ld_src + c;
    Chunk<E> x;
    if (c + V <= o.cols) {
      x = *reinterpret_cast<const Chunk<E>*>(p);
    } else {
#pragma unroll
      for (int k = 0; k < V; ++k) x.v[k] = c + k < o.cols ? p[k] : E(0.f);
    }
    *reinterpret_cast<Chunk<E>*>(dst + r * o.ld_dst + c) = x;
  }
}

}  // namespace

hipError_t launch_pack(bool bf16, const PackArgs& a, const Table& t, hipStream_t st) {
  const int64_t V = bf16 ? 8 : 4;
  int64_t n = 0;
  for (const PackOne* o : {&a.a, &a.b}) {
    const int64_t c = o->dst ? o->rows * (o->ld_dst / V) : 0;
    n = c > n ? c : n;
  }
  if (!n) return hipSuccess;
  const unsigned y = (a.a.src ? 1u : 0u) + (a.b.dst ? unsigned(a.experts ? a.experts : 1) : 0u);
  int64_t x = (n + 255) / 256;
  const int64_t most = 8 * kCUs;
  if (x > most) x = most;
  const dim3 g{unsigned(x), y}, b{256};
  if (bf16)
    hipLaunchKernelGGL((pack_kernel<__bf16>), g, b, 0, st, a, t);
  else
    hipLaunchKernelGGL((pack_kernel<float>), g, b, 0, st, a, t);
  return hipGetLastError();
}

}  // namespace layers
}  // namespace muon
