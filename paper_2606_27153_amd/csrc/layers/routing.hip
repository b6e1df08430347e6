// Tokens to their experts and back: the choices of an MoE router sorted by expert,
// every token's row copied to its experts' rows, the experts' outputs weighted and
// added up, and the gradients of both.
//
//   position[t, j]  row of token t's j-th choice, -1 if it chose no expert
//   rows[position[t, j]] = x[t]                  dx[t] = sum_j drows[position[t, j]]
//   y[t] = r[t] + sum_j w[t, j] rows[position[t, j]]
//   drows[position[t, j]] = w[t, j] dy[t],  dw[t, j] = <dy[t], rows[position[t, j]]>
//
// Every pass goes by token: what a token has is read once, what its choices have is
// read or written in whole rows wherever they lie, so that each byte moves once.
// A thread has 8 columns (16 bytes of bf16) of a token and goes over its choices.
#include "sort.h"

namespace muon {
namespace layers {
namespace {

struct ExpertJob {
  const void* ids;
  int32_t* offsets;    // experts + 1
  int32_t* position;   // n
  int32_t* source;     // n: the choice of each row, -1 behind the last
  int32_t id_bytes, experts, bins, bits;
  __device__ __forceinline__ int digit(int i, int& key) const {
    const int64_t e = id_at(ids, id_bytes, i);
    return key = e >= 0 && e < experts ? int(e) : experts;
  }
  __device__ __forceinline__ void start(int d, int first) const { offsets[d] = first; }
  __device__ __forceinline__ void put(int i, int, int d, int place) const {
    const bool live = d < experts;
    position[i] = live ? place : -1;
    source[place] = live ? i : -1;
  }
};

constexpr int kGroup = 4;   // choices whose loads are in flight together

// A choice's row, -1 where it has none (or names one that does not exist).
__device__ __forceinline__ int row_of(const int32_t* position, int64_t slot, int64_t rows) {
  const int p = position[slot];
  return p >= 0 && p < rows ? p : -1;
}
template <typename E>
__device__ __forceinline__ float weight_of(const RouteArgs& a, int64_t slot) {
  if (!a.weights) return 1.f;
  return a.wf32 ? static_cast<const float*>(a.weights)[slot] : float(static_cast<const E*>(a.weights)[slot]);
}

// The thread's token and first column; false past the last.
__device__ __forceinline__ bool token_chunk(const RouteArgs& a, int64_t& t, int& c, int& n) {
  const int chunks = (a.cols + 7) / 8;
  const int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x;
  t = i / chunks;
  c = int(i - t * chunks) * 8;
  n = min(8, a.cols - c);
  return t < a.tokens;
}

template <typename E>
__global__ __launch_bounds__(256) void dispatch_kernel(RouteArgs a) {
  int64_t t;
  int c, n;
  if (!token_chunk(a, t, c, n)) return;
  const int64_t all = int64_t(a.tokens) * a.top;
  const int live = min(max(a.offsets[a.experts], 0), int(all));
  float v[8];
  load8(static_cast<const E*>(a.x) + t * a.ldx + c, n, v);
  const float zero[8] = {};
  E* rows = static_cast<E*>(a.rows) + c;
  for (int j = 0; j < a.top; ++j) {
    const int64_t slot = t * a.top + j;
    const int p = row_of(a.position, slot, all);
    if (p >= 0) store8(rows + p * a.ldr, n, v);
    if (slot >= live) store8(rows + slot * a.ldr, n, zero);   // rows behind the last expert's
  }
}

// y[t] = r[t] + sum_j w[t, j] rows[position[t, j]]; without weights, the gradient of
// dispatch.
template <typename E>
__global__ __launch_bounds__(256) void gather_kernel(RouteArgs a) {
  int64_t t;
  int c, n;
  if (!token_chunk(a, t, c, n)) return;
  const int64_t all = int64_t(a.tokens) * a.top;
  const E* rows = static_cast<const E*>(a.rows) + c;
  float v[8] = {};
  if (a.res) load8(static_cast<const E*>(a.res) + t * a.ldres + c, n, v);
  for (int j = 0; j < a.top; j += kGroup) {
    float x[kGroup][8], w[kGroup];
    int p[kGroup];
#pragma unroll
    for (int k = 0; k < kGroup; ++k) {
      const int64_t slot = t * a.top + min(j + k, a.top - 1);
      p[k] = row_of(a.position, slot, all);
      if (j + k >= a.top) p[k] = -1;
      w[k] = weight_of<E>(a, slot);
    }
#pragma unroll
    for (int k = 0; k < kGroup; ++k) load8(rows + max(p[k], 0) * a.ldr, n, x[k]);
#pragma unroll
    for (int k = 0; k < kGroup; ++k)
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = p[k] >= 0 ? fmaf(w[k], x[k][e], v[e]) : v[e];
  }
  store8(static_cast<E*>(a.y) + t * a.ldy + c, n, v);
}

// A wave per choice: its row's gradient, and the product of both rows for the
// weight's.
template <typename E>
__global__ __launch_bounds__(256) void combine_grad_kernel(RouteArgs a) {
  const int lane = threadIdx.x & 63;
  const int64_t slot = int64_t(blockIdx.x) * 4 + (threadIdx.x >> 6), all = int64_t(a.tokens) * a.top;
  if (slot >= all) return;
  const int64_t t = slot / a.top;
  const int p = row_of(a.position, slot, all);
  const int live = min(max(a.offsets[a.experts], 0), int(all));
  const float w = weight_of<E>(a, slot);
  const E* dy = static_cast<const E*>(a.dy) + t * a.lddy;
  const E* h = static_cast<const E*>(a.rows) + max(p, 0) * a.ldr;
  E* dh = static_cast<E*>(a.drows);
  float dot = 0.f;
  for (int c = lane * 8; c < a.cols; c += 512) {
    const int n = min(8, a.cols - c);
    if (p >= 0) {
      float g[8], x[8];
      load8(dy + c, n, g);
      if (a.dweights) {
        load8(h + c, n, x);
#pragma unroll
        for (int e = 0; e < 8; ++e) dot = fmaf(g[e], x[e], dot);
      }
      if (dh) {
#pragma unroll
        for (int e = 0; e < 8; ++e) g[e] *= w;
        store8(dh + p * a.lddr + c, n, g);
      }
    }
    if (dh && slot >= live) {
      const float zero[8] = {};
      store8(dh + slot * a.lddr + c, n, zero);
    }
  }
  if (!a.dweights) return;
#pragma unroll
  for (int d = 32; d; d >>= 1) dot += __shfl_xor(dot, d);
  if (lane == 0) {
    if (a.wf32)
      static_cast<float*>(a.dweights)[slot] = dot;
    else
      static_cast<E*>(a.dweights)[slot] = E(dot);
  }
}

bool grid_of(int64_t blocks, dim3& g) {
  g = dim3{unsigned(blocks)};
  return blocks < (int64_t(1) << 31);
}

template <typename E>
hipError_t launch(int pass, const RouteArgs& a, hipStream_t st) {
  const int64_t chunks = (int64_t(a.cols) + 7) / 8;
  const int64_t blocks = pass == ROUTE_COMBINE_GRAD ? (int64_t(a.tokens) * a.top + 3) / 4
                                                    : (a.tokens * chunks + 255) / 256;
  dim3 g;
  if (!grid_of(blocks, g)) return hipErrorInvalidConfiguration;
  if (!blocks) return hipSuccess;
  if (pass == ROUTE_DISPATCH) hipLaunchKernelGGL((dispatch_kernel<E>), g, dim3{256}, 0, st, a);
  if (pass == ROUTE_GATHER) hipLaunchKernelGGL((gather_kernel<E>), g, dim3{256}, 0, st, a);
  if (pass == ROUTE_COMBINE_GRAD) hipLaunchKernelGGL((combine_grad_kernel<E>), g, dim3{256}, 0, st, a);
  return hipGetLastError();
}

}  // namespace

size_t expert_sort_bytes(int64_t n) { return sort_bytes(n); }

hipError_t launch_expert_sort(const void* ids, int id_bytes, int64_t n, int experts, int32_t* offsets,
                              int32_t* position, int32_t* source, int32_t* counts, hipStream_t st) {
  ExpertJob job{ids, offsets, position, source, id_bytes, experts, experts + 1, 1};
  while ((1 << job.bits) < job.bins) ++job.bits;
  return launch_sort(job, n, counts, st);
}

hipError_t launch_route(bool bf16, int pass, const RouteArgs& a, hipStream_t st) {
  return bf16 ? launch<__bf16>(pass, a, st) : launch<float>(pass, a, st);
}

}  // namespace layers
}  // namespace muon
