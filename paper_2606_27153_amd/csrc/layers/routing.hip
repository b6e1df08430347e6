// Tokens to their experts and back: the choices of an MoE router sorted by expert,
// every token's row copied to its experts' rows, the experts' outputs weighted and
// added up, and the gradients of both.
//
//   position[t, j]  row of token t's j-th choice, -1 if it chose no expert
//   rows[position[t, j]] = x[t]                  dx[t] = sum_j drows[position[t, j]]
//   y[t] = r[t] + sum_j w[t, j] rows[position[t, j]]
//   drows[position[t, j]] = w[t, j] dy[t],  dw[t, j] = <dy[t], rows[position[t, j]]>
//
// Bound by memory.  What is read or added up once for a token goes by token, what
// is read and written for each choice by row.  A thread has 8 columns (16 bytes of bf16) at a time.
// Results in bf16 are stored past the caches' order of use: combine's gradient 187 -> 170 us at the
// sizes below, the sums by token 95 -> 84, and a product over the experts that reads
// them next is not slower for it, be they 3 MB or 400.
#include "sort.h"

namespace muon {
namespace layers {
namespace {

struct ExpertJob {
  const void* ids;
  int32_t* offsets;    // experts + 1
  int32_t* position;   // n
  int32_t* source;     // n: the choice of each row; behind the last, ~ those of no expert
  int32_t id_bytes, experts, bins, bits;
  __device__ __forceinline__ int digit(int i, int& key) const {
    const int64_t e = id_at(ids, id_bytes, i);
    return key = e >= 0 && e < experts ? int(e) : experts;
  }
  __device__ __forceinline__ void start(int d, int first) const { offsets[d] = first; }
  __device__ __forceinline__ void put(int i, int, int d, int place) const {
    const bool live = d < experts;
    position[i] = live ? place : -1;
    source[place] = live ? i : ~i;
  }
};

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

// The thread's row (of `rows`) and first column; false past the last.
__device__ __forceinline__ bool row_chunk(const RouteArgs& a, int64_t rows, int64_t& r, int& c, int& n) {
  const int chunks = (a.cols + 7) / 8;
  const int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x;
  r = i / chunks;
  c = int(i - r * chunks) * 8;
  n = min(8, a.cols - c);
  return r < rows;
}

// By token: its row is read once and stored at its choices' rows; the rows behind the
// last expert's are cleared by the threads of the tokens that their numbers fall to.
// 16384 x 2048 tokens of 6 choices in bf16 take 74 to 77 us, 6.2 TB/s, most of it stores
// (by row, each reading its token from the cache, 122).
// Choices whose places are looked up together: all of most routers at once.  6, or kernels of their
// own for 2, 4, 6 and 8, take as long (1 to 16 choices; those kernels 23 us for 21 of one choice).
constexpr int kStores = 8;
template <typename E, bool WHOLE>
__global__ __launch_bounds__(256) void dispatch_kernel(RouteArgs a) {
  int64_t t;
  int c, n;
  if (!row_chunk(a, a.tokens, t, c, n)) return;
  const int64_t all = int64_t(a.tokens) * a.top;
  float v[8];
  load_8<WHOLE>(static_cast<const E*>(a.x) + t * a.ldx + c, n, v);
  const float zero[8] = {};
  E* rows = static_cast<E*>(a.rows) + c;
  for (int j = 0; j < a.top; j += kStores) {
    int p[kStores], s[kStores];
#pragma unroll
    for (int k = 0; k < kStores; ++k) {
      const int64_t slot = t * a.top + min(j + k, a.top - 1);
      p[k] = row_of(a.position, slot, all);
      s[k] = a.source[slot];
    }
#pragma unroll
    for (int k = 0; k < kStores; ++k) {
      if (j + k >= a.top) continue;
      if (p[k] >= 0) store_8_run<WHOLE>(rows + p[k] * a.ldr, n, v);
      if (s[k] < 0) store_8_run<WHOLE>(rows + (t * a.top + j + k) * a.ldr, n, zero);
    }
  }
}
// y[t] = r[t] + sum_j w[t, j] rows[position[t, j]]; without weights, the gradient of
// dispatch.  K choices' loads are in flight together.  16384 x 2048 tokens of 6 choices
// 84 us on average with a residual and without (6.0 TB/s), loads past the caches' order of
// use; with ordinary loads and stores 135 and 106.  In fp32 176 and 202 with ordinary ones (past the
// caches 191 and 212; 4096 x 1024 18 and 20, 25 and 26).
template <typename E, int K, bool WHOLE>
__global__ __launch_bounds__(256) void gather_kernel(RouteArgs a) {
  int64_t t;
  int c, n;
  if (!row_chunk(a, a.tokens, t, c, n)) return;
  const int64_t all = int64_t(a.tokens) * a.top;
  const E* rows = static_cast<const E*>(a.rows) + c;
  float v[8] = {};
  if (a.res) load_8_run<WHOLE>(static_cast<const E*>(a.res) + t * a.ldres + c, n, v);
  for (int j = 0; j < a.top; j += K) {
    float x[K][8], w[K];
    int p[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int64_t slot = t * a.top + min(j + k, a.top - 1);
      p[k] = row_of(a.position, slot, all);
      if (j + k >= a.top) p[k] = -1;
      w[k] = weight_of<E>(a, slot);
    }
#pragma unroll
    for (int k = 0; k < K; ++k) load_8_run<WHOLE>(rows + max(p[k], 0) * a.ldr, n, x[k]);
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = p[k] >= 0 ? fmaf(w[k], x[k][e], v[e]) : v[e];
  }
  store_8_run<WHOLE>(static_cast<E*>(a.y) + t * a.ldy + c, n, v);
}

// A wave per row: its gradient, and the product of both rows for the weight's.  A row
// behind the last expert's stands for a choice of no expert: both are 0.  Two chunks of
// 512 columns are in flight; both large streams go through memory in order, the tokens'
// gradients come from the cache: 170 us at 16384 x 2048 and 6 choices, 5.1 TB/s (by token,
// with its gradient in registers, half as slow again).
template <typename E, bool WHOLE>
__global__ __launch_bounds__(256) void combine_grad_kernel(RouteArgs a) {
  const int lane = threadIdx.x & 63;
  const int64_t r = int64_t(blockIdx.x) * 4 + (threadIdx.x >> 6), all = int64_t(a.tokens) * a.top;
  if (r >= all) return;
  const int from = __builtin_amdgcn_readfirstlane(a.source[r]);
  const int slot = from < 0 ? ~from : from;
  const bool named = slot < all, live = from >= 0 && named;
  const float w = live ? weight_of<E>(a, slot) : 0.f;
  const E* dy = static_cast<const E*>(a.dy) + (live ? slot / a.top : 0) * a.lddy;
  const E* h = a.dweights ? static_cast<const E*>(a.rows) + r * a.ldr : dy;
  E* dh = a.drows ? static_cast<E*>(a.drows) + r * a.lddr : nullptr;
  float dot = 0.f;
  for (int c = lane * 8; c < a.cols; c += 1024) {
    const int n = min(8, a.cols - c), n2 = min(8, a.cols - c - 512);
    const bool two = n2 > 0;
    float g[2][8], x[2][8];
    const int c2 = two ? c + 512 : c;
    load_8<WHOLE>(dy + c, n, g[0]);
    load_8_once<WHOLE>(h + c, n, x[0]);
    load_8<WHOLE>(dy + c2, two ? n2 : n, g[1]);
    load_8_once<WHOLE>(h + c2, two ? n2 : n, x[1]);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      dot = fmaf(g[0][e], x[0][e], dot);
      g[0][e] = live ? g[0][e] * w : 0.f;
    }
    if (dh) store_8_once<WHOLE>(dh + c, n, g[0]);
    if (two) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        dot = fmaf(g[1][e], x[1][e], dot);
        g[1][e] = live ? g[1][e] * w : 0.f;
      }
      if (dh) store_8_once<WHOLE>(dh + c2, n2, g[1]);
    }
  }
  if (!a.dweights || !named) return;
#pragma unroll
  for (int d = 32; d; d >>= 1) dot += __shfl_xor(dot, d);
  if (!live) dot = 0.f;
  if (lane == 0) {
    if (a.wf32)
      static_cast<float*>(a.dweights)[slot] = dot;
    else
      static_cast<E*>(a.dweights)[slot] = E(dot);
  }
}

bool grid_of(int64_t blocks, dim3& g) {
  g = dim3{unsigned(blocks)};
  return blocks < kMaxGrid;
}

template <typename E, bool WHOLE>
hipError_t launch(int pass, const RouteArgs& a, hipStream_t st) {
  const int64_t chunks = (int64_t(a.cols) + 7) / 8, rows = int64_t(a.tokens) * a.top;
  const int64_t blocks = pass == ROUTE_COMBINE_GRAD ? (rows + 3) / 4
                                                    : (a.tokens * chunks + 255) / 256;
  dim3 g, b{256};
  if (!grid_of(blocks, g)) return hipErrorInvalidConfiguration;
  if (!blocks) return hipSuccess;
  if (pass == ROUTE_DISPATCH) hipLaunchKernelGGL((dispatch_kernel<E, WHOLE>), g, b, 0, st, a);
  if (pass == ROUTE_COMBINE_GRAD) hipLaunchKernelGGL((combine_grad_kernel<E, WHOLE>), g, b, 0, st, a);
  if (pass == ROUTE_GATHER) {
    if (a.top <= 2)
      hipLaunchKernelGGL((gather_kernel<E, 2, WHOLE>), g, b, 0, st, a);
    else if (a.top <= 4)
      hipLaunchKernelGGL((gather_kernel<E, 4, WHOLE>), g, b, 0, st, a);
    else if (a.top <= 6)
      hipLaunchKernelGGL((gather_kernel<E, 6, WHOLE>), g, b, 0, st, a);
    else
      hipLaunchKernelGGL((gather_kernel<E, 8, WHOLE>), g, b, 0, st, a);
  }
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
  if (a.cols % 8)
    return bf16 ? launch<__bf16, false>(pass, a, st) : launch<float, false>(pass, a, st);
  return bf16 ? launch<__bf16, true>(pass, a, st) : launch<float, true>(pass, a, st);
}

}  // namespace layers
}  // namespace muon
