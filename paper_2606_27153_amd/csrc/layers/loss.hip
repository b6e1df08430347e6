// Softmax cross entropy over the columns of z = x W, of which only pieces exist.
//
//   lse[i] = m + log sum_v exp(z[i, v] - m),  loss[i] = lse[i] - z[i, t[i]]
//   dz[i, v] = (exp(z[i, v] - lse[i]) - [v = t[i]]) g[i]
//
// A strip of columns leaves (m, sum of exp(z - m)) per row; the strips are joined
// at the end: any number of them, in order.  The gradient's pieces are made from
// z computed again and lse.  Everything is fp32 until dz is rounded to the operands' type.
// A row without a target has loss 0 and a gradient of 0, whatever its logits hold.
//
// The products are all that counts (the tile kernels', whose epilogues are the strips
// and the gradient: mm_tile.h): 16384 rows x 4096 over 128000 columns in bf16 take 54.6
// ms both ways: four products of 17.2 TFLOP at 1200 to 1380 TFLOP/s; one row
// reads the weight at 6.1 TB/s.  Of this file's kernels the outer product writes the weight's
// gradient of few rows (200 to 450 us of 4096 x 128000); the others take 5 to 25 us each, those
// that pass over x and dx 42 and 86.
//
// dz is rounded to bf16 where the operands are: the matrix cores take both operands of a
// product in the same type, and a second product of what the rounding leaves would cost another
// 4 N D V operations.  dx and dW are then 1.66e-3 to 2.3e-3 from 64 bits (relative norm), where
// dz in 32 bits gives 1.65e-3 to 1.8e-3, the outputs' own rounding.
//
// An upstream gradient that is one number is no factor of dz but of the products
// that read it (alpha): rounding g (p - 1) to bf16 would give all rows the same
// relative error, up to 2^-9, where those of p - 1 and p are independent.
#include "device.h"

namespace muon {
namespace layers {
namespace {

__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d);
  return v;
}
__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
  for (int d = 32; d; d >>= 1) v = fmaxf(v, __shfl_xor(v, d));
  return v;
}
// exp(v - m) where m is the largest; a strip of nothing but -inf has sum 0.
__device__ __forceinline__ float reference(float m) { return m == -INFINITY ? 0.f : m; }

// One block: how many rows have a target, and the factor of a mean's gradients.
__global__ __launch_bounds__(1024) void mean_kernel(LossArgs a, float* alpha) {
  __shared__ int counts[16];
  int n = 0;
  for (int i = threadIdx.x; i < a.rows; i += 1024) n += label_of(a, i) >= 0;
#pragma unroll
  for (int d = 32; d; d >>= 1) n += __shfl_xor(n, d);
  if ((threadIdx.x & 63) == 0) counts[threadIdx.x >> 6] = n;
  __syncthreads();
  if (threadIdx.x) return;
  n = 0;
  for (int w = 0; w < 16; ++w) n += counts[w];
  *alpha = *a.dloss / float(max(n, 1));
}

// 8 logits of a row from column c of the piece on (-inf past its end).
__device__ __forceinline__ void load_logits(const LossArgs& a, int64_t row, int c, float (&v)[8]) {
  const int n = a.cols - c;
  load8(a.raw + row * a.cols + c, n, v);
  for (int s = 1; s < a.splits; ++s) {
    float x[8];
    load8(a.raw + (int64_t(s) * a.rows + row) * a.cols + c, n, x);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] += x[e];
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = e < n ? v[e] : -INFINITY;
}

__global__ __launch_bounds__(256) void strip_kernel(LossArgs a) {
  static_assert(kRawStrip == 256 * 8, "a thread has 8 columns");
  __shared__ float red[2][4];
  const int64_t row = blockIdx.y;
  const int c = (blockIdx.x * 256 + threadIdx.x) * 8, lane = threadIdx.x & 63, wid = threadIdx.x >> 6;
  float v[8];
  if (c < a.cols) {
    load_logits(a, row, c, v);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = -INFINITY;
  }
  const int label = label_of(a, row), at = label - a.first - c;
  if (label >= 0 && at >= 0 && at < 8) {
    float z = v[0];
#pragma unroll
    for (int e = 1; e < 8; ++e) z = at == e ? v[e] : z;
    a.logit[row] = z;
  }
  float m = v[0];
#pragma unroll
  for (int e = 1; e < 8; ++e) m = fmaxf(m, v[e]);
  m = wave_max(m);
  if (lane == 0) red[0][wid] = m;
  __syncthreads();
  m = reference(fmaxf(fmaxf(red[0][0], red[0][1]), fmaxf(red[0][2], red[0][3])));
  float s = 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) s += __expf(v[e] - m);
  s = wave_sum(s);
  if (lane == 0) red[1][wid] = s;
  __syncthreads();
  if (threadIdx.x == 0)
    a.part[int64_t(a.strip + blockIdx.x) * a.rows + row] =
        make_float2(m, red[1][0] + red[1][1] + red[1][2] + red[1][3]);
}

// (m, s) of two sets of columns.
__device__ __forceinline__ float2 join(float2 a, float2 b) {
  const float top = fmaxf(a.y == 0.f ? -INFINITY : a.x, b.y == 0.f ? -INFINITY : b.x), r = reference(top);
  return make_float2(r, (a.y == 0.f ? 0.f : a.y * __expf(a.x - r)) + (b.y == 0.f ? 0.f : b.y * __expf(b.x - r)));
}

// 2^shift rows of a block, whose 16 waves and their lanes share the strips.
__global__ __launch_bounds__(1024) void finish_kernel(LossArgs a, int shift) {
  __shared__ float2 red[16][64];
  const int lane = threadIdx.x & 63, wid = threadIdx.x >> 6, in = lane & ((1 << shift) - 1);
  const int64_t row = (int64_t(blockIdx.x) << shift) + in;
  const int lists = 1024 >> shift, list = wid * (64 >> shift) + (lane >> shift);
  float m = -INFINITY, s = 0.f;
  if (row < a.rows) {
    for (int i = list; i < a.strips; i += 8 * lists) {
      float2 p[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        p[k] = a.part[int64_t(min(i + k * lists, a.strips - 1)) * a.rows + row];
        if (i + k * lists >= a.strips) p[k].y = 0.f;
      }
      float top = m;
#pragma unroll
      for (int k = 0; k < 8; ++k) top = fmaxf(top, p[k].y == 0.f ? -INFINITY : p[k].x);
      const float r = reference(top);
      s = s == 0.f ? 0.f : s * __expf(m - r);
#pragma unroll
      for (int k = 0; k < 8; ++k) s += p[k].y == 0.f ? 0.f : p[k].y * __expf(p[k].x - r);
      m = r;
    }
  }
  float2 v = make_float2(m, s);
  for (int d = 32; d >> shift; d >>= 1) {
    const float2 o = make_float2(__shfl_xor(v.x, d), __shfl_xor(v.y, d));
    v = lane & d ? join(o, v) : join(v, o);
  }
  red[wid][lane] = v;
  __syncthreads();
  if (wid || lane >> shift || row >= a.rows) return;
  for (int w = 1; w < 16; ++w) v = join(v, red[w][lane]);
  const float lse = reference(v.x) + logf(v.y);
  a.lse[row] = lse;
  a.loss[row] = label_of(a, row) >= 0 ? lse - a.logit[row] : 0.f;
}

// One block: the sum or mean of the rows' losses.
__global__ __launch_bounds__(1024) void total_kernel(LossArgs a) {
  __shared__ float sums[16];
  __shared__ int counts[16];
  float s = 0.f;
  int n = 0;
  for (int i = threadIdx.x; i < a.rows; i += 1024) {
    s += a.loss[i];
    n += label_of(a, i) >= 0;
  }
  s = wave_sum(s);
#pragma unroll
  for (int d = 32; d; d >>= 1) n += __shfl_xor(n, d);
  if ((threadIdx.x & 63) == 0) {
    sums[threadIdx.x >> 6] = s;
    counts[threadIdx.x >> 6] = n;
  }
  __syncthreads();
  if (threadIdx.x) return;
  s = 0.f;
  n = 0;
  for (int w = 0; w < 16; ++w) {
    s += sums[w];
    n += counts[w];
  }
  *a.total = a.mean ? s / float(max(n, 1)) : s;
}

template <typename E>
__global__ __launch_bounds__(256) void grad_kernel(LossArgs a) {
  const int64_t row = blockIdx.y;
  const int c = (blockIdx.x * 256 + threadIdx.x) * 8;
  if (c >= a.cols) return;
  float v[8];
  load_logits(a, row, c, v);
  const int label = label_of(a, row);
  const float lse = a.lse[row], g = a.each ? a.dloss[row] : 1.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float p = __expf(v[e] - lse) - (label - a.first - c == e ? 1.f : 0.f);
    v[e] = label >= 0 && c + e < a.cols ? p * g : 0.f;
  }
  // (rows of dz are whole groups of 8, with zeros after the piece's end)
  store8(static_cast<E*>(a.dz) + row * a.lddz + c, 8, v);
}

// x with zeros in the rows without a target (and behind its columns), for the weight's
// gradient: whatever they hold, their 0 of dz must not make NaN of it.  16384 x 4096 in
// bf16 take 42 us of a step's 54500.
template <typename E, bool WHOLE>
__global__ __launch_bounds__(256) void rows_kernel(LossArgs a, const E* x, int64_t ldx, E* y, int64_t ldy,
                                                   int64_t cols) {
  const int64_t chunks = (ldy + 7) / 8, i = int64_t(blockIdx.x) * 256 + threadIdx.x, r = i / chunks;
  if (r >= a.rows) return;
  const int64_t c = (i - r * chunks) * 8;
  const bool live = label_of(a, r) >= 0;
  float v[8];
  load_8<WHOLE>(x + r * ldx + c, int(min(int64_t(8), cols - c)), v);
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = live ? v[e] : 0.f;
  store_8<WHOLE>(y + r * ldy + c, int(min(int64_t(8), ldy - c)), v);
}

// The weight's gradient of few rows: out[r][c] = alpha sum_m a[m][r] b[m][c] with the rows m of
// x, without those of no target, and of dz.  A thread keeps 16 bytes' columns of every b[m]
// and walks down 32 rows of `out`, whose a are in LDS: each store of a wave is one run of
// bytes.  Bound by the stores and, towards the most rows, as much by the M multiply-adds an
// element: 4096 x 128000 of 8 rows 200 us in bf16 (5.2 TB/s) and 380 in fp32 (5.5), of 20 rows
// in fp32 450.  The tile kernels, which have one slab of K to do and wait for their
// stores, take 310 and 590 of any few rows.  Where `out` is narrow, a block's threads are
// 2^shift columns' by as many rows as there are.  X_DOWN: a is x, else b is.
constexpr int kOuterRows = 32;
template <typename E, int M, bool X_DOWN>
__global__ __launch_bounds__(256) void outer_kernel(LossArgs l, const E* x, int64_t ldx, int64_t inner, E* out,
                                                    int64_t ldo, int shift) {
  constexpr int N = 16 / sizeof(E);
  __shared__ __attribute__((aligned(16))) float down[kOuterRows][M];
  const E* const dz = static_cast<const E*>(l.dz);
  const int64_t rows = X_DOWN ? inner : l.cols, cols = X_DOWN ? l.cols : inner;
  const int64_t r0 = int64_t(blockIdx.y) * kOuterRows;
  const int64_t c = ((int64_t(blockIdx.x) << shift) + (threadIdx.x & ((1 << shift) - 1))) * N;
  const int n = int(min(int64_t(N), cols - c)), deep = int(min(int64_t(kOuterRows), rows - r0));
  for (int i = threadIdx.x; i < kOuterRows * M; i += 256) {
    const int m = i / kOuterRows, r = i % kOuterRows;
    float v = 0.f;
    if (m < l.rows && r < deep) {
      if constexpr (X_DOWN)
        v = label_of(l, m) >= 0 ? float(x[m * ldx + r0 + r]) : 0.f;
      else
        v = float(dz[m * l.lddz + r0 + r]);
    }
    down[r][m] = v;
  }
  struct __attribute__((packed, aligned(sizeof(E)))) Run {
    E v[N];
  };
  float b[M][N];
#pragma unroll
  for (int m = 0; m < M; ++m) {
    const int at = min(m, l.rows - 1);
    const bool live = m < l.rows && (X_DOWN || label_of(l, at) >= 0);
    const E* from = X_DOWN ? dz + at * l.lddz + c : x + at * ldx + c;
    if (n == N) {
      const Run t = *reinterpret_cast<const Run*>(from);
#pragma unroll
      for (int e = 0; e < N; ++e) b[m][e] = live ? float(t.v[e]) : 0.f;
    } else {
#pragma unroll
      for (int e = 0; e < N; ++e) b[m][e] = live && e < n ? float(from[e]) : 0.f;
    }
  }
  const float f = l.alpha ? *l.alpha : 1.f;
  __syncthreads();
  if (n <= 0) return;
  for (int r = threadIdx.x >> shift; r < deep; r += 256 >> shift) {
    E* const to = out + (r0 + r) * ldo + c;
    float v[N] = {};
#pragma unroll
    for (int m = 0; m < M; m += 4) {
      const float4 a = *reinterpret_cast<const float4*>(&down[r][m]);
#pragma unroll
      for (int e = 0; e < N; ++e) {
        v[e] = fmaf(a.x, b[m][e], v[e]);
        v[e] = fmaf(a.y, b[m + 1][e], v[e]);
        v[e] = fmaf(a.z, b[m + 2][e], v[e]);
        v[e] = fmaf(a.w, b[m + 3][e], v[e]);
      }
    }
    Run w;
#pragma unroll
    for (int e = 0; e < N; ++e) w.v[e] = E(v[e] * f);
    if (n == N) {
      typedef uint32_t Words __attribute__((ext_vector_type(4), aligned(2)));
      __builtin_nontemporal_store(__builtin_bit_cast(Words, w), reinterpret_cast<Words*>(to));
    } else {
#pragma unroll
      for (int e = 0; e < N; ++e)
        if (e < n) to[e] = w.v[e];
    }
  }
}

// The input's gradient: the partial results added up, times alpha; 0 in rows without a target
// (also where a weight that is not finite or an infinite alpha would leave NaN).
template <typename E>
__global__ __launch_bounds__(256) void sum_kernel(LossArgs a, const float* part, int splits, E* y, int64_t ldy,
                                                  int64_t cols) {
  const int64_t chunks = (cols + 7) / 8, i = int64_t(blockIdx.x) * 256 + threadIdx.x, r = i / chunks;
  if (r >= a.rows) return;
  const int64_t c = (i - r * chunks) * 8;
  const int n = int(min(int64_t(8), cols - c));
  const float f = a.alpha ? *a.alpha : 1.f;
  const bool live = label_of(a, r) >= 0;
  float v[8] = {};
  for (int s = 0; s < splits; s += 4) {   // in order, 4 in flight
    float x[4][8];
#pragma unroll
    for (int k = 0; k < 4; ++k) load8(part + (int64_t(min(s + k, splits - 1)) * a.rows + r) * cols + c, n, x[k]);
#pragma unroll
    for (int k = 0; k < 4; ++k)
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] += s + k < splits ? x[k][e] : 0.f;
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = live ? v[e] * f : 0.f;
  store8(y + r * ldy + c, n, v);
}

unsigned strips_of(const LossArgs& a) { return unsigned((a.cols + kRawStrip - 1) / kRawStrip); }

}  // namespace

hipError_t launch_loss_mean(const LossArgs& a, float* alpha, hipStream_t st) {
  hipLaunchKernelGGL(mean_kernel, dim3{1}, dim3{1024}, 0, st, a, alpha);
  return hipGetLastError();
}

hipError_t launch_loss_strips(const LossArgs& a, hipStream_t st) {
  if (a.rows > 65535) return hipErrorInvalidConfiguration;
  hipLaunchKernelGGL(strip_kernel, (dim3{strips_of(a), unsigned(a.rows)}), dim3{256}, 0, st, a);
  return hipGetLastError();
}

hipError_t launch_loss_finish(const LossArgs& a, hipStream_t st) {
  // 64 rows read whole lines; fewer where there are not enough for every CU
  int shift = 6;
  while (shift && (a.rows >> shift) < kCUs) --shift;
  hipLaunchKernelGGL(finish_kernel, dim3{unsigned((int64_t(a.rows) + (1 << shift) - 1) >> shift)}, dim3{1024}, 0, st, a,
                     shift);
  return hipGetLastError();
}

hipError_t launch_loss_total(const LossArgs& a, hipStream_t st) {
  hipLaunchKernelGGL(total_kernel, dim3{1}, dim3{1024}, 0, st, a);
  return hipGetLastError();
}

hipError_t launch_loss_grad(bool bf16, const LossArgs& a, hipStream_t st) {
  if (a.rows > 65535) return hipErrorInvalidConfiguration;
  const dim3 g{strips_of(a), unsigned(a.rows)};
  if (bf16)
    hipLaunchKernelGGL((grad_kernel<__bf16>), g, dim3{256}, 0, st, a);
  else
    hipLaunchKernelGGL((grad_kernel<float>), g, dim3{256}, 0, st, a);
  return hipGetLastError();
}

hipError_t launch_loss_rows(bool bf16, const LossArgs& a, const void* x, int64_t ldx, void* y, int64_t ldy,
                            int64_t cols, hipStream_t st) {
  const int64_t blocks = (a.rows * ((ldy + 7) / 8) + 255) / 256;
  if (blocks >= kMaxGrid) return hipErrorInvalidConfiguration;
  const dim3 g{unsigned(blocks)}, b{256};
  auto run = [&](auto kernel, auto one) {
    typedef decltype(one) E;
    hipLaunchKernelGGL(kernel, g, b, 0, st, a, static_cast<const E*>(x), ldx, static_cast<E*>(y), ldy, cols);
  };
  if (cols % 8)
    bf16 ? run(rows_kernel<__bf16, false>, __bf16()) : run(rows_kernel<float, false>, float());
  else
    bf16 ? run(rows_kernel<__bf16, true>, __bf16()) : run(rows_kernel<float, true>, float());
  return hipGetLastError();
}

hipError_t launch_loss_outer(bool bf16, bool x_down, const LossArgs& a, const void* x, int64_t ldx, int64_t inner,
                             void* out, int64_t ldo, hipStream_t st) {
  const int64_t down = x_down ? inner : a.cols, across = x_down ? a.cols : inner, lane = bf16 ? 8 : 4;
  int shift = 8;
  while (shift > 3 && across <= lane << (shift - 1)) --shift;
  const int64_t wide = lane << shift;
  const dim3 g{unsigned((across + wide - 1) / wide), unsigned((down + kOuterRows - 1) / kOuterRows)}, b{256};
  if (a.rows > outer_rows(bf16) || g.x >= kMaxGrid || g.y > 65535) return hipErrorInvalidConfiguration;
  auto run = [&](auto kernel, auto one) {
    typedef decltype(one) E;
    hipLaunchKernelGGL(kernel, g, b, 0, st, a, static_cast<const E*>(x), ldx, inner, static_cast<E*>(out), ldo,
                       shift);
  };
  auto rows = [&](auto one) {
    typedef decltype(one) E;
    if (a.rows <= 4)
      x_down ? run(outer_kernel<E, 4, true>, one) : run(outer_kernel<E, 4, false>, one);
    else if (a.rows <= 8)
      x_down ? run(outer_kernel<E, 8, true>, one) : run(outer_kernel<E, 8, false>, one);
    else if (a.rows <= 16)
      x_down ? run(outer_kernel<E, 16, true>, one) : run(outer_kernel<E, 16, false>, one);
    else if constexpr (sizeof(E) == 4)
      x_down ? run(outer_kernel<E, 32, true>, one) : run(outer_kernel<E, 32, false>, one);
  };
  bf16 ? rows(__bf16()) : rows(float());
  return hipGetLastError();
}

hipError_t launch_loss_sum(bool bf16, const LossArgs& a, const float* part, int splits, void* y, int64_t ldy,
                           int64_t cols, hipStream_t st) {
  const int64_t blocks = (a.rows * ((cols + 7) / 8) + 255) / 256;
  if (blocks >= kMaxGrid) return hipErrorInvalidConfiguration;
  const dim3 g{unsigned(blocks)}, b{256};
  if (bf16)
    hipLaunchKernelGGL((sum_kernel<__bf16>), g, b, 0, st, a, part, splits, static_cast<__bf16*>(y), ldy, cols);
  else
    hipLaunchKernelGGL((sum_kernel<float>), g, b, 0, st, a, part, splits, static_cast<float*>(y), ldy, cols);
  return hipGetLastError();
}

}  // namespace layers
}  // namespace muon
