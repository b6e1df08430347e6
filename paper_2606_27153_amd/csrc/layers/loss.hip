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
// An upstream gradient that is one number is no factor of dz but of the products
// that read it (alpha): rounding g (p - 1) to bf16 would give all rows the same
// relative error, up to 2^-9, where those of p - 1 and p are independent.
#include "device.h"

namespace muon {
namespace layers {
namespace {

constexpr float kLog2e = 1.4426950408889634f;

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

// One block: the labels, how many there are, and what the gradients are scaled with.
__global__ __launch_bounds__(1024) void label_kernel(LossArgs a) {
  __shared__ int counts[16];
  int count = 0;
  for (int i = threadIdx.x; i < a.rows; i += 1024) {
    const int64_t t = a.target_bytes == 8 ? static_cast<const int64_t*>(a.targets)[i]
                                          : int64_t(static_cast<const int32_t*>(a.targets)[i]);
    const bool live = t >= 0 && t < a.vocab && t != a.ignore;
    count += live;
    a.label[i] = live ? int(t) : -1;
    if (a.dloss) a.grad[i] = !live ? 0.f : a.each ? a.dloss[i] : 1.f;
  }
  if (!a.dloss) return;
#pragma unroll
  for (int d = 32; d; d >>= 1) count += __shfl_xor(count, d);
  if ((threadIdx.x & 63) == 0) counts[threadIdx.x >> 6] = count;
  __syncthreads();
  if (threadIdx.x == 0) {
    int n = 0;
    for (int w = 0; w < 16; ++w) n += counts[w];
    *a.alpha = a.each ? 1.f : a.mean ? *a.dloss / float(max(n, 1)) : *a.dloss;
  }
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
  const int at = a.label[row] - a.first - c;
  if (a.label[row] >= 0 && at >= 0 && at < 8) {
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

// 64 rows of a block, whose 16 waves share the strips.
__global__ __launch_bounds__(1024) void finish_kernel(LossArgs a) {
  __shared__ float2 red[16][64];
  const int lane = threadIdx.x & 63, wid = threadIdx.x >> 6;
  const int64_t row = int64_t(blockIdx.x) * 64 + lane;
  float m = -INFINITY, s = 0.f;
  if (row < a.rows) {
    const int per = (a.strips + 15) / 16, s0 = wid * per, s1 = min(a.strips, s0 + per);
    for (int i = s0; i < s1; i += 8) {
      float2 p[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) p[k] = a.part[int64_t(min(i + k, s1 - 1)) * a.rows + row];
      float top = m;
#pragma unroll
      for (int k = 0; k < 8; ++k) top = fmaxf(top, p[k].y == 0.f ? -INFINITY : p[k].x);
      const float r = reference(top);
      s = s == 0.f ? 0.f : s * __expf(m - r);
#pragma unroll
      for (int k = 0; k < 8; ++k) s += i + k < s1 && p[k].y != 0.f ? p[k].y * __expf(p[k].x - r) : 0.f;
      m = top;
    }
  }
  red[wid][lane] = make_float2(m, s);
  __syncthreads();
  if (wid || row >= a.rows) return;
  float top = -INFINITY, sum = 0.f;
  for (int w = 0; w < 16; ++w) top = fmaxf(top, red[w][lane].x);
  const float r = reference(top);
  for (int w = 0; w < 16; ++w) sum += red[w][lane].y == 0.f ? 0.f : red[w][lane].y * __expf(red[w][lane].x - r);
  const float lse = r + logf(sum);
  a.lse[row] = lse;
  a.loss[row] = a.label[row] >= 0 ? lse - a.logit[row] : 0.f;
}

// One block: the sum or mean of the rows' losses.
__global__ __launch_bounds__(1024) void total_kernel(LossArgs a) {
  __shared__ float sums[16];
  __shared__ int counts[16];
  float s = 0.f;
  int n = 0;
  for (int i = threadIdx.x; i < a.rows; i += 1024) {
    s += a.loss[i];
    n += a.label[i] >= 0;
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
  const int label = a.label[row];
  const float lse = a.lse[row], g = a.grad[row];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float p = __expf(v[e] - lse) - (label - a.first - c == e ? 1.f : 0.f);
    v[e] = label >= 0 && c + e < a.cols ? p * g : 0.f;
  }
  // (rows of dz are whole groups of 8, with zeros after the piece's end)
  store8(static_cast<E*>(a.dz) + row * a.lddz + c, 8, v);
}

template <typename E>
__global__ __launch_bounds__(256) void sum_kernel(const float* part, int splits, const float* alpha, E* y, int64_t ldy,
                                                  int64_t rows, int64_t cols) {
  const int64_t chunks = (cols + 7) / 8, i = int64_t(blockIdx.x) * 256 + threadIdx.x, r = i / chunks;
  if (r >= rows) return;
  const int64_t c = (i - r * chunks) * 8;
  const int n = int(min(int64_t(8), cols - c));
  const float f = *alpha;
  float v[8];
  load8(part + r * cols + c, n, v);
  for (int s = 1; s < splits; ++s) {
    float x[8];
    load8(part + (s * rows + r) * cols + c, n, x);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] += x[e];
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] *= f;
  store8(y + r * ldy + c, n, v);
}

unsigned strips_of(const LossArgs& a) { return unsigned((a.cols + kRawStrip - 1) / kRawStrip); }

}  // namespace

hipError_t launch_loss_labels(const LossArgs& a, hipStream_t st) {
  hipLaunchKernelGGL(label_kernel, dim3{1}, dim3{1024}, 0, st, a);
  return hipGetLastError();
}

hipError_t launch_loss_strips(const LossArgs& a, hipStream_t st) {
  if (a.rows > 65535) return hipErrorInvalidConfiguration;
  hipLaunchKernelGGL(strip_kernel, (dim3{strips_of(a), unsigned(a.rows)}), dim3{256}, 0, st, a);
  return hipGetLastError();
}

hipError_t launch_loss_finish(const LossArgs& a, hipStream_t st) {
  hipLaunchKernelGGL(finish_kernel, dim3{unsigned((int64_t(a.rows) + 63) / 64)}, dim3{1024}, 0, st, a);
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

hipError_t launch_loss_sum(bool bf16, const float* part, int splits, const float* alpha, void* y, int64_t ldy,
                           int64_t rows, int64_t cols, hipStream_t st) {
  const int64_t blocks = (rows * ((cols + 7) / 8) + 255) / 256;
  if (blocks >= (int64_t(1) << 31)) return hipErrorInvalidConfiguration;
  const dim3 g{unsigned(blocks)};
  if (bf16)
    hipLaunchKernelGGL((sum_kernel<__bf16>), g, dim3{256}, 0, st, part, splits, alpha, static_cast<__bf16*>(y), ldy,
                       rows, cols);
  else
    hipLaunchKernelGGL((sum_kernel<float>), g, dim3{256}, 0, st, part, splits, alpha, static_cast<float*>(y), ldy,
                       rows, cols);
  return hipGetLastError();
}

}  // namespace layers
}  // namespace muon
