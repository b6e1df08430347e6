// Layer norm over the columns, forward and backward, for rows of any length,
// stride and alignment.
//
//   mean = sum x / n,  rstd = 1 / sqrt(sum (x - mean)^2 / n + eps)
//   y = (x - mean) rstd w + b
//   h = (x - mean) rstd,  g = dy w
//   dx = rstd (g - sum g / n - h sum(g h) / n),  dw = sum_rows dy h,  db = sum_rows dy
//
// All sums are fp32.  The variance is summed around the mean (a second pass),
// not as E[x^2] - mean^2, which cancels for rows far from 0.
#include "device.h"

namespace muon {
namespace layers {
namespace {

template <int T>
__device__ __forceinline__ float block_sum(float v, float* red) {
#pragma unroll
  for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d);
  if (T > 64) {
    __syncthreads();   // red may still be read from the previous sum
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0.f;
#pragma unroll
    for (int i = 0; i < T / 64; ++i) v += red[i];
  }
  return v;
}

__device__ __forceinline__ float weight_at(const void* w, int wf32, int64_t i, const __bf16*) {
  return wf32 ? static_cast<const float*>(w)[i] : float(static_cast<const __bf16*>(w)[i]);
}
__device__ __forceinline__ float weight_at(const void* w, int, int64_t i, const float*) {
  return static_cast<const float*>(w)[i];
}

template <typename E>
__global__ __launch_bounds__(256) void norm_forward_loop_kernel(NormArgs a) {
  __shared__ float red[4];
  const int64_t r = blockIdx.x;
  const E* x = static_cast<const E*>(a.x) + r * a.ldx;
  float s = 0.f;
  for (int c = threadIdx.x; c < a.cols; c += 256) s += float(x[c]);
  const float mean = block_sum<256>(s, red) / float(a.cols);
  s = 0.f;
  for (int c = threadIdx.x; c < a.cols; c += 256) {
    const float d = float(x[c]) - mean;
    s = fmaf(d, d, s);
  }
  const float rstd = 1.f / sqrtf(block_sum<256>(s, red) / float(a.cols) + a.eps);
  if (threadIdx.x == 0) {
    if (a.mean) a.mean[r] = mean;
    if (a.rstd) a.rstd[r] = rstd;
  }
  E* y = static_cast<E*>(a.y) + r * a.ldy;
  for (int c = threadIdx.x; c < a.cols; c += 256) {
    float v = (float(x[c]) - mean) * rstd;
    if (a.weight) v *= weight_at(a.weight, a.wf32, c, x);
    if (a.bias) v += weight_at(a.bias, a.wf32, c, x);
    y[c] = E(v);
  }
}

// A block takes every gridDim.x-th row; its sums over rows collect in its own
// rows of part (dw, then db).
template <typename E>
__global__ __launch_bounds__(256) void norm_backward_loop_kernel(NormArgs a) {
  __shared__ float red[4];
  float* pw = a.dweight ? a.part + int64_t(blockIdx.x) * 2 * a.cols : nullptr;
  float* pb = a.dbias ? a.part + (int64_t(blockIdx.x) * 2 + 1) * a.cols : nullptr;
  // a thread comes back to the same columns for every row
  for (int c = threadIdx.x; c < a.cols; c += 256) {
    if (pw) pw[c] = 0.f;
    if (pb) pb[c] = 0.f;
  }
  for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
    const E* x = static_cast<const E*>(a.x) + r * a.ldx;
    const E* dy = static_cast<const E*>(a.dy) + r * a.lddy;
    const float mean = a.mean[r], rstd = a.rstd[r];
    float s1 = 0.f, s2 = 0.f;
    for (int c = threadIdx.x; c < a.cols; c += 256) {
      const float h = (float(x[c]) - mean) * rstd, d = float(dy[c]);
      const float g = a.weight ? d * weight_at(a.weight, a.wf32, c, x) : d;
      s1 += g;
      s2 = fmaf(g, h, s2);
      if (pw) pw[c] = fmaf(d, h, pw[c]);
      if (pb) pb[c] += d;
    }
    s1 = block_sum<256>(s1, red) / float(a.cols);
    s2 = block_sum<256>(s2, red) / float(a.cols);
    if (!a.dx) continue;
    E* dx = static_cast<E*>(a.dx) + r * a.lddx;
    for (int c = threadIdx.x; c < a.cols; c += 256) {
      const float h = (float(x[c]) - mean) * rstd, d = float(dy[c]);
      const float g = a.weight ? d * weight_at(a.weight, a.wf32, c, x) : d;
      dx[c] = E(rstd * (g - s1 - h * s2));
    }
  }
}

// Sums the blocks' partial rows in order: 64 columns per block, its 4 waves
// every fourth partial.  blockIdx.y: 0 for dw, 1 for db.
template <typename E>
__global__ __launch_bounds__(256) void norm_column_sum_kernel(NormArgs a, int blocks) {
  __shared__ float red[4][64];
  void* out = blockIdx.y ? a.dbias : a.dweight;
  if (!out) return;
  const int lane = threadIdx.x & 63, wid = threadIdx.x >> 6;
  const int col = blockIdx.x * 64 + lane;
  float s = 0.f;
  if (col < a.cols)
    for (int b = wid; b < blocks; b += 4) s += a.part[(int64_t(b) * 2 + blockIdx.y) * a.cols + col];
  red[wid][lane] = s;
  __syncthreads();
  if (wid || col >= a.cols) return;
  s = red[0][lane] + red[1][lane] + red[2][lane] + red[3][lane];
  if (a.wf32)
    static_cast<float*>(out)[col] = s;
  else
    static_cast<E*>(out)[col] = E(s);
}

template <typename E>
hipError_t forward(const NormArgs& a, hipStream_t st) {
  if (!a.rows) return hipSuccess;
  hipLaunchKernelGGL((norm_forward_loop_kernel<E>), dim3(unsigned(a.rows)), dim3(256), 0, st, a);
  return hipGetLastError();
}

template <typename E>
hipError_t backward(const NormArgs& a, hipStream_t st) {
  const int blocks = a.rows ? norm_blocks(a.rows, a.cols) : 0;
  if (blocks) {
    hipLaunchKernelGGL((norm_backward_loop_kernel<E>), dim3(unsigned(blocks)), dim3(256), 0, st, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (a.dweight || a.dbias)
    hipLaunchKernelGGL((norm_column_sum_kernel<E>), dim3(unsigned((int64_t(a.cols) + 63) / 64), 2), dim3(256), 0, st,
                       a, blocks);
  return hipGetLastError();
}

}  // namespace

int norm_blocks(int64_t rows, int64_t cols) {
  (void)cols;
  const int64_t n = (rows + 3) / 4;
  return int(n < 1 ? 1 : n < 1024 ? n : 1024);
}

hipError_t launch_norm_forward(bool bf16, const NormArgs& a, hipStream_t st) {
  return bf16 ? forward<__bf16>(a, st) : forward<float>(a, st);
}

hipError_t launch_norm_backward(bool bf16, const NormArgs& a, hipStream_t st) {
  return bf16 ? backward<__bf16>(a, st) : backward<float>(a, st);
}

}  // namespace layers
}  // namespace muon
