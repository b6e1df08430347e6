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

// Rows that fit the registers of T threads stay there: one read of x (and dy),
// one write.  T is 64 -- a wave per row, four rows per block, no barrier -- for
// short rows, then a block of 256 or 1024 threads per row.  Loads and stores are 16 bytes at any alignment;
// a row's last, partial chunk is moved element by element.
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
template <typename E>
struct __attribute__((packed, aligned(sizeof(E)))) Chunk {
  E v[16 / sizeof(E)];
};
template <typename E>
__device__ __forceinline__ Chunk<E> load_chunk(const E* p, int n) {   // n: elements that exist
  constexpr int V = 16 / sizeof(E);
  Chunk<E> c;
  if (n >= V) {
    c = *reinterpret_cast<const Chunk<E>*>(p);
  } else {
#pragma unroll
    for (int e = 0; e < V; ++e) c.v[e] = e < n ? p[e] : E(0.f);
  }
  return c;
}
template <typename E>
__device__ __forceinline__ void store_chunk(E* p, int n, const Chunk<E>& c) {
  constexpr int V = 16 / sizeof(E);
  if (n >= V) {
    *reinterpret_cast<Chunk<E>*>(p) = c;
  } else {
#pragma unroll
    for (int e = 0; e < V; ++e)
      if (e < n) p[e] = c.v[e];
  }
}
// V weights from column c on, as fp32 (1 or 0 where there are none).
template <typename E>
__device__ __forceinline__ void load_weights(const void* w, int wf32, int c, int n, float none,
                                             float (&v)[16 / sizeof(E)]) {
  constexpr int V = 16 / sizeof(E);
#pragma unroll
  for (int e = 0; e < V; ++e) v[e] = none;
  if (!w || n <= 0) return;
  if (wf32) {
#pragma unroll
    for (int q = 0; q < V; q += 4) {
      const Chunk<float> x = load_chunk(static_cast<const float*>(w) + c + q, n - q);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[q + e] = x.v[e];
    }
  } else {
    const Chunk<E> x = load_chunk(static_cast<const E*>(w) + c, n);
#pragma unroll
    for (int e = 0; e < V; ++e) v[e] = float(x.v[e]);
  }
}

template <typename E, int NV, int T>
__global__ __launch_bounds__(T < 256 ? 256 : T) void norm_forward_kernel(NormArgs a) {
  constexpr int V = 16 / int(sizeof(E));
  __shared__ float red[T / 64];
  const int t = T == 64 ? threadIdx.x & 63 : threadIdx.x;
  const int64_t r = T == 64 ? int64_t(blockIdx.x) * 4 + (threadIdx.x >> 6) : blockIdx.x;
  if (r >= a.rows) return;
  const E* x = static_cast<const E*>(a.x) + r * a.ldx;
  Chunk<E> c[NV];
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int col = (t + j * T) * V;
    c[j] = load_chunk(x + col, a.cols - col);
  }
  float s = 0.f;
#pragma unroll
  for (int j = 0; j < NV; ++j)
#pragma unroll
    for (int e = 0; e < V; ++e) s += float(c[j].v[e]);
  const float mean = block_sum<T>(s, red) / float(a.cols);
  s = 0.f;
#pragma unroll
  for (int j = 0; j < NV; ++j)
#pragma unroll
    for (int e = 0; e < V; ++e) {
      const float d = (t + j * T) * V + e < a.cols ? float(c[j].v[e]) - mean : 0.f;
      s = fmaf(d, d, s);
    }
  const float rstd = 1.f / sqrtf(block_sum<T>(s, red) / float(a.cols) + a.eps);
  if (t == 0) {
    if (a.mean) a.mean[r] = mean;
    if (a.rstd) a.rstd[r] = rstd;
  }
  E* y = static_cast<E*>(a.y) + r * a.ldy;
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int col = (t + j * T) * V, n = a.cols - col;
    float w[V], b[V];
    load_weights<E>(a.weight, a.wf32, col, n, 1.f, w);
    load_weights<E>(a.bias, a.wf32, col, n, 0.f, b);
    Chunk<E> o;
#pragma unroll
    for (int e = 0; e < V; ++e) o.v[e] = E(fmaf((float(c[j].v[e]) - mean) * rstd, w[e], b[e]));
    store_chunk(y + col, n, o);
  }
}

// A block (T 64: each of its four waves) takes every gridDim.x-th (4
// gridDim.x-th) row and keeps its columns' sums over those rows in registers;
// they go to the block's rows of part at the end (T 64: the waves' sums added in
// order through LDS).  SUMS: whether dw and db are wanted.  The next row's loads
// are issued before the current row is reduced, and the weights stay in
// registers, except with 1024 threads, which have 128 registers each.
template <typename E, int NV, int T, bool SUMS>
__global__ __launch_bounds__(T < 256 ? 256 : T) void norm_backward_kernel(NormArgs a) {
  constexpr int V = 16 / int(sizeof(E));
  constexpr int ROWS = T == 64 ? 4 : 1;
  __shared__ float red[2][T / 64];
  __shared__ float sums[SUMS && T == 64 ? 64 * NV * V : 1];
  const int t = T == 64 ? threadIdx.x & 63 : threadIdx.x, wid = threadIdx.x >> 6;
  const int64_t r0 = int64_t(blockIdx.x) * ROWS + (T == 64 ? wid : 0), step = int64_t(gridDim.x) * ROWS;
  constexpr bool AHEAD = T < 1024;
  float w[AHEAD ? NV : 1][V], pw[NV][V], pb[NV][V];
  auto weights = [&](int j, float (&v)[V]) {
    const int col = (t + j * T) * V;
    load_weights<E>(a.weight, a.wf32, col, a.cols - col, 1.f, v);
  };
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    if constexpr (AHEAD) weights(j, w[j]);
#pragma unroll
    for (int e = 0; e < V; ++e) pw[j][e] = pb[j][e] = 0.f;
  }
  Chunk<E> x[NV], d[NV];
  float mean = 0.f, rstd = 0.f;
  auto load = [&](int64_t r) {
    if (r >= a.rows) return;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int col = (t + j * T) * V;
      x[j] = load_chunk(static_cast<const E*>(a.x) + r * a.ldx + col, a.cols - col);
      d[j] = load_chunk(static_cast<const E*>(a.dy) + r * a.lddy + col, a.cols - col);
    }
    mean = a.mean[r];
    rstd = a.rstd[r];
  };
  if constexpr (AHEAD) load(r0);
  for (int64_t r = r0; r < a.rows; r += step) {
    if constexpr (!AHEAD) load(r);
    float s1 = 0.f, s2 = 0.f;
    Chunk<E> xr[NV], dr[NV];
    const float m = mean, rs = rstd;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      xr[j] = x[j];
      dr[j] = d[j];
    }
    if constexpr (AHEAD) load(r + step);
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      float(&wj)[V] = w[AHEAD ? j : 0];
      if constexpr (!AHEAD) weights(j, wj);
#pragma unroll
      for (int e = 0; e < V; ++e) {
        // (past the last column dy is 0)
        const float h = (float(xr[j].v[e]) - m) * rs, dd = float(dr[j].v[e]), g = dd * wj[e];
        s1 += g;
        s2 = fmaf(g, h, s2);
        if constexpr (SUMS) {
          pw[j][e] = fmaf(dd, h, pw[j][e]);
          pb[j][e] += dd;
        }
      }
    }
    s1 = block_sum<T>(s1, red[0]) / float(a.cols);
    s2 = block_sum<T>(s2, red[1]) / float(a.cols);
    if (a.dx) {
      E* dx = static_cast<E*>(a.dx) + r * a.lddx;
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        const int col = (t + j * T) * V;
        float(&wj)[V] = w[AHEAD ? j : 0];
        if constexpr (!AHEAD) weights(j, wj);
        Chunk<E> o;
#pragma unroll
        for (int e = 0; e < V; ++e) {
          const float h = (float(xr[j].v[e]) - m) * rs;
          o.v[e] = E(rs * (float(dr[j].v[e]) * wj[e] - s1 - h * s2));
        }
        store_chunk(dx + col, a.cols - col, o);
      }
    }
  }
  if constexpr (SUMS) {
    for (int k = 0; k < 2; ++k) {
      float* part = a.part + (int64_t(blockIdx.x) * 2 + k) * a.cols;
      if constexpr (T == 64) {
        for (int q = 0; q < 4; ++q) {
          if (wid == q) {
#pragma unroll
            for (int j = 0; j < NV; ++j)
#pragma unroll
              for (int e = 0; e < V; ++e) {
                float& at = sums[(t + j * T) * V + e];
                at = (q ? at : 0.f) + (k ? pb[j][e] : pw[j][e]);
              }
          }
          __syncthreads();
        }
        for (int c = threadIdx.x; c < a.cols; c += 256) part[c] = sums[c];
        __syncthreads();
      } else {
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
          for (int e = 0; e < V; ++e) {
            const int col = (t + j * T) * V + e;
            if (col < a.cols) part[col] = k ? pb[j][e] : pw[j][e];
          }
      }
    }
  }
}

// Longer rows: read again for each sum.
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

// Sums the blocks' partial rows in order: 64 columns per block, its 16 waves
// every 16th partial.  blockIdx.y: 0 for dw, 1 for db.
template <typename E>
__global__ __launch_bounds__(1024) void norm_column_sum_kernel(NormArgs a, int blocks) {
  __shared__ float red[16][64];
  void* out = blockIdx.y ? a.dbias : a.dweight;
  if (!out) return;
  const int lane = threadIdx.x & 63, wid = threadIdx.x >> 6;
  const int col = blockIdx.x * 64 + lane;
  float s = 0.f;
  if (col < a.cols) {
#pragma unroll 8
    for (int b = wid; b < blocks; b += 16) s += a.part[(int64_t(b) * 2 + blockIdx.y) * a.cols + col];
  }
  red[wid][lane] = s;
  __syncthreads();
  if (wid || col >= a.cols) return;
  s = 0.f;
#pragma unroll
  for (int i = 0; i < 16; ++i) s += red[i][lane];
  if (a.wf32)
    static_cast<float*>(out)[col] = s;
  else
    static_cast<E*>(out)[col] = E(s);
}

// Threads per row, so that a thread holds at most 32 elements forward, 24 (16
// with 1024 threads) backward, where the sums take registers too.  0: the row
// does not fit.
int forward_threads(int64_t cols) { return cols <= 2048 ? 64 : cols <= 8192 ? 256 : cols <= 32768 ? 1024 : 0; }
int backward_threads(int64_t cols) { return cols <= 1536 ? 64 : cols <= 6144 ? 256 : cols <= 16384 ? 1024 : 0; }

// f(chunks per thread tag, threads tag) for rows of `cols` on t threads: the
// smallest chunk count that covers them, in quarters of 32 elements.
template <typename E, class F>
void with_shape(int64_t cols, int t, F f) {
  constexpr int V = 16 / int(sizeof(E)), Q = 8 / V;
  const int64_t nv = (cols + int64_t(V) * t - 1) / (int64_t(V) * t);
  const auto at = [&](auto threads) {
    if (nv <= Q) f(IntTag<Q>{}, threads);
    else if (nv <= 2 * Q) f(IntTag<2 * Q>{}, threads);
    else if (nv <= 3 * Q) f(IntTag<3 * Q>{}, threads);
    else f(IntTag<4 * Q>{}, threads);
  };
  if (t == 64) at(IntTag<64>{});
  else if (t == 256) at(IntTag<256>{});
  else at(IntTag<1024>{});
}

template <typename E>
hipError_t forward(const NormArgs& a, hipStream_t st) {
  if (!a.rows) return hipSuccess;
  const int t = forward_threads(a.cols);
  if (!t) {
    hipLaunchKernelGGL((norm_forward_loop_kernel<E>), dim3(unsigned(a.rows)), dim3(256), 0, st, a);
  } else {
    const dim3 g{unsigned(t == 64 ? (a.rows + 3) / 4 : a.rows)}, b{unsigned(t == 64 ? 256 : t)};
    with_shape<E>(a.cols, t, [&](auto nv, auto tt) {
      hipLaunchKernelGGL((norm_forward_kernel<E, decltype(nv)::value, decltype(tt)::value>), g, b, 0, st, a);
    });
  }
  return hipGetLastError();
}

template <typename E>
hipError_t backward(const NormArgs& a, hipStream_t st) {
  const int blocks = a.rows ? norm_blocks(a.rows, a.cols) : 0;
  const int t = backward_threads(a.cols);
  if (blocks) {
    if (!t) {
      hipLaunchKernelGGL((norm_backward_loop_kernel<E>), dim3(unsigned(blocks)), dim3(256), 0, st, a);
    } else {
      const dim3 g{unsigned(blocks)}, b{unsigned(t == 64 ? 256 : t)};
      with_shape<E>(a.cols, t, [&](auto nv, auto tt) {
        constexpr int NV = decltype(nv)::value, TT = decltype(tt)::value;
        if constexpr (NV * 16 / int(sizeof(E)) > (TT == 1024 ? 16 : 24)) return;   // (never: backward_threads)
        else if (a.dweight || a.dbias)
          hipLaunchKernelGGL((norm_backward_kernel<E, NV, TT, true>), g, b, 0, st, a);
        else
          hipLaunchKernelGGL((norm_backward_kernel<E, NV, TT, false>), g, b, 0, st, a);
      });
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (a.dweight || a.dbias)
    hipLaunchKernelGGL((norm_column_sum_kernel<E>), dim3(unsigned((int64_t(a.cols) + 63) / 64), 2), dim3(1024), 0, st,
                       a, blocks);
  return hipGetLastError();
}

}  // namespace

// Blocks of the backward pass: two to four rows per wave at least, no more
// blocks than keep the chip full (their partial sums are written and read too).
int norm_blocks(int64_t rows, int64_t cols) {
  const int t = backward_threads(cols);
  const int64_t per = t == 64 ? 8 : 4, most = t == 64 ? 1024 : t == 1024 ? 256 : 512;
  const int64_t n = (rows + per - 1) / per;
  return int(n < 1 ? 1 : n < most ? n : most);
}

hipError_t launch_norm_forward(bool bf16, const NormArgs& a, hipStream_t st) {
  return bf16 ? forward<__bf16>(a, st) : forward<float>(a, st);
}

hipError_t launch_norm_backward(bool bf16, const NormArgs& a, hipStream_t st) {
  return bf16 ? backward<__bf16>(a, st) : backward<float>(a, st);
}

}  // namespace layers
}  // namespace muon
