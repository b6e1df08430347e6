// Layer norm over the columns, forward and backward, for rows of any length,
// stride and alignment.
//
//   mean = sum x / n,  rstd = 1 / sqrt(sum (x - mean)^2 / n + eps)
//   y = (x - mean) rstd w + b
//   h = (x - mean) rstd,  g = dy w
//   dx = rstd (g - sum g / n - h sum(g h) / n),  dw = sum_rows dy h,  db = sum_rows dy
//
// All sums are fp32.  The variance is summed around the mean (a second pass),
// not as E[x^2] - mean^2, which cancels for rows far from 0.  Memory bound:
// 16384 x 4096 in bf16 49 us forward (5.4 TB/s) and 85 us backward (4.7 TB/s of x,
// dy and dx; its partial sums are another 25 MB), in fp32 94 and 158; 5832 x 1152
// 17 to 18 us backward (fp32: 19), where a wave has four rows and the chain of its loads
// and sums shows.
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
// one write.  T is 64 -- a wave per row, no barrier -- for short rows, then 256,
// 512 or 1024 threads.  A block holds a few rows at a time and takes every
// gridDim.x-th group of them; the next group's loads are issued before the
// current one is reduced, so that the memory never waits for the reductions.
// Loads and stores are 16 bytes at any alignment, and no load sits in a branch
// (which would end in a wait for it).
template <typename E>
struct __attribute__((packed, aligned(sizeof(E)))) Chunk {
  E v[16 / sizeof(E)];
};
template <typename E>
__device__ __forceinline__ Chunk<E> load_chunk(const E* p) {
  return *reinterpret_cast<const Chunk<E>*>(p);
}
// Thread t's chunk j of a row of n >= V columns: its first column, moved back
// where it would pass the row's end, and how many of its elements are then the
// chunk before's (V: all; they hold the same values, and count as 0 in sums).
struct Place {
  int col, dup;
};
template <int V, int T>
__device__ __forceinline__ Place place(int t, int j, int n) {
  const int want = (t + j * T) * V, col = min(want, n - V);
  return Place{col, want - col};
}
// V weights from column c on, as fp32 (`none` where there are none).
template <typename E>
__device__ __forceinline__ void load_weights(const void* w, int wf32, int c, float none,
                                             float (&v)[16 / sizeof(E)]) {
  constexpr int V = 16 / sizeof(E);
  if (!w) {
#pragma unroll
    for (int e = 0; e < V; ++e) v[e] = none;
  } else if (wf32) {
#pragma unroll
    for (int q = 0; q < V; q += 4) {
      const Chunk<float> x = load_chunk(static_cast<const float*>(w) + c + q);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[q + e] = x.v[e];
    }
  } else {
    const Chunk<E> x = load_chunk(static_cast<const E*>(w) + c);
#pragma unroll
    for (int e = 0; e < V; ++e) v[e] = float(x.v[e]);
  }
}

// Rows a block holds at a time, and its threads.
template <int T>
struct Shape {
  static constexpr int ROWS = T == 64 ? 4 : 1;
  static constexpr int THREADS = T * ROWS;
  static constexpr int WAVES = T / 64;   // of a row
};

// Sums of N values over the T threads of a row, the same for all of them.  buf:
// LDS for the waves' sums, N x THREADS / 64 floats that no wave may still read
// from an earlier sum (two buffers in turn: a barrier lies between their uses).
template <int T, int N>
__device__ __forceinline__ void row_sums(float (&v)[N], float* buf) {
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int d = 32; d; d >>= 1) v[i] += __shfl_xor(v[i], d);
  if constexpr (T > 64) {
    constexpr int W = Shape<T>::WAVES;
    const int wid = threadIdx.x >> 6;
    if ((threadIdx.x & 63) == 0) {
#pragma unroll
      for (int i = 0; i < N; ++i) buf[wid * N + i] = v[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = 0.f;
#pragma unroll
    for (int w = 0; w < W; ++w)
#pragma unroll
      for (int i = 0; i < N; ++i) v[i] += buf[(wid / W * W + w) * N + i];
  }
}

template <typename E, int NV, int T>
__global__ __launch_bounds__(Shape<T>::THREADS) void norm_forward_kernel(NormArgs a) {
  using S = Shape<T>;
  constexpr int V = 16 / int(sizeof(E));
  __shared__ float red[2][S::THREADS / 64];
  const int t = threadIdx.x % T;
  const int64_t step = int64_t(gridDim.x) * S::ROWS;
  float w[NV][V], b[NV][V];
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int col = place<V, T>(t, j, a.cols).col;
    load_weights<E>(a.weight, a.wf32, col, 1.f, w[j]);
    load_weights<E>(a.bias, a.wf32, col, 0.f, b[j]);
  }
  Chunk<E> next[NV];
  auto load = [&](int64_t r) {
    const E* x = static_cast<const E*>(a.x) + min(r, int64_t(a.rows) - 1) * a.ldx;
#pragma unroll
    for (int j = 0; j < NV; ++j) next[j] = load_chunk(x + place<V, T>(t, j, a.cols).col);
  };
  // (rows past the last read it again)
  int64_t r = int64_t(blockIdx.x) * S::ROWS + threadIdx.x / T;
  load(r);
  for (int64_t first = int64_t(blockIdx.x) * S::ROWS; first < a.rows; first += step, r += step) {
    Chunk<E> c[NV];
#pragma unroll
    for (int j = 0; j < NV; ++j) c[j] = next[j];
    load(r + step);
    float s[1] = {0.f};
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int dup = place<V, T>(t, j, a.cols).dup;
#pragma unroll
      for (int e = 0; e < V; ++e) s[0] += e >= dup ? float(c[j].v[e]) : 0.f;
    }
    row_sums<T>(s, red[0]);
    const float mean = s[0] / float(a.cols);
    s[0] = 0.f;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int dup = place<V, T>(t, j, a.cols).dup;
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const float d = e >= dup ? float(c[j].v[e]) - mean : 0.f;
        s[0] = fmaf(d, d, s[0]);
      }
    }
    row_sums<T>(s, red[1]);
    const float rstd = 1.f / sqrtf(s[0] / float(a.cols) + a.eps);
    if (r >= a.rows) continue;
    if (t == 0) {
      if (a.mean) a.mean[r] = mean;
      if (a.rstd) a.rstd[r] = rstd;
    }
    E* y = static_cast<E*>(a.y) + r * a.ldy;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const Place at = place<V, T>(t, j, a.cols);
      Chunk<E> o;
#pragma unroll
      for (int e = 0; e < V; ++e) o.v[e] = E(fmaf((float(c[j].v[e]) - mean) * rstd, w[j][e], b[j][e]));
      if (at.dup < V) *reinterpret_cast<Chunk<E>*>(y + at.col) = o;
    }
  }
}

// The columns' sums over a block's rows stay in registers; at the end its rows'
// threads add theirs in order through LDS, into the block's rows of part.  SUMS:
// whether dw and db are wanted.  The weights lie in LDS in fp32: the registers
// they would take are worth another wave, and read from the caches for each row
// they would hold up both its passes.
template <typename E, int NV, int T, bool SUMS>
__global__ __launch_bounds__(Shape<T>::THREADS, T < 1024 && NV * 16 / sizeof(E) <= 16 ? 3 : 1) void
norm_backward_kernel(NormArgs a) {
  using S = Shape<T>;
  constexpr int V = 16 / int(sizeof(E));
  __shared__ float red[2][2 * S::THREADS / 64];
  __shared__ __attribute__((aligned(16))) float sums[SUMS && S::ROWS > 1 ? S::ROWS : 1][SUMS && S::ROWS > 1 ? T * NV * V : 1];
  // thread t's chunk j at (j T + t) V, as it holds it
  __shared__ __attribute__((aligned(16))) float weights[T * NV * V];
  const int t = threadIdx.x % T, row = threadIdx.x / T;
  auto weight = [&](int j, float (&v)[V]) {
#pragma unroll
    for (int q = 0; q < V; q += 4) {
      typedef float f4 __attribute__((ext_vector_type(4)));
      const f4 x = *reinterpret_cast<const f4*>(weights + (j * T + t) * V + q);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[q + e] = x[e];
    }
  };
  const int64_t step = int64_t(gridDim.x) * S::ROWS;
  float pw[NV][V], pb[NV][V];
#pragma unroll
  for (int j = 0; j < NV; ++j)
#pragma unroll
    for (int e = 0; e < V; ++e) pw[j][e] = pb[j][e] = 0.f;
  // (with 512 threads the registers hold one row only)
  constexpr bool AHEAD = T < 512;
  Chunk<E> x[NV], d[NV];
  float mean = 0.f, rstd = 0.f;
  auto load = [&](int64_t r) {
    const int64_t at = min(r, int64_t(a.rows) - 1);
    const E* xp = static_cast<const E*>(a.x) + at * a.ldx;
    const E* dp = static_cast<const E*>(a.dy) + at * a.lddy;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int col = place<V, T>(t, j, a.cols).col;
      x[j] = load_chunk(xp + col);
      d[j] = load_chunk(dp + col);
    }
    mean = a.mean[at];
    rstd = a.rstd[at];
  };
  int64_t r = int64_t(blockIdx.x) * S::ROWS + row;
  if constexpr (AHEAD) load(r);
  if (row == 0) {
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      float v[V];
      load_weights<E>(a.weight, a.wf32, place<V, T>(t, j, a.cols).col, 1.f, v);
#pragma unroll
      for (int e = 0; e < V; ++e) weights[(j * T + t) * V + e] = v[e];
    }
  }
  __syncthreads();
  int turn = 0;
  for (int64_t first = int64_t(blockIdx.x) * S::ROWS; first < a.rows; first += step, r += step, turn ^= 1) {
    if constexpr (!AHEAD) load(r);
    Chunk<E> xr[NV], dr[NV];
    const float m = mean, rs = rstd;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      xr[j] = x[j];
      dr[j] = d[j];
    }
    if constexpr (AHEAD) load(r + step);
    // (read anew in each pass, not kept in registers)
    asm volatile("" ::: "memory");
    float s[2] = {0.f, 0.f};
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      float w[V];
      const Place at = place<V, T>(t, j, a.cols);
      weight(j, w);
      const int from = r < a.rows ? at.dup : V;   // (nothing of rows past the last)
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const float h = (float(xr[j].v[e]) - m) * rs, dd = float(dr[j].v[e]);
        if (e < from) continue;
        const float g = dd * w[e];
        s[0] += g;
        s[1] = fmaf(g, h, s[1]);
        if constexpr (SUMS) {
          pw[j][e] = fmaf(dd, h, pw[j][e]);
          pb[j][e] += dd;
        }
      }
    }
    row_sums<T>(s, red[turn]);
    asm volatile("" ::: "memory");
    const float s1 = s[0] / float(a.cols), s2 = s[1] / float(a.cols);
    if (a.dx && r < a.rows) {
      E* dx = static_cast<E*>(a.dx) + r * a.lddx;
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        float w[V];
        const Place at = place<V, T>(t, j, a.cols);
        weight(j, w);
        Chunk<E> o;
#pragma unroll
        for (int e = 0; e < V; ++e) {
          const float h = (float(xr[j].v[e]) - m) * rs;
          o.v[e] = E(rs * (float(dr[j].v[e]) * w[e] - s1 - h * s2));
        }
        if (at.dup < V) *reinterpret_cast<Chunk<E>*>(dx + at.col) = o;
      }
    }
  }
  if constexpr (SUMS) {
    typedef float f4 __attribute__((ext_vector_type(4)));
    struct __attribute__((packed, aligned(4))) P4 {
      f4 v;
    };
    for (int k = 0; k < 2; ++k) {
      float* part = a.part + (int64_t(blockIdx.x) * 2 + k) * a.cols;
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        float v[V];
#pragma unroll
        for (int e = 0; e < V; ++e) v[e] = k ? pb[j][e] : pw[j][e];
        if constexpr (S::ROWS > 1) {
          // (as the threads hold them)
#pragma unroll
          for (int q = 0; q < V; q += 4)
            *reinterpret_cast<f4*>(&sums[row][(j * T + t) * V + q]) = f4{v[q], v[q + 1], v[q + 2], v[q + 3]};
        } else {
          const Place at = place<V, T>(t, j, a.cols);
          if (at.dup == 0) {
#pragma unroll
            for (int q = 0; q < V; q += 4)
              *reinterpret_cast<P4*>(part + at.col + q) = P4{f4{v[q], v[q + 1], v[q + 2], v[q + 3]}};
          } else {
#pragma unroll
            for (int e = 0; e < V; ++e)
              if (e >= at.dup) part[at.col + e] = v[e];
          }
        }
      }
      if constexpr (S::ROWS > 1) {
        __syncthreads();
        const int whole = a.cols / V * V;   // the columns from here on lie in a chunk that was moved back
        for (int c = threadIdx.x; c < a.cols; c += S::THREADS) {
          const int at = c < whole ? c : whole + c - (a.cols - V);
          float v = 0.f;
#pragma unroll
          for (int q = 0; q < S::ROWS; ++q) v += sums[q][at];
          part[c] = v;
        }
        __syncthreads();
      }
    }
  }
}

// Other rows: read again for each sum.
template <typename E>
__global__ __launch_bounds__(256) void norm_forward_loop_kernel(NormArgs a) {
  __shared__ float red[4];
  for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
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

// Sums the blocks' partial rows: 32 columns per block, a thread every 32nd
// partial of one of them, then their sums in order.  blockIdx.y: 0 for dw, 1 for db.
template <typename E>
__global__ __launch_bounds__(1024) void norm_column_sum_kernel(NormArgs a, int blocks) {
  __shared__ float red[32][33];
  void* out = blockIdx.y ? a.dbias : a.dweight;
  if (!out) return;
  const int c = threadIdx.x & 31, g = threadIdx.x >> 5;
  const int col = blockIdx.x * 32 + c;
  float s = 0.f;
  if (col < a.cols) {
#pragma unroll 8
    for (int b = g; b < blocks; b += 32) s += a.part[(int64_t(b) * 2 + blockIdx.y) * a.cols + col];
  }
  red[g][c] = s;
  __syncthreads();
  if (g || col >= a.cols) return;
  s = 0.f;
#pragma unroll
  for (int i = 0; i < 32; ++i) s += red[i][c];
  if (a.wf32)
    static_cast<float*>(out)[col] = s;
  else
    static_cast<E*>(out)[col] = E(s);
}

// Threads per row, so that a thread holds at most 32 elements (16 with 1024
// threads) forward, 24 (32 with 512 threads, which hold no second row) backward,
// where the sums take registers too.  0: the row
// does not fit, or is shorter than a chunk.
int forward_threads(int64_t cols) {
  return cols < 8 || cols > 16384 ? 0 : cols <= 2048 ? 64 : cols <= 8192 ? 256 : 1024;
}
int backward_threads(int64_t cols) {
  return cols < 8 || cols > 16384 ? 0 : cols <= 1536 ? 64 : cols <= 6144 ? 256 : 512;
}

// f(chunks per thread tag, threads tag) for rows of `cols` on t threads (64, 256 or
// MOST): the
// smallest chunk count that covers them, in quarters of 32 elements.
template <typename E, int MOST, class F>
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
  else at(IntTag<MOST>{});
}

template <typename E>
hipError_t forward(const NormArgs& a, hipStream_t st) {
  if (!a.rows) return hipSuccess;
  const int t = forward_threads(a.cols);
  if (!t) {
    const unsigned blocks = unsigned(a.rows < 65536 ? a.rows : 65536);
    hipLaunchKernelGGL((norm_forward_loop_kernel<E>), dim3(blocks), dim3(256), 0, st, a);
  } else {
    with_shape<E, 1024>(a.cols, t, [&](auto nv, auto tt) {
      using S = Shape<decltype(tt)::value>;
      // 2048 threads per CU: what the chip holds of rows of one chunk per thread (54 to
      // 62 registers); of two to four bf16 chunks a thread has 84 to 164, and 3 to 5
      // blocks of 256 run at a time (fp32: 62 to 184, 2 to 8)
      const int64_t groups = (int64_t(a.rows) + S::ROWS - 1) / S::ROWS, most = int64_t(kCUs) * 2048 / S::THREADS;
      const dim3 g{unsigned(groups < most ? groups : most)}, b{S::THREADS};
      // (1024 threads hold 16 elements each: forward_threads)
      constexpr int NV = decltype(nv)::value;
      if constexpr (S::WAVES < 16 || NV * 16 / int(sizeof(E)) <= 16)
        hipLaunchKernelGGL((norm_forward_kernel<E, NV, decltype(tt)::value>), g, b, 0, st, a);
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
      with_shape<E, 512>(a.cols, t, [&](auto nv, auto tt) {
        constexpr int NV = decltype(nv)::value, TT = decltype(tt)::value;
        const dim3 g{unsigned(blocks)}, b{Shape<TT>::THREADS};
        // (a thread holds no more: backward_threads)
        if constexpr (NV * 16 / int(sizeof(E)) <= (TT == 512 ? 32 : 24)) {
          if (a.dweight || a.dbias)
            hipLaunchKernelGGL((norm_backward_kernel<E, NV, TT, true>), g, b, 0, st, a);
          else
            hipLaunchKernelGGL((norm_backward_kernel<E, NV, TT, false>), g, b, 0, st, a);
        }
      });
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (a.dweight || a.dbias)
    hipLaunchKernelGGL((norm_column_sum_kernel<E>), dim3(unsigned((int64_t(a.cols) + 31) / 32), 2), dim3(1024), 0, st,
                       a, blocks);
  return hipGetLastError();
}

}  // namespace

// Blocks of the backward pass: 3 of 256 threads, 1 of 512 per CU, and at least four
// rows per thread group, so that their partial sums stay few.  The chip holds them all
// at once but for fp32 rows of 1025 to 1536 and of 4097 to 6144 columns, whose threads
// take 190 and 206 registers: two of their blocks fit on a CU, the others follow.
int norm_blocks(int64_t rows, int64_t cols) {
  const int t = backward_threads(cols);
  const int64_t group = t == 64 ? 4 : 1, most = kCUs * (t == 512 ? 1 : 3);
  const int64_t n = (rows + 4 * group - 1) / (4 * group);
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
