// dz = dy act'(z) and the bias gradient db = sum of dz's rows, in one pass
// over dy and z.
//
// A block owns 64 lanes x V columns and one chunk of rows; its 4 waves take
// every fourth row of the chunk, a lane V consecutive columns (16 bytes where
// the rows allow it).  The waves' column sums meet in LDS, the chunks' in a
// second kernel that adds them in order, so the sum does not depend on timing.
// The sums take dz before it is rounded.  dz itself is rounded to the operands'
// type, for the two products that read it to run on the matrix cores: in bf16
// that is one more rounding of 2^-8 on each of a sum's terms, about as much as
// the rounding of the sum.  Memory bound: reads dy and z, writes dz; 5832 x 4304 in
// bf16 28 us (5.3 TB/s), the column sums 4.7.
#include "device.h"

namespace muon {
namespace layers {
namespace {

constexpr int kWaves = 4;

template <typename E, int V>
struct alignas(sizeof(E) * V) Vec {
  E v[V];
};

template <typename E, int V, int ACT, bool SUM>
__global__ __launch_bounds__(256) void act_grad_kernel(ActGradArgs a, int chunk) {
  __shared__ float red[SUM ? kWaves : 1][SUM ? 64 * V : 1];
  const int lane = threadIdx.x & 63, wid = threadIdx.x >> 6;
  const int col = (blockIdx.x * 64 + lane) * V;
  const int r0 = blockIdx.y * chunk, r1 = min(a.rows, r0 + chunk);
  const bool on = col < a.N;
  float s[V] = {};
  if (on) {
    const E* dy = static_cast<const E*>(a.dy) + col;
    const E* z = static_cast<const E*>(a.z) + col;
    E* dz = static_cast<E*>(a.dz) + col;
    for (int r = r0 + wid; r < r1; r += kWaves) {
      const Vec<E, V> g = *reinterpret_cast<const Vec<E, V>*>(dy + r * a.lddy);
      Vec<E, V> zz, o;
      if constexpr (ACT != MUON_ACT_NONE) zz = *reinterpret_cast<const Vec<E, V>*>(z + r * a.ldz);
#pragma unroll
      for (int i = 0; i < V; ++i) {
        float v = float(g.v[i]);
        if constexpr (ACT != MUON_ACT_NONE) v *= act_grad_one<ACT>(float(zz.v[i]));
        o.v[i] = E(v);
        if constexpr (SUM) s[i] += v;
      }
      if constexpr (ACT != MUON_ACT_NONE) *reinterpret_cast<Vec<E, V>*>(dz + r * a.lddz) = o;
    }
  }
  if constexpr (SUM) {
#pragma unroll
    for (int i = 0; i < V; ++i) red[wid][lane * V + i] = s[i];
    __syncthreads();
    for (int i = threadIdx.x; i < 64 * V; i += 256) {
      const int c = blockIdx.x * 64 * V + i;
      if (c < a.N) a.part[int64_t(blockIdx.y) * a.N + c] = red[0][i] + red[1][i] + red[2][i] + red[3][i];
    }
  }
}

// Adds `chunks` rows of fp32 partial sums: 16 columns per block, a thread every
// 64th row of one of them, then their sums in order.
template <typename E>
__global__ __launch_bounds__(1024) void column_sum_kernel(const float* part, int chunks, int N, E* out) {
  __shared__ float red[64][17];
  const int c = threadIdx.x & 15, g = threadIdx.x >> 4;
  const int col = blockIdx.x * 16 + c;
  float s = 0.f;
  if (col < N) {
#pragma unroll 4
    for (int r = g; r < chunks; r += 64) s += part[int64_t(r) * N + col];
  }
  red[g][c] = s;
  __syncthreads();
  if (g || col >= N) return;
  s = 0.f;
#pragma unroll
  for (int i = 0; i < 64; ++i) s += red[i][c];
  out[col] = E(s);
}

// Chunks of rows: enough blocks to fill the chip a few times over, at least 16
// rows each.
int chunk_count(int64_t rows, int64_t N, int V) {
  const int64_t across = (N + 64 * V - 1) / (64 * V);
  const int64_t want = (1024 + across - 1) / across;
  const int64_t most = (rows + 15) / 16;
  const int64_t n = want < most ? want : most;
  return int(n < 1 ? 1 : n);
}

template <typename E, int V, bool SUM>
void launch_act(const ActGradArgs& a, dim3 g, int chunk, hipStream_t st) {
  const dim3 b{256};
  switch (a.z ? a.act : MUON_ACT_NONE) {
    case MUON_ACT_RELU: hipLaunchKernelGGL((act_grad_kernel<E, V, MUON_ACT_RELU, SUM>), g, b, 0, st, a, chunk); break;
    case MUON_ACT_GELU: hipLaunchKernelGGL((act_grad_kernel<E, V, MUON_ACT_GELU, SUM>), g, b, 0, st, a, chunk); break;
    case MUON_ACT_GELU_TANH:
      hipLaunchKernelGGL((act_grad_kernel<E, V, MUON_ACT_GELU_TANH, SUM>), g, b, 0, st, a, chunk);
      break;
    case MUON_ACT_SILU: hipLaunchKernelGGL((act_grad_kernel<E, V, MUON_ACT_SILU, SUM>), g, b, 0, st, a, chunk); break;
    default:
      if constexpr (SUM) hipLaunchKernelGGL((act_grad_kernel<E, V, MUON_ACT_NONE, true>), g, b, 0, st, a, chunk);
      break;
  }
}

template <typename E>
hipError_t launch(const ActGradArgs& a, hipStream_t st) {
  constexpr int W = 16 / sizeof(E);
  const auto fits = [](const void* p, int64_t ld) {
    return !p || (reinterpret_cast<uintptr_t>(p) % 16 == 0 && ld * int64_t(sizeof(E)) % 16 == 0);
  };
  const bool wide = a.N % W == 0 && fits(a.dy, a.lddy) && fits(a.z, a.ldz) && fits(a.dz, a.lddz);
  const int V = wide ? W : 1;
  const int want = act_grad_chunks(a.rows, a.N);
  const int chunk = a.rows ? (a.rows + want - 1) / want : 1;
  const int chunks = a.rows ? (a.rows + chunk - 1) / chunk : 0;
  const dim3 g{unsigned((int64_t(a.N) + 64 * V - 1) / (64 * V)), unsigned(chunks)};
  if (chunks) {
    if (wide) {
      if (a.dbias) launch_act<E, W, true>(a, g, chunk, st); else launch_act<E, W, false>(a, g, chunk, st);
    } else {
      if (a.dbias) launch_act<E, 1, true>(a, g, chunk, st); else launch_act<E, 1, false>(a, g, chunk, st);
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (a.dbias)
    hipLaunchKernelGGL((column_sum_kernel<E>), dim3(unsigned((int64_t(a.N) + 15) / 16)), dim3(1024), 0, st, a.part,
                       chunks, a.N, static_cast<E*>(a.dbias));
  return hipGetLastError();
}

}  // namespace

int act_grad_chunks(int64_t rows, int64_t N) {
  const int n = chunk_count(rows, N, 8);
  return n < 65535 ? n : 65535;
}

hipError_t launch_act_grad(bool bf16, const ActGradArgs& a, hipStream_t st) {
  return bf16 ? launch<__bf16>(a, st) : launch<float>(a, st);
}

}  // namespace layers
}  // namespace muon
