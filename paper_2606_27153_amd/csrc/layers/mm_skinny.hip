// Matrix products with few rows: one token, a decode batch, an expert with a
// handful of tokens.  C = A B with A row (K-contiguous), B row or tr.
//
// The weight is read once and everything else is small, so the kernel is bound
// by the stream of B, which goes from memory straight into MFMA operand
// registers: no LDS, no barrier in the loop, every alignment.  One token through
// a 4096 x 14336 bf16 weight takes 23 us, 5.1 TB/s, what a large copy reaches (fp32:
// 40 us); 48 rows over 64 experts of 2048 x 1408 37 us (5.5 TB/s; fp32: 83).  A block
// owns 16 MT rows and COLS columns of C (128 in bf16, 64 in fp32) over a range of K,
// which its four waves cut into four; their sums meet in LDS at the end.
// Ranges of K on different blocks (splits) leave fp32 partial results that
// mm_reduce_kernel adds in order.
//
// bf16, a K step of 32 with 16 x 16 x 32 MFMAs: lane l holds 8 consecutive K from
// k0 + 8 (l / 16) on.  B row: 16 bytes of column 16 b + l % 16 are the operand
// of column block b.  B tr: 16 bytes are 8 columns, 8 (l % 16) on, of one K;
// eight of them (K k0 + 8 (l / 16) + i) are transposed in registers, one v_perm
// for every two elements, into the operands of 8 column blocks that hold every
// eighth column.  fp32: 16 x 16 x 4 MFMAs, a K step of 16, where one K per lane
// and operand needs no transposition.
#include "../ns_gemm_kernel.h"
#include "device.h"

namespace muon {
namespace layers {
namespace {

constexpr int kWaves = 4;

template <typename E>
struct __attribute__((packed, aligned(sizeof(E)))) Chunk {   // 16 bytes at any alignment
  E v[16 / sizeof(E)];
};
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// 16 bytes from p, of which the first n elements exist (the others are 0).
template <typename E>
__device__ __forceinline__ u32x4 load_chunk(const E* p, int n) {
  constexpr int EPC = 16 / sizeof(E);
  Chunk<E> c;
  if (n >= EPC) {
    c = *reinterpret_cast<const Chunk<E>*>(p);
  } else {
#pragma unroll
    for (int e = 0; e < EPC; ++e) c.v[e] = e < n ? p[e] : E(0.f);
  }
  return __builtin_bit_cast(u32x4, c);
}

template <typename E, int MT, bool BTR, int GROUP>
struct Skinny {
  static constexpr int EPC = 16 / int(sizeof(E));
  static constexpr int BK = 4 * EPC;                 // K step
  static constexpr int NB = EPC;                     // column blocks of 16
  static constexpr int COLS = 16 * NB;

  // Operands of one K step as they come from memory: b[i] is column block i (B
  // row) or K EPC g + i of EPC columns (B tr).
  struct Step {
    u32x4 a[MT], b[EPC];
  };
  // One lane's place: its row of A per row tile, its column(s) of B.
  const E* a[MT];
  const E* b[BTR ? 1 : NB];
  int64_t ldb;
  int g;

  // The step at element k of the operands' rows; TAIL: K ends at k1, within it.
  template <bool TAIL>
  __device__ __forceinline__ void load(int k, int k1, Step& s) const {
    const int kk = k + g * EPC, n = TAIL ? k1 - kk : EPC;
#pragma unroll
    for (int t = 0; t < MT; ++t) s.a[t] = load_chunk(a[t] + kk, n);
    if constexpr (BTR) {
      const E* q = b[0] + kk * ldb;
#pragma unroll
      for (int i = 0; i < EPC; ++i) s.b[i] = load_chunk(q + i * ldb, i < n ? EPC : 0);
    } else {
#pragma unroll
      for (int i = 0; i < NB; ++i) s.b[i] = load_chunk(b[i] + kk, n);
    }
  }
  __device__ __forceinline__ void multiply(const Step& s, f32x4 (&acc)[NB][MT]) const {
    if constexpr (sizeof(E) == 2) {
#pragma unroll
      for (int i = 0; i < NB; ++i) {
        u32x4 f;
        if constexpr (BTR) {
#pragma unroll
          for (int p = 0; p < 4; ++p)
            f[p] = __builtin_amdgcn_perm(s.b[2 * p + 1][i / 2], s.b[2 * p][i / 2], i & 1 ? 0x07060302 : 0x05040100);
        } else {
          f = s.b[i];
        }
#pragma unroll
        for (int t = 0; t < MT; ++t)
          acc[i][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, s.a[t]),
                                                              __builtin_bit_cast(bf16x8, f), acc[i][t], 0, 0, 0);
      }
    } else {
      // MFMA q takes K k0 + 4 g + q of both operands
#pragma unroll
      for (int q = 0; q < 4; ++q)
#pragma unroll
        for (int i = 0; i < NB; ++i)
#pragma unroll
          for (int t = 0; t < MT; ++t) {
            const uint32_t av = s.a[t][q], bv = BTR ? s.b[q][i] : s.b[i][q];
            acc[i][t] = __builtin_amdgcn_mfma_f32_16x16x4f32(__builtin_bit_cast(float, av),
                                                             __builtin_bit_cast(float, bv), acc[i][t], 0, 0, 0);
          }
    }
  }
};

template <typename E>
__device__ __forceinline__ void finish8(const Product& p, int64_t m, int64_t c, int n, float (&v)[8]) {
  if (p.bias) {
    const E* b = static_cast<const E*>(p.bias) + c;
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < n) v[e] += float(b[e]);
  }
  if (p.z) store8(static_cast<E*>(p.z) + m * p.ldz + c, n, v);
  with_act(p.act, [&](auto tag) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = act_one<decltype(tag)::value>(v[e]);
  });
  if (p.res) {
    float r[8];
    load8(static_cast<const E*>(p.res) + m * p.ldr + c, n, r);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] += r[e];
  }
  store8(static_cast<E*>(p.c) + m * p.ldc + c, n, v);
}

template <typename E, int MT, bool BTR, int GROUP>
__global__ __launch_bounds__(256, MT == 4 ? 1 : 2) void mm_skinny_kernel(Product p, typename TableOf<GROUP>::T tab) {
  using S = Skinny<E, MT, BTR, GROUP>;
  constexpr int ROWS = 16 * MT, LD = S::COLS + 4;
  __shared__ __attribute__((aligned(16))) float red[2][ROWS * LD];
  const int lane = threadIdx.x & 63, wid = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int strips = (p.N + S::COLS - 1) / S::COLS;
  const int n0 = int(blockIdx.x) % strips * S::COLS, cols = min(S::COLS, p.N - n0);
  int64_t m0 = int64_t(blockIdx.x) / strips * ROWS;
  int rows = int(min(int64_t(ROWS), p.M - m0));
  const E* b = static_cast<const E*>(p.b);
  int K = p.K;
  if constexpr (GROUP == GROUP_ROWS) {
    RowTile t;
    if (!find_row_tile<ROWS>(p.offsets, p.experts, p.M, int(blockIdx.x) / strips, lane, t)) return;
    m0 = t.row0;
    rows = t.rows;
    if (t.expert < 0) K = 0;
    b = static_cast<const E*>(tab.p[max(t.expert, 0)]);
  }
  // this wave's range of K: whole steps
  const int steps = (K + S::BK - 1) / S::BK, parts = p.splits * kWaves;
  const int per = (steps + parts - 1) / parts * S::BK;
  const int k0 = min(int64_t(K), int64_t(int(blockIdx.y) * kWaves + wid) * per), k1 = min(K, k0 + per);

  S s;
  s.g = lane >> 4;
  s.ldb = p.ldb;
#pragma unroll
  for (int t = 0; t < MT; ++t)
    s.a[t] = static_cast<const E*>(p.a) + (m0 + min(16 * t + (lane & 15), rows - 1)) * p.lda;
  // B tr: the lane's first column, moved back where its chunk would pass the
  // last one (N >= EPC); the columns that it then shares with the lane before
  // are that lane's.
  const int mine = (lane & 15) * S::EPC, first = min(mine, p.N - n0 - S::EPC);
  if constexpr (BTR) {
    s.b[0] = b + n0 + first;
  } else {
#pragma unroll
    for (int i = 0; i < S::NB; ++i) s.b[i] = b + (n0 + min(16 * i + (lane & 15), cols - 1)) * p.ldb;
  }
  f32x4 acc[S::NB][MT];
#pragma unroll
  for (int i = 0; i < S::NB; ++i)
#pragma unroll
    for (int t = 0; t < MT; ++t) acc[i][t] = f32x4{0.f, 0.f, 0.f, 0.f};

  // the part of a step at the end of K, an odd step, then pairs: two steps in flight
  const int full = (k1 - k0) / S::BK;
  if (k0 + full * S::BK < k1) {
    typename S::Step st;
    s.template load<true>(k0 + full * S::BK, k1, st);
    s.multiply(st, acc);
  }
  if (full & 1) {
    typename S::Step st;
    s.template load<false>(k0 + (full - 1) * S::BK, k1, st);
    s.multiply(st, acc);
  }
  if (full > 1) {
    const int last = k0 + ((full & ~1) - 1) * S::BK;
    typename S::Step s0, s1;
    s.template load<false>(k0, k1, s0);
    for (int k = k0; k < last; k += 2 * S::BK) {
      s.template load<false>(k + S::BK, k1, s1);
      s.multiply(s0, acc);
      s.template load<false>(min(k + 2 * S::BK, last), k1, s0);   // (past the last pair: not used)
      s.multiply(s1, acc);
    }
  }

  // Waves 2 and 3 hand their sums to 0 and 1, then 1 to 0's place: element r of
  // acc[i][t] is row 16 t + 4 (lane / 16) + r, column first + i (B tr) or
  // 16 i + lane % 16.
  auto each = [&](float* to, auto f) {
#pragma unroll
    for (int t = 0; t < MT; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int i = 0; i < S::NB; ++i) {
          const int row = 16 * t + 4 * (lane >> 4) + r;
          const int col = BTR ? first + i : 16 * i + (lane & 15);
          if (!BTR || col >= mine) f(to[row * LD + col], acc[i][t][r]);
        }
  };
  if (wid >= 2) each(red[wid - 2], [](float& m, float v) { m = v; });
  __syncthreads();
  if (wid < 2) each(red[wid], [](float& m, float v) { m += v; });
  __syncthreads();
  constexpr int CPR = S::COLS / 8;   // 8-column chunks of a row
  for (int i = threadIdx.x; i < ROWS * CPR; i += 256) {
    const int row = i / CPR, c = i % CPR * 8, n = cols - c;
    if (row >= rows || n <= 0) continue;
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = red[0][row * LD + c + e] + red[1][row * LD + c + e];
    if (p.splits > 1 || p.raw) {
      float* to = p.part + (int64_t(blockIdx.y) * p.M + m0 + row) * p.N + n0 + c;
      if (p.add) {
        float x[8];
        load8(to, n, x);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] += x[e];
      }
      store8(to, n, v);
    } else {
      finish8<E>(p, m0 + row, n0 + c, n, v);
    }
  }
}

// Adds the partial results of a split product in order and finishes them: a
// thread per 8 columns of a row.
template <typename E>
__global__ __launch_bounds__(256) void mm_reduce_kernel(Product p) {
  const int64_t cpr = (int64_t(p.N) + 7) / 8, i = int64_t(blockIdx.x) * 256 + threadIdx.x;
  if (i >= p.M * cpr) return;
  const int64_t m = i / cpr, c = i % cpr * 8;
  const int n = int(min(int64_t(8), p.N - c));
  float v[8];
  load8(p.part + m * p.N + c, n, v);
  for (int s = 1; s < p.splits; ++s) {
    float x[8];
    load8(p.part + (int64_t(s) * p.M + m) * p.N + c, n, x);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] += x[e];
  }
  finish8<E>(p, m, c, n, v);
}

template <typename E, int MT, bool BTR, int GROUP>
hipError_t launch_one(const Product& p, const Table* t, hipStream_t st) {
  using S = Skinny<E, MT, BTR, GROUP>;
  const int64_t strips = (int64_t(p.N) + S::COLS - 1) / S::COLS;
  int64_t tiles = (int64_t(p.M) + 16 * MT - 1) / (16 * MT);
  if (GROUP == GROUP_ROWS) tiles = row_tiles_bound(p.M, p.experts, 16 * MT);
  const int64_t blocks = strips * tiles;
  if (blocks >= (int64_t(1) << 24)) return hipErrorInvalidConfiguration;
  if (!blocks) return hipSuccess;
  const dim3 g{unsigned(blocks), unsigned(p.splits)}, b{256};
  if constexpr (GROUP == GROUP_NONE)
    hipLaunchKernelGGL((mm_skinny_kernel<E, MT, BTR, GROUP>), g, b, 0, st, p, NoTable{});
  else
    hipLaunchKernelGGL((mm_skinny_kernel<E, MT, BTR, GROUP>), g, b, 0, st, p, *t);
  return hipGetLastError();
}

template <typename E, int MT>
hipError_t launch_mt(int form, int group, const Product& p, const Table* t, hipStream_t st) {
  if (group == GROUP_ROWS)
    return form == FORM_RT ? launch_one<E, MT, true, GROUP_ROWS>(p, t, st)
                           : launch_one<E, MT, false, GROUP_ROWS>(p, t, st);
  return form == FORM_RT ? launch_one<E, MT, true, GROUP_NONE>(p, t, st)
                         : launch_one<E, MT, false, GROUP_NONE>(p, t, st);
}

template <typename E>
hipError_t launch(int form, int group, int mt, const Product& p, const Table* t, hipStream_t st) {
  if (mt == 1) return launch_mt<E, 1>(form, group, p, t, st);
  if (mt == 2) return launch_mt<E, 2>(form, group, p, t, st);
  return launch_mt<E, 4>(form, group, p, t, st);
}

}  // namespace

hipError_t launch_skinny(bool bf16, int form, int group, int mt, const Product& p, const Table* t, hipStream_t st) {
  return bf16 ? launch<__bf16>(form, group, mt, p, t, st) : launch<float>(form, group, mt, p, t, st);
}

hipError_t launch_reduce(bool bf16, const Product& p, hipStream_t st) {
  const int64_t n = p.M * ((int64_t(p.N) + 7) / 8);
  const dim3 g{unsigned((n + 255) / 256)}, b{256};
  if (bf16)
    hipLaunchKernelGGL((mm_reduce_kernel<__bf16>), g, b, 0, st, p);
  else
    hipLaunchKernelGGL((mm_reduce_kernel<float>), g, b, 0, st, p);
  return hipGetLastError();
}

}  // namespace layers
}  // namespace muon
