// Device helpers of the layer operators: activations, element access, and
// where a block of a grouped product works.
#ifndef MUON_LAYERS_DEVICE_H
#define MUON_LAYERS_DEVICE_H

#include "layers.h"

namespace muon {
namespace layers {
namespace {

// 1 / (1 + exp(-v)); exp overflows to infinity for v < -88, which gives the limit 0.
// The hardware's reciprocal is good to one unit in the last place, a tenth of
// the instructions of a division.
__device__ __forceinline__ float sigmoid(float v) { return __builtin_amdgcn_rcpf(1.f + __expf(-v)); }

// The normal distribution function, and e = exp(-z^2 / 2), which its density
// needs too.  Beyond |z| it is e / 2 erfcx(a), a = |z| / sqrt(2), with
// erfcx(a) = exp(a^2) erfc(a) = t P(t), t = 1 / (1 + 0.4 a), smooth over all of
// 0 < t <= 1: P is the polynomial of degree 8 whose largest relative error there
// is least (1.3e-7, twice fp32's own rounding).  So the far side's small values are good relative
// to themselves, which 1 + erf is not in fp32: it keeps no digit of them below -5.
// Without branches: the library's erf, of which a wave takes both sides,
// made a 512 x 256 x 1024 product in fp32 12.3 us instead of 10.7.
__device__ __forceinline__ float normal_cdf(float z, float& e) {
  const float t = __builtin_amdgcn_rcpf(fmaf(0.28284271247461901f, fabsf(z), 1.f));
  e = __expf(-0.5f * z * z);
  float p = fmaf(0.0502544306f, t, -0.1828743097f);
  p = fmaf(p, t, 0.1690469545f);
  p = fmaf(p, t, -0.005579537297f);
  p = fmaf(p, t, 0.141420327f);
  p = fmaf(p, t, 0.1685443262f);
  p = fmaf(p, t, 0.20784246f);
  p = fmaf(p, t, 0.2256696073f);
  p = fmaf(p, t, 0.2256758619f);
  const float tail = 0.5f * p * t * e;
  return z < 0.f ? tail : 1.f - tail;
}

constexpr float kGeluC = 0.7978845608028654f;   // sqrt(2 / pi)
constexpr float kGeluA = 0.044715f;

// act(z).  tanh(u) = 2 sigmoid(2u) - 1 turns the tanh form into z sigmoid(2u).
template <int ACT>
__device__ __forceinline__ float act_one(float z) {
  if constexpr (ACT == MUON_ACT_RELU) return z < 0.f ? 0.f : z;   // (NaN stays)
  if constexpr (ACT == MUON_ACT_GELU) {
    float e;
    return z * normal_cdf(z, e);
  }
  if constexpr (ACT == MUON_ACT_GELU_TANH) return z * sigmoid(2.f * kGeluC * z * fmaf(kGeluA * z, z, 1.f));
  if constexpr (ACT == MUON_ACT_SILU) return z * sigmoid(z);
  return z;
}

// act'(z).  Far out (|z| > 30) the second term's sigmoid factor s (1 - s) is 0
// to fp32; z is clamped there so that an overflowing square does not make it NaN.
template <int ACT>
__device__ __forceinline__ float act_grad_one(float z) {
  if constexpr (ACT == MUON_ACT_RELU) return z > 0.f ? 1.f : z != z ? z : 0.f;
  if constexpr (ACT == MUON_ACT_GELU) {
    const float c = fminf(fmaxf(z, -30.f), 30.f);
    float e;
    const float cdf = normal_cdf(c, e);
    return z != z ? z : fmaf(c * 0.3989422804014327f, e, cdf);
  }
  if constexpr (ACT == MUON_ACT_GELU_TANH) {
    const float c = fminf(fmaxf(z, -30.f), 30.f);
    const float s = sigmoid(2.f * kGeluC * c * fmaf(kGeluA * c, c, 1.f));
    return z != z ? z : s + c * s * (1.f - s) * 2.f * kGeluC * fmaf(3.f * kGeluA * c, c, 1.f);
  }
  if constexpr (ACT == MUON_ACT_SILU) {
    const float c = fminf(fmaxf(z, -100.f), 100.f);
    const float s = sigmoid(c);
    return z != z ? z : s * fmaf(c, 1.f - s, 1.f);
  }
  return 1.f;
}

// f(tag) with the activation as a compile-time value.
template <int V>
struct IntTag {
  static constexpr int value = V;
};
template <bool ANY = true, class F>
__device__ __forceinline__ void with_act(int act, F f) {
  if constexpr (!ANY) {
    f(IntTag<MUON_ACT_NONE>{});
    return;
  }
  switch (act) {
    case MUON_ACT_RELU: f(IntTag<MUON_ACT_RELU>{}); break;
    case MUON_ACT_GELU: f(IntTag<MUON_ACT_GELU>{}); break;
    case MUON_ACT_GELU_TANH: f(IntTag<MUON_ACT_GELU_TANH>{}); break;
    case MUON_ACT_SILU: f(IntTag<MUON_ACT_SILU>{}); break;
    default: f(IntTag<MUON_ACT_NONE>{}); break;
  }
}
// f(IntTag<0>) .. f(IntTag<N - 1>): a loop that is unrolled whatever its size.
template <int N, int I = 0, class F>
__device__ __forceinline__ void static_for(const F& f) {
  if constexpr (I < N) {
    f(IntTag<I>{});
    static_for<N, I + 1>(f);
  }
}
__device__ __forceinline__ float act_of(int act, float z) {
  switch (act) {
    case MUON_ACT_RELU: return act_one<MUON_ACT_RELU>(z);
    case MUON_ACT_GELU: return act_one<MUON_ACT_GELU>(z);
    case MUON_ACT_GELU_TANH: return act_one<MUON_ACT_GELU_TANH>(z);
    case MUON_ACT_SILU: return act_one<MUON_ACT_SILU>(z);
    default: return z;
  }
}

// 8 (or the first n < 8) consecutive elements at any alignment.
template <typename E>
struct __attribute__((packed, aligned(sizeof(E)))) Packed8 {
  E v[8];
};
template <typename E>
__device__ __forceinline__ void load8(const E* p, int n, float (&v)[8]) {
  if (n >= 8) {
    const Packed8<E> x = *reinterpret_cast<const Packed8<E>*>(p);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = float(x.v[e]);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = e < n ? float(p[e]) : 0.f;
  }
}
template <typename E>
__device__ __forceinline__ void store8(E* p, int n, const float (&v)[8]) {
  if (n >= 8) {
    Packed8<E> x;
#pragma unroll
    for (int e = 0; e < 8; ++e) x.v[e] = E(v[e]);
    *reinterpret_cast<Packed8<E>*>(p) = x;
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < n) p[e] = E(v[e]);
  }
}

// The same where all 8 exist (WHOLE): no branch around a load, which would end in a
// wait for it.
template <bool WHOLE, typename E>
__device__ __forceinline__ void load_8(const E* p, int n, float (&v)[8]) {
  load8(p, WHOLE ? 8 : n, v);
}
// Of data that is read once: past the caches' order of use, which leaves them to what is
// read again.
template <bool WHOLE, typename E>
__device__ __forceinline__ void load_8_once(const E* p, int n, float (&v)[8]) {
  typedef uint32_t Words __attribute__((ext_vector_type(4), aligned(2)));
  if constexpr (WHOLE) {
    Words w[sizeof(E) / 2];
#pragma unroll
    for (int i = 0; i < int(sizeof(E) / 2); ++i) w[i] = __builtin_nontemporal_load(reinterpret_cast<const Words*>(p) + i);
    const Packed8<E> x = __builtin_bit_cast(Packed8<E>, w);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = float(x.v[e]);
  } else {
    load8(p, n, v);
  }
}
template <bool WHOLE, typename E>
__device__ __forceinline__ void store_8(E* p, int n, const float (&v)[8]) {
  store8(p, WHOLE ? 8 : n, v);
}

// Past the caches' order of use as well, which leaves them to what is read.
template <bool WHOLE, typename E>
__device__ __forceinline__ void store_8_once(E* p, int n, const float (&v)[8]) {
  typedef uint32_t Words __attribute__((ext_vector_type(4), aligned(2)));
  if constexpr (WHOLE) {
    Packed8<E> x;
#pragma unroll
    for (int e = 0; e < 8; ++e) x.v[e] = E(v[e]);
    struct Both {
      Words w[sizeof(E) / 2];
    };
    const Both b = __builtin_bit_cast(Both, x);
#pragma unroll
    for (int i = 0; i < int(sizeof(E) / 2); ++i) __builtin_nontemporal_store(b.w[i], reinterpret_cast<Words*>(p) + i);
  } else {
    store8(p, n, v);
  }
}

// The same where what is past the caches has to be whole lines: in 16 bits, of which a
// wave's instruction has one run of bytes.  In 32 bits each of a thread's two has half of every
// 32 bytes, which the caches put together: 16384 x 2048 tokens at 6 choices' rows 211 us for 358
// past them, a table's gradient of 128000 x 4096 600 for 915.
template <bool WHOLE, typename E>
__device__ __forceinline__ void load_8_run(const E* p, int n, float (&v)[8]) {
  if constexpr (sizeof(E) == 2)
    load_8_once<WHOLE>(p, n, v);
  else
    load_8<WHOLE>(p, n, v);
}
template <bool WHOLE, typename E>
__device__ __forceinline__ void store_8_run(E* p, int n, const float (&v)[8]) {
  if constexpr (sizeof(E) == 2)
    store_8_once<WHOLE>(p, n, v);
  else
    store_8<WHOLE>(p, n, v);
}

// Number i of a list of int64 or int32.
__device__ __forceinline__ int64_t id_at(const void* ids, int bytes, int64_t i) {
  return bytes == 8 ? static_cast<const int64_t*>(ids)[i] : int64_t(static_cast<const int32_t*>(ids)[i]);
}
// The column of a row's target, -1 if it has none.
__device__ __forceinline__ int label_of(const LossArgs& a, int64_t row) {
  const int64_t t = id_at(a.targets, a.target_bytes, row);
  return t >= 0 && t < a.vocab && t != a.ignore ? int(t) : -1;
}

// A plain product takes no table.
struct NoTable {};
template <int GROUP>
struct TableOf {
  typedef Table T;
};
template <>
struct TableOf<GROUP_NONE> {
  typedef NoTable T;
};

// ----------------------------------------------------------- expert ranges
// The offsets are taken in order and range whatever they hold: entry i counts
// as the largest of entries 0..i clamped to [0, rows].  Rows before the first
// entry and from the last one on belong to nobody.
__device__ __forceinline__ int clamp_row(int v, int rows) { return min(max(v, 0), rows); }

// Rows [lo, hi) of expert e (wave-uniform); all 64 lanes take part.
__device__ __forceinline__ void expert_range(const int32_t* off, int e, int rows, int lane, int& lo, int& hi) {
  int m = 0;
  for (int i = lane; i <= e; i += 64) m = max(m, clamp_row(off[i], rows));
#pragma unroll
  for (int d = 32; d; d >>= 1) m = max(m, __shfl_xor(m, d));
  lo = __builtin_amdgcn_readfirstlane(m);
  hi = max(lo, __builtin_amdgcn_readfirstlane(clamp_row(off[e + 1], rows)));
}

// The experts by size: the ranks (0: most rows; the lower index first among
// equals) of experts lane, lane + 64, ... .  All 64 lanes take part.
struct Ranks {
  static constexpr int N = MUON_GROUPED_MAX_EXPERTS / 64;
  int rank[N];
};
__device__ __forceinline__ void rank_experts(const int32_t* off, int experts, int rows, int lane, Ranks& r) {
  int size[Ranks::N];
  int top = clamp_row(off[0], rows);
#pragma unroll
  for (int q = 0; q < Ranks::N; ++q) {
    const int e = q * 64 + lane;
    size[q] = -1;
    r.rank[q] = -1;
    if (q * 64 >= experts) continue;
    int hi = clamp_row(off[min(e, experts - 1) + 1], rows);
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int v = __shfl_up(hi, d);
      if (lane >= d) hi = max(hi, v);
    }
    hi = max(hi, top);
    int lo = __shfl_up(hi, 1);
    if (lane == 0) lo = top;
    top = __builtin_amdgcn_readlane(hi, 63);
    if (e < experts) {
      size[q] = hi - lo;
      r.rank[q] = 0;
    }
  }
#pragma unroll
  for (int p = 0; p < Ranks::N; ++p) {
    for (int j = p * 64; j < min(experts, p * 64 + 64); ++j) {
      const int s = __builtin_amdgcn_readlane(size[p], j & 63);
#pragma unroll
      for (int q = 0; q < Ranks::N; ++q)
        if (q * 64 < experts && size[q] >= 0) r.rank[q] += s > size[q] || (s == size[q] && j < q * 64 + lane);
    }
  }
}
// The expert of rank `want` (< experts).
__device__ __forceinline__ int expert_of_rank(const Ranks& r, int want) {
  int e = 0;
#pragma unroll
  for (int q = 0; q < Ranks::N; ++q) {
    const unsigned long long at = __ballot(r.rank[q] == want);
    if (at) e = q * 64 + __builtin_ctzll(at);
  }
  return e;
}

// Row tile `want` (of TM rows each) of a product grouped by rows: the experts'
// tiles in order, then those of the rows nobody owns.  Group g is the rows
// before the first offset (g = 0), expert g - 1, or the rows after the last
// (g = experts + 1).  Returns false past the last tile.  All 64 lanes take part;
// the answers are wave-uniform.
struct RowTile {
  int expert;   // -1: rows nobody owns
  int row0;     // first row of the tile
  int rows;     // rows of the tile, 1..TM
};
template <int TM>
__device__ __forceinline__ bool find_row_tile(const int32_t* off, int experts, int rows, int want, int lane,
                                              RowTile& t) {
  int top = 0, tiles = 0;
  for (int base = 0; base < experts + 2; base += 64) {
    const int g = base + lane;
    int hi = g <= experts ? clamp_row(off[g], rows) : rows;   // group g ends where entry g says
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int v = __shfl_up(hi, d);
      if (lane >= d) hi = max(hi, v);
    }
    hi = max(hi, top);
    int lo = __shfl_up(hi, 1);
    if (lane == 0) lo = top;
    const int cnt = g < experts + 2 ? hi - lo : 0;
    const int mine = (cnt + TM - 1) / TM;
    int sum = mine;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int v = __shfl_up(sum, d);
      if (lane >= d) sum += v;
    }
    sum += tiles;
    const unsigned long long past = __ballot(want < sum);
    if (past) {
      const int src = __builtin_ctzll(past);
      const int mt = want - (__builtin_amdgcn_readlane(sum, src) - __builtin_amdgcn_readlane(mine, src));
      const int n = __builtin_amdgcn_readlane(cnt, src);
      const int gg = base + src;
      t.expert = gg >= 1 && gg <= experts ? gg - 1 : -1;
      t.row0 = __builtin_amdgcn_readlane(lo, src) + mt * TM;
      t.rows = min(TM, n - mt * TM);
      return true;
    }
    top = __builtin_amdgcn_readlane(hi, 63);
    tiles = __builtin_amdgcn_readlane(sum, 63);
  }
  return false;
}
// Most row tiles of any offsets: whole tiles, plus a partial one per group.
inline int64_t row_tiles_bound(int64_t rows, int64_t experts, int64_t tm) {
  const int64_t groups = experts + 2;
  return rows <= groups ? rows : (rows - groups) / tm + groups;
}

}  // namespace
}  // namespace layers
}  // namespace muon

#endif  // MUON_LAYERS_DEVICE_H
