// The AdamW step over many tensors: one launch for up to 56 of them.
//
// A workgroup has 4096 elements of one tensor, which it finds by its number.  Each
// byte is moved once: 22 an element with bf16 parameters and gradients and fp32 states, 10
// with states in 8 bits.
//
// States in 8 bits: 32 lanes have a block of 256 elements.  What is rounded is the
// average as fp32 arithmetic without fused operations gives it, so that the codes
// are a function of the inputs that any program can reproduce bit by bit.
#include "adamw.h"

namespace muon {
namespace adamw {
namespace {

// N neighbours at any alignment, of which the first n exist; WHOLE: all of them, which
// leaves no branch around a load (it would end in a wait for it).
template <typename E, int N>
struct __attribute__((packed, aligned(sizeof(E)))) Packed {
  E v[N];
};
template <bool FIRST, typename A, typename B>
struct Pick {
  typedef A T;
};
template <typename A, typename B>
struct Pick<false, A, B> {
  typedef B T;
};
template <bool WHOLE, bool ONCE = true, typename E, int N>
__device__ __forceinline__ void load(const E* p, int64_t n, float (&v)[N]) {
  if (WHOLE || n >= N) {
    // ONCE: past the caches' order of use, as everything is read once (977 us for 1009 of 8-bit states)
    typedef uint32_t Words __attribute__((ext_vector_type(2), aligned(2)));
    typedef uint32_t Words4 __attribute__((ext_vector_type(4), aligned(2)));
    constexpr bool FOUR = N * sizeof(E) % 16 == 0;
    typedef typename Pick<FOUR, Words4, Words>::T W;
    W w[N * sizeof(E) / sizeof(W)];
#pragma unroll
    for (int i = 0; i < int(N * sizeof(E) / sizeof(W)); ++i)
      w[i] = ONCE ? __builtin_nontemporal_load(reinterpret_cast<const W*>(p) + i) : reinterpret_cast<const W*>(p)[i];
    const Packed<E, N> x = __builtin_bit_cast(Packed<E, N>, w);
#pragma unroll
    for (int e = 0; e < N; ++e) v[e] = float(x.v[e]);
  } else {
#pragma unroll
    for (int e = 0; e < N; ++e) v[e] = e < n ? float(p[e]) : 0.f;
  }
}
// Past them as well: 131 million elements with 32-bit states 496 us for 529, 525 million with
// 8-bit ones and the values read out 1428 for 1535.
template <bool WHOLE, bool ONCE = true, typename E, int N>
__device__ __forceinline__ void store(E* p, int64_t n, const float (&v)[N]) {
  if (WHOLE || n >= N) {
    Packed<E, N> x;
#pragma unroll
    for (int e = 0; e < N; ++e) x.v[e] = E(v[e]);
    typedef uint32_t Words __attribute__((ext_vector_type(2), aligned(2)));
    typedef uint32_t Words4 __attribute__((ext_vector_type(4), aligned(2)));
    constexpr bool FOUR = N * sizeof(E) % 16 == 0;
    typedef typename Pick<FOUR, Words4, Words>::T W;
    struct All {
      W w[N * sizeof(E) / sizeof(W)];
    };
    const All b = __builtin_bit_cast(All, x);
#pragma unroll
    for (int i = 0; i < int(N * sizeof(E) / sizeof(W)); ++i) {
      if constexpr (ONCE)
        __builtin_nontemporal_store(b.w[i], reinterpret_cast<W*>(p) + i);
      else
        reinterpret_cast<W*>(p)[i] = b.w[i];
    }
  } else {
#pragma unroll
    for (int e = 0; e < N; ++e)
      if (e < n) p[e] = E(v[e]);
  }
}
// 8 codes, element e's in bits 8 (e % 4) of word e / 4.
struct Codes {
  uint32_t w[2];
  __device__ __forceinline__ uint32_t operator[](int e) const { return w[e / 4] >> (8 * (e % 4)) & 255; }
};
template <bool WHOLE, bool ONCE>
__device__ __forceinline__ Codes load_codes(const uint8_t* p, int64_t n) {
  typedef uint32_t Words __attribute__((ext_vector_type(2), aligned(1)));
  if (WHOLE || n >= 8) {
    const Words* q = reinterpret_cast<const Words*>(p);
    const Words w = ONCE ? __builtin_nontemporal_load(q) : *q;
    return Codes{w[0], w[1]};
  }
  Codes x{};
#pragma unroll
  for (int e = 0; e < 8; ++e) x.w[e / 4] |= (e < n ? uint32_t(p[e]) : 0) << (8 * (e % 4));
  return x;
}
template <bool WHOLE>
__device__ __forceinline__ void store_codes(uint8_t* p, int64_t n, const Codes& x) {
  if (WHOLE || n >= 8) {
    typedef uint32_t Words __attribute__((ext_vector_type(2), aligned(1)));
    __builtin_nontemporal_store(Words{x.w[0], x.w[1]}, reinterpret_cast<Words*>(p));
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < n) p[e] = uint8_t(x[e]);
  }
}

template <bool SIGNED>
__device__ __forceinline__ float decode(uint32_t code, int base) {
  const uint32_t size = SIGNED ? code & 127 : code;
  uint32_t bits = size ? (size + base) << 20 : 0;
  if (SIGNED) bits |= (code & 128) << 24;
  return __builtin_bit_cast(float, bits);
}
// The largest of the 32 lanes that have a block.
__device__ __forceinline__ uint32_t block_max(uint32_t v) {
#pragma unroll
  for (int d = 16; d; d >>= 1) v = max(v, uint32_t(__shfl_xor(int(v), d)));
  return v;
}
template <bool SIGNED>
__device__ __forceinline__ int base_of(uint32_t largest) {
  constexpr int TOP = SIGNED ? 127 : 255;
  return min(max(int(largest >> 20) + 1 - TOP, 0), 2047 - TOP);
}
// up: 16 random bits, added below the ones that stay (of the 20 that go, the lowest 4 do not
// reach a carry).
template <bool SIGNED>
__device__ __forceinline__ uint32_t encode(float v, int base, uint32_t up) {
  constexpr int TOP = SIGNED ? 127 : 255;
  const uint32_t all = __builtin_bit_cast(uint32_t, v), bits = all & 0x7fffffffu;
  const int low = SIGNED ? 0 : int(bits != 0);
  const int size = max(min(int(((bits >> 4) + up) >> 16) - base, TOP), low);
  return SIGNED && size ? size | (all >> 31 << 7) : size;
}

// Products and sums that stay apart.
__device__ __forceinline__ float average(float a, float b, float c, float x) {
#pragma clang fp contract(off)
  const float kept = a * b, added = c * x;
  return kept + added;
}

// The workgroup's tensor: the last that begins at or before it.
__device__ __forceinline__ int find_tensor(const Args& a, int block) {
  int lo = 0, hi = a.count;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (a.t[mid].first <= block)
      lo = mid;
    else
      hi = mid;
  }
  return lo;
}

// An element's averages and parameter.  The hardware's root and reciprocal are good
// to one unit in the last place (8-bit states: 1545 us for 525 million elements with the values
// read out, where the correctly rounded ones took 1627).  They know no numbers below 2^-126, so
// v counts as that at least: without eps, an element whose gradients were always
// tiny steps by m / 2^-63, no more than the formula's order, and one that had none stays.
__device__ __forceinline__ void update(const Args& a, const Tensor& t, float g, float& w, float& m, float& v) {
  m = average(m, a.b1, a.c1, g);
  v = average(v, a.b2, a.c2, g * g);
  w = fmaf(-t.step, m * __builtin_amdgcn_rcpf(fmaf(__builtin_amdgcn_sqrtf(fmaxf(v, 0x1p-126f)), t.scale, a.eps)), w * a.keep);
}

// fp32 states: a lane has 4 neighbours, 16 bytes of each average, so that every
// access of a wave is one run of bytes (with 8 neighbours, two halves of lines, 131 million elements
// took 714 us where these took 557).
template <bool WHOLE, typename P, typename G>
__device__ __forceinline__ void step32(const Args& a, const Tensor& t, int64_t start) {
  constexpr int N = 4, U = 2;
  for (int c = 0; c < kChunk; c += 256 * N * U) {
    float w[U][N], d[U][N], m[U][N], v[U][N];
    const int64_t i = start + c + threadIdx.x * N;
    if (!WHOLE && i >= t.n) return;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t k = i + u * 256 * N, n = t.n - k;
      load<WHOLE>(static_cast<const P*>(t.p) + k, n, w[u]);
      load<WHOLE>(static_cast<const G*>(t.g) + k, n, d[u]);
      load<WHOLE>(static_cast<const float*>(t.m) + k, n, m[u]);
      load<WHOLE>(static_cast<const float*>(t.v) + k, n, v[u]);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t k = i + u * 256 * N, n = t.n - k;
#pragma unroll
      for (int e = 0; e < N; ++e) update(a, t, d[u][e], w[u][e], m[u][e], v[u][e]);
      store<WHOLE>(static_cast<P*>(t.p) + k, n, w[u]);
      store<WHOLE>(static_cast<float*>(t.m) + k, n, m[u]);
      store<WHOLE>(static_cast<float*>(t.v) + k, n, v[u]);
    }
  }
}

template <typename P, typename G>
__global__ __launch_bounds__(256) void step32_kernel(Args a) {
  const Tensor& t = a.t[find_tensor(a, blockIdx.x)];
  const int64_t start = int64_t(int(blockIdx.x) - t.first) * kChunk;
  if (start + kChunk <= t.n)
    step32<true, P, G>(a, t, start);
  else
    step32<false, P, G>(a, t, start);
}

// States in 8 bits: 32 lanes have a block of 256 elements; all of them stay for its
// maximum, those past the end with zeros.  All of a workgroup's loads come first: 525 million
// elements and their values 1419 us, where those of each half waited for the stores of the
// one before 1455.
template <bool WHOLE, typename P, typename G>
__device__ __forceinline__ void step8(const Args& a, const Tensor& t, int64_t start) {
  uint32_t key = t.key;
  if (start >> 32) key = mix(key + uint32_t(start >> 32));   // (a chunk does not cross a multiple of 2^32)
  constexpr int U = kChunk / 2048;
  // 8 fp32 neighbours are two halves of every 32 bytes of a wave's run, which the caches have to
  // put together (134 million parameters with gradients in fp32 385 us for 465, in bf16 338
  // for 405; their gradients alone, with bf16 parameters, lose 5%)
  constexpr bool ONCE = sizeof(P) == 2;
  float w[U][8], d[U][8];
  Codes om[U], ov[U];
  int obm[U], obv[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int64_t i = start + u * 2048 + threadIdx.x * 8, n = max(t.n - i, int64_t(0));
    load<WHOLE, ONCE>(static_cast<const P*>(t.p) + i, n, w[u]);
    load<WHOLE, ONCE || sizeof(G) == 2>(static_cast<const G*>(t.g) + i, n, d[u]);
    om[u] = load_codes<WHOLE, true>(static_cast<const uint8_t*>(t.m) + i, n);
    ov[u] = load_codes<WHOLE, true>(static_cast<const uint8_t*>(t.v) + i, n);
    const int16_t* base = t.bases + i / kBlock * 2;
    obm[u] = WHOLE || n ? base[0] : 0;
    obv[u] = WHOLE || n ? base[1] : 0;
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int64_t i = start + u * 2048 + threadIdx.x * 8, n = max(t.n - i, int64_t(0));
    float m[8], v[8];
    int16_t* base = t.bases + i / kBlock * 2;
    uint32_t top_m = 0, top_v = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      m[e] = decode<true>(om[u][e], obm[u]);
      v[e] = decode<false>(ov[u][e], obv[u]);
      update(a, t, d[u][e], w[u][e], m[e], v[e]);
      top_m = max(top_m, __builtin_bit_cast(uint32_t, m[e]) & 0x7fffffffu);
      top_v = max(top_v, __builtin_bit_cast(uint32_t, v[e]) & 0x7fffffffu);
    }
    store<WHOLE, ONCE>(static_cast<P*>(t.p) + i, n, w[u]);
    const int bm = base_of<true>(block_max(top_m)), bv = base_of<false>(block_max(top_v));
    Codes cm{}, cv{};
    uint32_t at = uint32_t(i) * 0x9E3779B1u;
#pragma unroll
    for (int e = 0; e < 8; ++e, at += 0x9E3779B1u) {
      const uint32_t h = mix(at ^ key);
      cm.w[e / 4] |= encode<true>(m[e], bm, h & 0xffff) << (8 * (e % 4));
      cv.w[e / 4] |= encode<false>(v[e], bv, h >> 16) << (8 * (e % 4));
    }
    store_codes<WHOLE>(static_cast<uint8_t*>(t.m) + i, n, cm);
    store_codes<WHOLE>(static_cast<uint8_t*>(t.v) + i, n, cv);
    if ((threadIdx.x & 31) == 0 && n) {
      base[0] = int16_t(bm);
      base[1] = int16_t(bv);
    }
  }
}

template <typename P, typename G>
__global__ __launch_bounds__(256) void step8_kernel(Args a) {
  const Tensor& t = a.t[find_tensor(a, blockIdx.x)];
  const int64_t start = int64_t(int(blockIdx.x) - t.first) * kChunk;
  if (start + kChunk <= t.n)
    step8<true, P, G>(a, t, start);
  else
    step8<false, P, G>(a, t, start);
}

template <bool WHOLE>
__device__ __forceinline__ void values(const uint8_t* m, const uint8_t* v, const int16_t* bases, int64_t start,
                                       int64_t count, __bf16* mo, __bf16* vo) {
  constexpr int U = kChunk / 2048;
  Codes cm[U]{}, cv[U]{};
  int bm[U], bv[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int64_t i = start + u * 2048 + threadIdx.x * 8, n = max(count - i, int64_t(0));
    const int16_t* base = bases + (WHOLE || n ? i : 0) / kBlock * 2;
    bm[u] = base[0];
    bv[u] = base[1];
    if (mo) cm[u] = load_codes<WHOLE, false>(m + i, n);
    if (vo) cv[u] = load_codes<WHOLE, false>(v + i, n);
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int64_t i = start + u * 2048 + threadIdx.x * 8, n = max(count - i, int64_t(0));
    float x[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = decode<true>(cm[u][e], bm[u]);
    if (mo) store<WHOLE>(mo + i, n, x);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = decode<false>(cv[u][e], bv[u]);
    if (vo) store<WHOLE>(vo + i, n, x);
  }
}

__global__ __launch_bounds__(256) void values_kernel(const uint8_t* m, const uint8_t* v, const int16_t* bases,
                                                     int64_t count, __bf16* mo, __bf16* vo) {
  const int64_t start = int64_t(blockIdx.x) * kChunk;
  if (start + kChunk <= count)
    values<true>(m, v, bases, start, count, mo, vo);
  else
    values<false>(m, v, bases, start, count, mo, vo);
}

template <typename P, typename G>
hipError_t launch(int bits, const Args& a, int64_t blocks, hipStream_t st) {
  const dim3 g{unsigned(blocks)}, b{256};
  if (bits == 32)
    hipLaunchKernelGGL((step32_kernel<P, G>), g, b, 0, st, a);
  else
    hipLaunchKernelGGL((step8_kernel<P, G>), g, b, 0, st, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_step(bool param_bf16, bool grad_bf16, int bits, const Args& a, int64_t blocks, hipStream_t st) {
  if (param_bf16)
    return grad_bf16 ? launch<__bf16, __bf16>(bits, a, blocks, st) : launch<__bf16, float>(bits, a, blocks, st);
  return grad_bf16 ? launch<float, __bf16>(bits, a, blocks, st) : launch<float, float>(bits, a, blocks, st);
}

hipError_t launch_values(const uint8_t* m, const uint8_t* v, const int16_t* bases, int64_t n, void* mo, void* vo,
                         hipStream_t st) {
  const int64_t blocks = (n + kChunk - 1) / kChunk;
  hipLaunchKernelGGL(values_kernel, dim3{unsigned(blocks)}, dim3{256}, 0, st, m, v, bases, n, static_cast<__bf16*>(mo),
                     static_cast<__bf16*>(vo));
  return hipGetLastError();
}

}  // namespace adamw
}  // namespace muon
