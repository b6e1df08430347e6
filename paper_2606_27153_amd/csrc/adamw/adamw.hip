// The AdamW step over many tensors: one launch for up to 56 of them.
//
// A workgroup has 4096 elements of one tensor, which it finds by its number; a
// lane has 8 neighbours at a time, so that every access is 8 to 32 bytes.  Each byte is
// moved once: 22 an element with bf16 parameters and gradients and fp32 states, 10
// with states in 8 bits.
//
// States in 8 bits: 32 lanes have a block of 256 elements.  What is rounded is the
// average as fp32 arithmetic without fused operations gives it, so that the codes
// are a function of the inputs that any program can reproduce bit by bit.
#include "adamw.h"

namespace muon {
namespace adamw {
namespace {

template <typename E>
struct __attribute__((packed, aligned(sizeof(E)))) Packed8 {
  E v[8];
};
template <typename E>
__device__ __forceinline__ void load8(const E* p, int64_t n, float (&v)[8]) {
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
__device__ __forceinline__ void store8(E* p, int64_t n, const float (&v)[8]) {
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
struct Codes {
  uint8_t c[8];
};
__device__ __forceinline__ Codes load_codes(const uint8_t* p, int64_t n) {
  Codes x;
  if (n >= 8) {
    const Packed8<uint8_t> y = *reinterpret_cast<const Packed8<uint8_t>*>(p);
#pragma unroll
    for (int e = 0; e < 8; ++e) x.c[e] = y.v[e];
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) x.c[e] = e < n ? p[e] : 0;
  }
  return x;
}
__device__ __forceinline__ void store_codes(uint8_t* p, int64_t n, const Codes& x) {
  if (n >= 8) {
    Packed8<uint8_t> y;
#pragma unroll
    for (int e = 0; e < 8; ++e) y.v[e] = x.c[e];
    *reinterpret_cast<Packed8<uint8_t>*>(p) = y;
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < n) p[e] = x.c[e];
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
template <bool SIGNED>
__device__ __forceinline__ uint8_t encode(float v, int base, uint32_t add) {
  constexpr int TOP = SIGNED ? 127 : 255;
  const uint32_t all = __builtin_bit_cast(uint32_t, v), bits = all & 0x7fffffffu;
  const int low = SIGNED ? 0 : int(bits != 0);
  const int size = max(min(int((bits + add) >> 20) - base, TOP), low);
  return uint8_t(SIGNED && size ? size | (all >> 31 << 7) : size);
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

template <typename P, typename G, int BITS>
__global__ __launch_bounds__(256) void step_kernel(Args a) {
  const Tensor& t = a.t[find_tensor(a, blockIdx.x)];
  const int64_t start = int64_t(int(blockIdx.x) - t.first) * kChunk;
  P* p = static_cast<P*>(t.p);
  const G* g = static_cast<const G*>(t.g);
  uint32_t key = t.key;
  if (start >> 32) key = mix(key + uint32_t(start >> 32));   // (a chunk does not cross a multiple of 2^32)
#pragma unroll
  for (int u = 0; u < kChunk / 2048; ++u) {
    const int64_t i = start + u * 2048 + threadIdx.x * 8, left = t.n - i;
    // (all lanes of a block stay for its maximum; those past the end have zeros)
    if (BITS == 32 && left <= 0) return;
    const int64_t n = left < 0 ? 0 : left;
    float w[8], d[8], m[8], v[8];
    load8(p + i, n, w);
    load8(g + i, n, d);
    int16_t* base = t.bases + i / kBlock * 2;
    if constexpr (BITS == 32) {
      load8(static_cast<const float*>(t.m) + i, n, m);
      load8(static_cast<const float*>(t.v) + i, n, v);
    } else {
      const Codes cm = load_codes(static_cast<const uint8_t*>(t.m) + i, n);
      const Codes cv = load_codes(static_cast<const uint8_t*>(t.v) + i, n);
      const int bm = n ? base[0] : 0, bv = n ? base[1] : 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        m[e] = decode<true>(cm.c[e], bm);
        v[e] = decode<false>(cv.c[e], bv);
      }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      m[e] = average(m[e], a.b1, a.c1, d[e]);
      v[e] = average(v[e], a.b2, a.c2, d[e] * d[e]);
      const float q = m[e] / fmaf(sqrtf(v[e]), t.scale, a.eps);
      w[e] = fmaf(-t.step, q, w[e] * a.keep);
    }
    store8(p + i, n, w);
    if constexpr (BITS == 32) {
      store8(static_cast<float*>(t.m) + i, n, m);
      store8(static_cast<float*>(t.v) + i, n, v);
    } else {
      uint32_t top_m = 0, top_v = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        top_m = max(top_m, __builtin_bit_cast(uint32_t, m[e]) & 0x7fffffffu);
        top_v = max(top_v, __builtin_bit_cast(uint32_t, v[e]) & 0x7fffffffu);
      }
      const int bm = base_of<true>(block_max(top_m)), bv = base_of<false>(block_max(top_v));
      Codes cm, cv;
      uint32_t at = uint32_t(i) * 0x9E3779B1u;
#pragma unroll
      for (int e = 0; e < 8; ++e, at += 0x9E3779B1u) {
        const uint32_t h = mix(at ^ key);
        cm.c[e] = encode<true>(m[e], bm, (h & 0xffff) << 4);
        cv.c[e] = encode<false>(v[e], bv, h >> 16 << 4);
      }
      store_codes(static_cast<uint8_t*>(t.m) + i, n, cm);
      store_codes(static_cast<uint8_t*>(t.v) + i, n, cv);
      if ((threadIdx.x & 31) == 0 && n) {
        base[0] = int16_t(bm);
        base[1] = int16_t(bv);
      }
    }
  }
}

__global__ __launch_bounds__(256) void values_kernel(const uint8_t* m, const uint8_t* v, const int16_t* bases,
                                                     int64_t count, __bf16* mo, __bf16* vo) {
  const int64_t i = (int64_t(blockIdx.x) * 256 + threadIdx.x) * 8, n = count - i;
  if (n <= 0) return;
  const int16_t* base = bases + i / kBlock * 2;
  float x[8];
  if (mo) {
    const Codes c = load_codes(m + i, n);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = decode<true>(c.c[e], base[0]);
    store8(mo + i, n, x);
  }
  if (vo) {
    const Codes c = load_codes(v + i, n);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = decode<false>(c.c[e], base[1]);
    store8(vo + i, n, x);
  }
}

template <typename P, typename G>
hipError_t launch(int bits, const Args& a, int64_t blocks, hipStream_t st) {
  const dim3 g{unsigned(blocks)}, b{256};
  if (bits == 32)
    hipLaunchKernelGGL((step_kernel<P, G, 32>), g, b, 0, st, a);
  else
    hipLaunchKernelGGL((step_kernel<P, G, 8>), g, b, 0, st, a);
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
  const int64_t blocks = (n + 2047) / 2048;
  hipLaunchKernelGGL(values_kernel, dim3{unsigned(blocks)}, dim3{256}, 0, st, m, v, bases, n, static_cast<__bf16*>(mo),
                     static_cast<__bf16*>(vo));
  return hipGetLastError();
}

}  // namespace adamw
}  // namespace muon
