// Matrix product on the vector units: any strides, sizes, alignment and type,
// and no scratch memory.  It runs what the other kernels cannot fetch when the
// caller's workspace has no room for copies (pack.hip).
//
// C = A B with the operands in one of three layouts, a block per 64 x 64 tile
// of C: K advances in slabs of 16, which the block converts to fp32 in LDS; a
// thread keeps 4 x 4 sums.  Bound by the vector units' fp32 rate and by the
// element-wise loads: 16384 x 14336 x 4096 in bf16 takes 26.1 ms (74 TFLOP/s),
// 17 times the 256 tile's time.
#include "device.h"

namespace muon {
namespace layers {
namespace {

constexpr int TM = 64, TN = 64, TK = 16;

template <typename E, int FORM, int GROUP>
__global__ __launch_bounds__(256) void mm_simple_kernel(Product p, Table tab) {
  __shared__ float sa[TK][TM + 4], sb[TK][TN + 4];
  const int tid = threadIdx.x, lane = tid & 63;
  const int nt = (p.N + TN - 1) / TN, mt = (p.M + TM - 1) / TM;
  const E* a = static_cast<const E*>(p.a);
  const E* b = static_cast<const E*>(p.b);
  E* c = static_cast<E*>(p.c);
  int64_t m0 = int64_t(blockIdx.x) / nt * TM;
  const int64_t n0 = int64_t(blockIdx.x) % nt * TN;
  int mrows = int(min(int64_t(TM), p.M - m0));
  int k0 = 0, k1 = p.K;
  if constexpr (GROUP == GROUP_ROWS) {
    RowTile t;
    if (!find_row_tile<TM>(p.offsets, p.experts, p.M, int(blockIdx.x) / nt, lane, t)) return;
    m0 = t.row0;
    mrows = t.rows;
    if (t.expert < 0)
      k1 = 0;
    else
      b = static_cast<const E*>(tab.p[t.expert]);
  }
  if constexpr (GROUP == GROUP_SUM) {
    const int e = int(int64_t(blockIdx.x) / (int64_t(nt) * mt));
    m0 = int64_t(blockIdx.x) / nt % mt * TM;
    mrows = int(min(int64_t(TM), p.M - m0));
    c = const_cast<E*>(static_cast<const E*>(tab.p[e]));
    if (!c) return;
    expert_range(p.offsets, e, p.K, lane, k0, k1);
  }
  const int ncols = int(min(int64_t(TN), p.N - n0));
  float acc[4][4] = {};
  const int tx = tid & 15, ty = tid >> 4;
  for (int k = k0; k < k1; k += TK) {
#pragma unroll
    for (int i = 0; i < TM * TK / 256; ++i) {
      const int at = tid + 256 * i;
      // consecutive threads along the operand's memory
      const int am = FORM == FORM_TT ? at % TM : at / TK, ak = FORM == FORM_TT ? at / TM : at % TK;
      float v = 0.f;
      if (am < mrows && k + ak < k1)
        v = float(FORM == FORM_TT ? a[int64_t(k + ak) * p.lda + m0 + am] : a[(m0 + am) * p.lda + k + ak]);
      sa[ak][am] = v;
      const int bn = FORM == FORM_RR ? at / TK : at % TN, bk = FORM == FORM_RR ? at % TK : at / TN;
      v = 0.f;
      if (bn < ncols && k + bk < k1)
        v = float(FORM == FORM_RR ? b[(n0 + bn) * p.ldb + k + bk] : b[int64_t(k + bk) * p.ldb + n0 + bn]);
      sb[bk][bn] = v;
    }
    __syncthreads();
#pragma unroll
    for (int kk = 0; kk < TK; ++kk)
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = fmaf(sa[kk][ty * 4 + i], sb[kk][tx * 4 + j], acc[i][j]);
    __syncthreads();
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int mi = ty * 4 + i, nj = tx * 4 + j;
      if (mi >= mrows || nj >= ncols) continue;
      const int64_t m = m0 + mi, n = n0 + nj;
      float v = acc[i][j];
      if (p.bias) v += float(static_cast<const E*>(p.bias)[n]);
      if (p.z) static_cast<E*>(p.z)[m * p.ldz + n] = E(v);
      v = act_of(p.act, v);
      if (p.res) v += float(static_cast<const E*>(p.res)[m * p.ldr + n]);
      c[m * p.ldc + n] = E(v);
    }
}

template <typename E>
hipError_t launch(int form, int group, const Product& p, const Table& t, hipStream_t st) {
  const int64_t nt = (int64_t(p.N) + TN - 1) / TN, mt = (int64_t(p.M) + TM - 1) / TM;
  int64_t blocks = nt * mt;
  if (group == GROUP_ROWS) blocks = nt * row_tiles_bound(p.M, p.experts, TM);
  if (group == GROUP_SUM) blocks *= p.experts;
  if (blocks == 0) return hipSuccess;
  if (blocks >= (int64_t(1) << 24)) return hipErrorInvalidConfiguration;
  const dim3 g{unsigned(blocks)}, b{256};
  if (group == GROUP_NONE) {
    if (form == FORM_RT) hipLaunchKernelGGL((mm_simple_kernel<E, FORM_RT, GROUP_NONE>), g, b, 0, st, p, t);
    if (form == FORM_RR) hipLaunchKernelGGL((mm_simple_kernel<E, FORM_RR, GROUP_NONE>), g, b, 0, st, p, t);
    if (form == FORM_TT) hipLaunchKernelGGL((mm_simple_kernel<E, FORM_TT, GROUP_NONE>), g, b, 0, st, p, t);
  } else if (group == GROUP_ROWS) {
    if (form == FORM_RT) hipLaunchKernelGGL((mm_simple_kernel<E, FORM_RT, GROUP_ROWS>), g, b, 0, st, p, t);
    if (form == FORM_RR) hipLaunchKernelGGL((mm_simple_kernel<E, FORM_RR, GROUP_ROWS>), g, b, 0, st, p, t);
  } else {
    hipLaunchKernelGGL((mm_simple_kernel<E, FORM_TT, GROUP_SUM>), g, b, 0, st, p, t);
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_simple(bool bf16, int form, int group, const Product& p, const Table* t, hipStream_t st) {
  static const Table none{};
  const Table& tab = t ? *t : none;
  return bf16 ? launch<__bf16>(form, group, p, tab, st) : launch<float>(form, group, p, tab, st);
}

}  // namespace layers
}  // namespace muon
