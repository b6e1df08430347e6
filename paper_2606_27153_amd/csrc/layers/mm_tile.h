// Matrix products on the matrix cores, one block of four waves per TM x TN
// tile of C.
//
// K advances in slabs of 128 bytes of a K-contiguous row (64 bf16, 32 fp32),
// which go straight from global memory into two LDS stages (16 bytes per lane
// and instruction).  A "row" operand's slab holds its rows, 128 bytes each; a
// "tr" operand's slab holds BK rows of TM (TN) elements as they lie in memory,
// and the fragment reads transpose: ds_read_b64_tr_b16 for bf16, single words
// for fp32.  16-byte chunks (32-byte segments) are XOR-swizzled with the row so
// that the fragment reads are free of bank conflicts.
//
// Each wave owns a (TM / 2) x (TN / 2) piece of 32 x 32 MFMA blocks.  A slab is
// four K steps; the fragments of the next step are read while the current
// step's MFMAs run, one memory instruction per MFMA or so.  The last step of a
// slab starts with the slab's only barrier (every wave has read the slab, the
// next one has landed) and also issues the loads of the slab after next into
// the stage just read, which leaves them a whole slab's time to arrive.
//
// The MFMAs take B as their first operand, so a lane holds 4 consecutive
// columns of a row of C; exchanging halves of the wave between two such groups
// gives it 8, and the epilogue (bias, activation, residual) and its stores
// work on 16 bytes of bf16 without passing through LDS.
//
// Rows and columns past the edge of C read the last valid ones again; their
// sums are never stored.  Where K ends inside a slab, the chunks past it come
// from a block of zeros.
#ifndef MUON_LAYERS_MM_TILE_H
#define MUON_LAYERS_MM_TILE_H

#include "../ns_gemm_kernel.h"
#include "device.h"

namespace muon {
namespace layers {
namespace {

template <typename E, int TM_, int TN_>
struct Tile {
  static constexpr int TM = TM_, TN = TN_;
  static constexpr int EPC = 16 / int(sizeof(E));   // elements of a 16-byte chunk
  static constexpr int BK = 8 * EPC;                // K elements of a slab
  static constexpr int WTM = TM / 2, WTN = TN / 2;  // wave piece
  static constexpr int NBM = WTM / 32, NBN = WTN / 32;
  static constexpr int ABYTES = TM * 128, BBYTES = TN * 128;
  static constexpr int STAGE = ABYTES + BBYTES;
};

__device__ const float4 kZeros[4] = {};

// 16 bytes per lane to LDS: lane l's land at lds + 16 l.
__device__ __forceinline__ void dma16_to(const void* p, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(p), "s"(lds) : "memory", "m0");
}
__device__ __forceinline__ uint32_t lds_addr(const char* p) {
  return uint32_t(reinterpret_cast<uintptr_t>((const lds_void_t*)(p)));
}

// One operand's slab loads.  T: rows (row operand) or columns (tr operand) of
// the tile.  1 KB chunk q of the slab belongs to wave q % 4.
template <typename E, int T, bool TR>
struct Loader {
  static constexpr int N = T / 32;                          // loads per wave and slab
  static constexpr int ROWB = TR ? T * int(sizeof(E)) : 128;  // bytes of an LDS row
  static constexpr int RPC = 1024 / ROWB;                   // LDS rows of a chunk
  static constexpr int LPR = ROWB / 16;                     // lanes per LDS row
  static constexpr int EPC = 16 / int(sizeof(E));
  static constexpr int BK = 8 * EPC;
  const char* base;      // uniform: the current slab's first element
  int64_t step;          // bytes from slab to slab
  uint32_t off[TR ? 1 : N];  // this lane's offsets; a tr operand's differ by `stride` from load to load
  uint32_t stride;
  int k;                 // this lane's K element (row operand) or K row (tr operand) in its first chunk

  // op: the tile's corner (row or column 0, the first K); ld in elements;
  // valid: rows or columns of the tile that exist (>= 1).
  __device__ __forceinline__ void init(const E* op, int64_t ld, int valid, int wid, int lane) {
    base = reinterpret_cast<const char*>(op);
    if constexpr (TR) {
      const int row = wid * RPC + lane / LPR, slot = lane % LPR;
      int chunk = slot;
      if constexpr (sizeof(E) == 2) chunk = (((slot >> 1) ^ seg_swz<ROWB>(row)) << 1) | (slot & 1);
      const int col = min(chunk * EPC, valid - EPC);
      step = BK * ld * int64_t(sizeof(E));
      off[0] = uint32_t(row * ld * int64_t(sizeof(E)) + col * int64_t(sizeof(E)));
      stride = uint32_t(4 * RPC * ld * int64_t(sizeof(E)));
      k = row;
    } else {
      step = BK * int64_t(sizeof(E));
      const int r0 = wid * 8 + (lane >> 3);
      k = ((lane & 7) ^ swz(r0)) * EPC;
#pragma unroll
      for (int i = 0; i < N; ++i)
        off[i] = uint32_t(min(r0 + 32 * i, valid - 1) * ld * int64_t(sizeof(E)) + k * int64_t(sizeof(E)));
      stride = 0;
    }
  }
  // Load i of the slab that starts kleft elements before the end of K (kleft
  // <= 0: past it; the slab is never read, the loads only keep the count).
  __device__ __forceinline__ void load(int i, uint32_t lds, int wid, int kleft) const {
    const bool in = k + (TR ? 4 * RPC * i : 0) < kleft;
    const char* from = base + (TR ? off[0] + i * stride : off[i]);
    dma16_to(in ? from : reinterpret_cast<const char*>(kZeros), lds + (wid + 4 * i) * 1024);
  }
  __device__ __forceinline__ void next() { base += step; }
};

// One operand's fragment reads.  NB 32-row blocks from row (column) w0 of the slab.
template <typename E, int T, int NB, bool TR>
struct Reader {
  static constexpr int ROWB = TR ? T * int(sizeof(E)) : 128;
  static constexpr bool F32 = sizeof(E) == 4;
  static constexpr int READS = !TR ? NB : F32 ? 4 * NB : 2 * NB;   // LDS instructions per K step
  typedef typename Frag<E>::T F;
  int at[TR ? (F32 ? 1 : 2 * NB) : 4];

  __device__ __forceinline__ void init(int w0, int lane) {
    if constexpr (!TR) {
#pragma unroll
      for (int s = 0; s < 4; ++s) at[s] = frag_off(w0, lane, s);
    } else if constexpr (F32) {
      at[0] = 4 * (lane >> 5) * ROWB + (w0 + (lane & 31)) * 4;
    } else {
      const int h = lane >> 5, g = (lane >> 4) & 1, i = lane & 15;
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          const int row = 8 * h + 4 * r + (i >> 2);
          const int seg = w0 / 16 + 2 * b + g;
          at[2 * b + r] = row * ROWB + ((seg ^ seg_swz<ROWB>(row)) << 5) + 8 * (i & 3);
        }
    }
  }
  // The other stage's addresses (the stages differ in one address bit).
  template <int STAGE>
  __device__ __forceinline__ void flip() {
#pragma unroll
    for (int i = 0; i < int(sizeof(at) / sizeof(at[0])); ++i) at[i] ^= STAGE;
  }
  // LDS instruction r (0 .. READS - 1) of K step s.
  // (st: the slab's place in LDS; at[] holds the stage.)
  __device__ __forceinline__ void read(const char* st, int s, int r, F (&f)[NB]) const {
    if constexpr (!TR) {
      f[r] = *reinterpret_cast<const F*>(st + at[s] + r * 4096);
    } else if constexpr (F32) {
      f[r / 4][r % 4] = *reinterpret_cast<const float*>(st + at[0] + (8 * s + r % 4) * ROWB + (r / 4) * 128);
    } else {
      const i16x4 v = lds_tr16(st + at[r] + s * 16 * ROWB);
      i16x8 x = __builtin_bit_cast(i16x8, f[r / 2]);
#pragma unroll
      for (int e = 0; e < 4; ++e) x[4 * (r & 1) + e] = v[e];
      f[r / 2] = __builtin_bit_cast(F, x);
    }
  }
};

template <typename E>
__device__ __forceinline__ f32x16 mfma(const typename Frag<E>::T& a, const typename Frag<E>::T& b, f32x16 c, int q) {
  if constexpr (sizeof(E) == 2)
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_32x32x2f32(a[q], b[q], c, 0, 0, 0);
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

// Where a block works: its tile's corner and extent in C, its operands, its K range.
template <typename E>
struct Work {
  const E* a;     // the tile's first row (column) at the range's first K
  const E* b;
  E* c;           // C(0, 0) of the product or of its expert
  int64_t m0, n0;
  int rows, cols; // rows and columns of the tile that exist
  int K;          // elements of the K range
};

// The blocks of an XCD (consecutive multiples of 8 apart) take consecutive
// tiles, so that its 32 CUs share operand panels in its L2.
__device__ __forceinline__ int xcd_order(int pid, int total) {
  const int q = total >> 3, r = total & 7, x = pid & 7, i = pid >> 3;
  return x * q + min(x, r) + i;
}
// The same in runs of `run` tiles per XCD, for a number of tiles that only the
// GPU knows: pid, rounded up to whole rounds of 8 runs, may name no tile.
__device__ __forceinline__ int xcd_runs(int pid, int run) {
  const int round = pid / (8 * run), r = pid % (8 * run);
  return (round * 8 + (r & 7)) * run + (r >> 3);
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

template <typename E, int TM, int TN, int FORM, int GROUP>
__device__ __forceinline__ bool locate(const Product& p, const typename TableOf<GROUP>::T& tab, int run, int lane, Work<E>& w) {
  const int nt = (p.N + TN - 1) / TN, mt = (p.M + TM - 1) / TM;
  const E* a = static_cast<const E*>(p.a);
  const E* b = static_cast<const E*>(p.b);
  w.c = static_cast<E*>(p.c);
  int k0 = 0, k1 = p.K;
  int ni;
  if constexpr (GROUP == GROUP_ROWS) {
    const int id = xcd_runs(blockIdx.x, run);
    RowTile t;
    if (!find_row_tile<TM>(p.offsets, p.experts, p.M, id / nt, lane, t)) return false;
    ni = id % nt;
    w.m0 = t.row0;
    w.rows = t.rows;
    if (t.expert < 0) k1 = 0;
    b = static_cast<const E*>(tab.p[max(t.expert, 0)]);
  } else {
    int id, mi;
    if constexpr (GROUP == GROUP_SUM) {
      id = xcd_runs(blockIdx.x, run);
      const int e = id / (mt * nt);
      if (e >= p.experts) return false;
      id -= e * (mt * nt);
      w.c = const_cast<E*>(static_cast<const E*>(tab.p[e]));
      if (!w.c) return false;
      expert_range(p.offsets, e, p.K, lane, k0, k1);
    } else {
      id = xcd_order(blockIdx.x, mt * nt);
      const int slabs = (p.K + Tile<E, TM, TN>::BK - 1) / Tile<E, TM, TN>::BK;
      const int per = (slabs + p.splits - 1) / p.splits * Tile<E, TM, TN>::BK;
      k0 = min(p.K, int(blockIdx.y) * per);
      k1 = min(p.K, k0 + per);
    }
    // bands of 8 tile rows, column by column
    const int band = id / (8 * nt), in = id - band * 8 * nt, h = min(8, mt - band * 8);
    ni = in / h;
    mi = band * 8 + in - ni * h;
    w.m0 = int64_t(mi) * TM;
    w.rows = min(TM, p.M - int(w.m0));
  }
  w.n0 = int64_t(ni) * TN;
  w.cols = min(TN, p.N - int(w.n0));
  w.K = k1 - k0;
  w.a = FORM == FORM_TT ? a + k0 * p.lda + w.m0 : a + w.m0 * p.lda + k0;
  w.b = FORM == FORM_RR ? b + w.n0 * p.ldb + k0 : b + k0 * p.ldb + w.n0;
  return true;
}

template <typename E, int TM, int TN, int FORM, int GROUP>
__global__ __launch_bounds__(256, TM* TN >= 256 * 256 ? 1 : 2) void mm_tile_kernel(
    Product p, typename TableOf<GROUP>::T tab, int run) {
  using C = Tile<E, TM, TN>;
  constexpr bool ATR = FORM == FORM_TT, BTR = FORM != FORM_RR;
  __shared__ __attribute__((aligned(2 * C::STAGE))) char lds[2 * C::STAGE];
  const int lane = threadIdx.x & 63, wid = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  Work<E> w;
  if (!locate<E, TM, TN, FORM, GROUP>(p, tab, run, lane, w)) return;
  const int wm = (wid >> 1) * C::WTM, wn = (wid & 1) * C::WTN;

  using LA = Loader<E, TM, ATR>;
  using LB = Loader<E, TN, BTR>;
  using RA = Reader<E, TM, C::NBM, ATR>;
  using RB = Reader<E, TN, C::NBN, BTR>;
  typedef typename Frag<E>::T F;
  LA la;
  LB lb;
  RA ra;
  RB rb;
  la.init(w.a, p.lda, w.rows, wid, lane);
  lb.init(w.b, p.ldb, w.cols, wid, lane);
  ra.init(wm, lane);
  rb.init(wn, lane);

  f32x16 acc[C::NBM][C::NBN];
#pragma unroll
  for (int i = 0; i < C::NBM; ++i)
#pragma unroll
    for (int j = 0; j < C::NBN; ++j)
#pragma unroll
      for (int q = 0; q < 16; ++q) acc[i][j][q] = 0.f;

  const int nk = (w.K + C::BK - 1) / C::BK;
  int kleft = w.K;   // K elements from the next slab to load on
  constexpr int LOADS = LA::N + LB::N;
  // load number i of the next slab (A's, then B's)
  auto load_one = [&](int i, uint32_t to) {
    if (i < LA::N)
      la.load(i, to, wid, kleft);
    else
      lb.load(i - LA::N, to + C::ABYTES, wid, kleft);
  };
  auto loaded = [&]() {
    la.next();
    lb.next();
    kleft -= C::BK;
  };

  F fa[2][C::NBM], fb[2][C::NBN];
  constexpr int READS = RA::READS + RB::READS;
  constexpr int Q = sizeof(E) == 2 ? 1 : 4;               // MFMAs per block and K step
  constexpr int MFMAS = C::NBM * C::NBN * Q;
  auto read_one = [&](int s, int r, int buf) {
    if (r < RB::READS)
      rb.read(lds + C::ABYTES, s, r, fb[buf]);
    else
      ra.read(lds, s, r - RB::READS, fa[buf]);
  };
  // MFMAs of a K step (fragments buf) with the reads of step rs and, with
  // LOAD, the loads of a slab spread over them.  No branch surrounds an MFMA:
  // the accumulators would be copied where the paths meet.
  auto k_step = [&](auto load_tag, int rs, int buf, uint32_t to) {
    constexpr bool LOAD = decltype(load_tag)::value;
#pragma unroll
    for (int t = 0; t < MFMAS; ++t) {
#pragma unroll
      for (int r = 0; r < READS; ++r)
        if (r * MFMAS / READS == t) read_one(rs, r, buf ^ 1);
      if constexpr (LOAD) {
#pragma unroll
        for (int i = 0; i < LOADS; ++i)
          if (i * MFMAS / LOADS == t) load_one(i, to);
      }
      const int q = t / (C::NBM * C::NBN), ij = t % (C::NBM * C::NBN), i = ij / C::NBN, j = ij % C::NBN;
      acc[i][j] = mfma<E>(fb[buf][j], fa[buf][i], acc[i][j], q);
      __builtin_amdgcn_sched_barrier(0);
    }
  };

  if (nk > 0) {
    uint32_t to = lds_addr(lds);
#pragma unroll
    for (int i = 0; i < LOADS; ++i) load_one(i, to);
    loaded();
#pragma unroll
    for (int i = 0; i < LOADS; ++i) load_one(i, to + C::STAGE);
    loaded();
    asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"i"(LOADS) : "memory");
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int r = 0; r < READS; ++r) read_one(0, r, 0);
    for (int kt = 0; kt < nk; ++kt) {
      k_step(BoolTag<false>{}, 1, 0, 0);
      k_step(BoolTag<false>{}, 2, 1, 0);
      k_step(BoolTag<false>{}, 3, 0, 0);
      asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
      __builtin_amdgcn_sched_barrier(0);
      ra.template flip<C::STAGE>();
      rb.template flip<C::STAGE>();
      k_step(BoolTag<true>{}, 0, 1, to);
      loaded();
      to ^= C::STAGE;
    }
    // the last slabs' loads (past K) and reads end before the block does
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
  }

  // ---------------------------------------------------------------- epilogue
  // Element q of block (i, j): row 32 i + lane % 32, column 32 j + 8 (q / 4) +
  // 4 (lane / 32) + q % 4.
  const int h = lane >> 5;
  const E* bias = static_cast<const E*>(p.bias);
  const E* res = static_cast<const E*>(p.res);
  E* z = static_cast<E*>(p.z);
  with_act(p.act, [&](auto act_tag) {
    constexpr int ACT = decltype(act_tag)::value;
#pragma unroll
    for (int j = 0; j < C::NBN; ++j)
#pragma unroll
      for (int g = 0; g < 4; g += 2) {
        const int col = wn + 32 * j + 8 * g + 8 * h;
        const int n = w.cols - col;
        float bv[8] = {};
        if (bias && n > 0) load8(bias + w.n0 + col, n, bv);
#pragma unroll
        for (int i = 0; i < C::NBM; ++i) {
          const int row = wm + 32 * i + (lane & 31);
          float v[8];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            // the upper half of group g against the lower half of group g + 1
            // (values of their own: a bit cast of a vector's element takes element 0)
            const float lo = acc[i][j][4 * g + e], hi = acc[i][j][4 * g + 4 + e];
            const auto s = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, lo),
                                                            __builtin_bit_cast(uint32_t, hi), false, false);
            const uint32_t s0 = s[0], s1 = s[1];
            v[e] = __builtin_bit_cast(float, s0);
            v[4 + e] = __builtin_bit_cast(float, s1);
          }
          if (row >= w.rows || n <= 0) continue;
          const int64_t m = w.m0 + row, c = w.n0 + col;
          if (p.splits > 1) {
            store8(p.part + (int64_t(blockIdx.y) * p.M + m) * p.N + c, n, v);
            continue;
          }
#pragma unroll
          for (int e = 0; e < 8; ++e) v[e] += bv[e];
          if (z) store8(z + m * p.ldz + c, n, v);
#pragma unroll
          for (int e = 0; e < 8; ++e) v[e] = act_one<ACT>(v[e]);
          if (res) {
            float rv[8];
            load8(res + m * p.ldr + c, n, rv);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] += rv[e];
          }
          store8(w.c + m * p.ldc + c, n, v);
        }
      }
  });
}

// Tiles in a row that one XCD takes of a grouped product (xcd_runs).
template <int GROUP>
int run_length(int64_t mt, int64_t nt) {
  return int(GROUP == GROUP_ROWS ? 2 * nt : mt * nt);
}

template <typename E, int TM, int TN, int FORM, int GROUP>
hipError_t launch_one(const Product& p, const Table* t, hipStream_t st) {
  const int64_t nt = (int64_t(p.N) + TN - 1) / TN, mt = (int64_t(p.M) + TM - 1) / TM;
  int64_t blocks = nt * mt;
  int run = 1;
  if constexpr (GROUP == GROUP_ROWS) blocks = nt * row_tiles_bound(p.M, p.experts, TM);
  if constexpr (GROUP == GROUP_SUM) blocks *= p.experts;
  if constexpr (GROUP != GROUP_NONE) {
    const int64_t want = run_length<GROUP>(mt, nt), most = (blocks + 7) / 8;
    run = int(want < most ? want : most);
    if (run < 1) run = 1;
    blocks = (blocks + 8 * run - 1) / (8 * run) * (8 * run);
  }
  if (blocks >= (int64_t(1) << 24)) return hipErrorInvalidConfiguration;
  if (!blocks) return hipSuccess;
  const dim3 g{unsigned(blocks), unsigned(p.splits)}, b{256};
  if constexpr (GROUP == GROUP_NONE)
    hipLaunchKernelGGL((mm_tile_kernel<E, TM, TN, FORM, GROUP>), g, b, 0, st, p, NoTable{}, run);
  else
    hipLaunchKernelGGL((mm_tile_kernel<E, TM, TN, FORM, GROUP>), g, b, 0, st, p, *t, run);
  return hipGetLastError();
}

// The forms and groupings the layers use.
template <typename E, int TM, int TN>
hipError_t launch_form(int form, int group, const Product& p, const Table* t, hipStream_t st) {
  if (group == GROUP_SUM) return launch_one<E, TM, TN, FORM_TT, GROUP_SUM>(p, t, st);
  if (group == GROUP_ROWS)
    return form == FORM_RT ? launch_one<E, TM, TN, FORM_RT, GROUP_ROWS>(p, t, st)
                           : launch_one<E, TM, TN, FORM_RR, GROUP_ROWS>(p, t, st);
  if (form == FORM_RT) return launch_one<E, TM, TN, FORM_RT, GROUP_NONE>(p, t, st);
  if (form == FORM_RR) return launch_one<E, TM, TN, FORM_RR, GROUP_NONE>(p, t, st);
  return launch_one<E, TM, TN, FORM_TT, GROUP_NONE>(p, t, st);
}

}  // namespace
}  // namespace layers
}  // namespace muon

#endif  // MUON_LAYERS_MM_TILE_H
