// Matrix products on the matrix cores, one block of four waves per TM x TN
// tile of C.
//
// K advances in slabs of 128 bytes of a K-contiguous row (64 bf16, 32 fp32).  An
// operand's slab is a unit of the LDS ring, filled straight from global memory
// (16 bytes per lane and instruction).  A "row" operand's unit holds its rows,
// 128 bytes each; a "tr" operand's holds BK rows of TM (TN) elements as they
// lie in memory, and the fragment reads transpose: ds_read_b64_tr_b16 for bf16, single
// words for fp32.  16-byte chunks (32-byte segments) are XOR-swizzled with the
// row so that the fragment reads are free of bank conflicts.
//
// Each wave owns a (TM / 2) x (TN / 2) piece of 32 x 32 MFMA blocks.  A slab is
// four K steps; the fragments of the next step are read while the current
// step's MFMAs run, one memory instruction per MFMA or so.  The ring has U
// units, A's and B's slabs in turn; before the last step of a slab comes the
// slab's only barrier (every wave has read the slab, the next one has landed),
// which frees two units.  The loads of the first go out during that step, those
// of the second over the next two: the path from the caches to LDS moves 64
// bytes a cycle, half of which the 256 tile needs, so a burst of all of them
// would hold up the MFMAs behind it.  5 units of the 256 tile (two blocks of
// the 128 tile) fill the 160 KB.
//
// The MFMAs take B as their first operand, so a lane holds 4 consecutive columns
// of a row of C, which the epilogue moves 16 bytes at a time (store_piece).
//
// Rows and columns past the edge of C read the last valid ones again; their
// sums are never stored.  Where K ends inside a slab, the chunks past it come
// from a block of zeros.
//
// Bound by the matrix cores and the chip's power (71% of the cycles are MFMA's at
// 1.4 GHz on 16384 x 14336 x 4096): launched back to back, 256 x 256 tiles take 794 to
// 805 us on 8192^3 with K-contiguous operands (1365 to 1385 TFLOP/s), 822 to 825 with a
// tr B, 825 to 833 with both tr, and reach 1295 TFLOP/s on 16384 x 14336 x 4096.  Four
// waves of 128 x 128 read half the LDS bytes per MFMA of eight of 128 x 64; with one
// wave per SIMD nothing hides a wave's own waits, which is what the ring and the spread
// loads are for (two whole-slab stages, loaded in one burst, took 13% longer on
// 8192^3).  128 x 256 tiles reach 1130 to 1215 TFLOP/s there, 128 x 128 with two
// blocks per CU 1060 to 1105, and fill the chip from a quarter of the size on; 64 x 64
// (560 to 670) serves products of a few hundred rows (1024 x 2048 x 2048 17 us).  fp32
// runs at 137 to 139 TFLOP/s on 128 x 128 tiles (4096^3, every form; 123 to 127 on
// 64 x 64), 154 being what the matrix cores sustain.
#ifndef MUON_LAYERS_MM_TILE_H
#define MUON_LAYERS_MM_TILE_H

#include "../ns_gemm_kernel.h"
#include "device.h"

namespace muon {
namespace layers {
namespace {

template <typename E, int TM_, int TN_, int U_>
struct Tile {
  static constexpr int TM = TM_, TN = TN_;          // C's tile
  static constexpr int U = U_;                      // units of the LDS ring
  static constexpr int EPC = 16 / int(sizeof(E));   // elements of a 16-byte chunk
  static constexpr int BK = 8 * EPC;                // K elements of a slab
  static constexpr int WTM = TM / 2, WTN = TN / 2;  // wave piece
  static constexpr int NBM = WTM / 32, NBN = WTN / 32;
  static constexpr int UA = TM * 128, UB = TN * 128;  // bytes of an operand's slab
  static_assert(TM == TN || U % 2 == 0, "a slot holds A's and B's slabs in turn where U is odd");
  // unit u's place in the ring, and the ring's bytes
  static constexpr int at(int u) { return u / 2 * (UA + UB) + (u & 1) * UA; }
  static constexpr int RING = U % 2 ? U * UA : U / 2 * (UA + UB);
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
  int left;              // K elements from the slab's first one on
  int k;                 // this lane's K element (row operand) or K row (tr operand) in its first chunk

  // op: the tile's corner (row or column 0, the first K); ld in elements;
  // valid: rows or columns of the tile that exist (>= 1).
  __device__ __forceinline__ void init(const E* op, int64_t ld, int valid, int K, int wid, int lane) {
    base = reinterpret_cast<const char*>(op);
    left = K;
    if constexpr (TR) {
      const int row = wid * RPC + lane / LPR, slot = lane % LPR;
      int chunk = slot;
      if constexpr (sizeof(E) == 2) chunk = (((slot >> 1) ^ seg_swz<ROWB>(row)) << 1) | (slot & 1);
      const int col = min(chunk * EPC, (valid + EPC - 1) / EPC * EPC - EPC);  // (rows are whole chunks)
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
  // Load i of the slab (past the end of K: zeros, which nothing reads; they
  // only keep the count of loads).
  __device__ __forceinline__ void load(int i, uint32_t lds, int wid) const {
    const bool in = k + (TR ? 4 * RPC * i : 0) < left;
    const char* from = base + (TR ? off[0] + i * stride : off[i]);
    dma16_to(in ? from : reinterpret_cast<const char*>(kZeros), lds + (wid + 4 * i) * 1024);
  }
  __device__ __forceinline__ void next() {
    base += step;
    left -= BK;
  }
};

// One operand's fragment reads.  NB 32-row blocks from row (column) w0 of the slab.
template <typename E, int T, int NB, bool TR>
struct Reader {
  static constexpr int ROWB = TR ? T * int(sizeof(E)) : 128;
  static constexpr bool F32 = sizeof(E) == 4;
  static constexpr int READS = !TR ? NB : F32 ? 4 * NB : 2 * NB;   // LDS instructions per K step
  typedef typename Frag<E>::T F;
  static constexpr int ADDRS = TR ? (F32 ? 1 : 2 * NB) : 4;
  int at[ADDRS];   // in the current unit

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
  // On to the unit `bytes` further in the ring.
  __device__ __forceinline__ void move(int bytes) {
#pragma unroll
    for (int i = 0; i < ADDRS; ++i) at[i] += bytes;
  }
  // LDS instruction r (0 .. READS - 1) of K step s.
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

template <bool FIRST, class A, class B>
__device__ __forceinline__ auto& pick(A& a, B& b) {
  if constexpr (FIRST)
    return a;
  else
    return b;
}

template <typename E>
__device__ __forceinline__ f32x16 mfma(const typename Frag<E>::T& a, const typename Frag<E>::T& b, f32x16 c, int q) {
  if constexpr (sizeof(E) == 2)
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_32x32x2f32(a[q], b[q], c, 0, 0, 0);
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

template <typename E, int TM, int TN, int U, int FORM, int GROUP>
__device__ __forceinline__ bool locate(const Product& p, const typename TableOf<GROUP>::T& tab, int pid, int run,
                                       int lane, const Ranks& ranks, Work<E>& w) {
  const int nt = (p.N + TN - 1) / TN, mt = (p.M + TM - 1) / TM;
  const E* a = static_cast<const E*>(p.a);
  const E* b = static_cast<const E*>(p.b);
  w.c = static_cast<E*>(p.c);
  int k0 = 0, k1 = p.K;
  int ni;
  if constexpr (GROUP != GROUP_SUM) {   // this block's range of K: whole slabs
    constexpr int BK = Tile<E, TM, TN, U>::BK;
    const int slabs = (p.K + BK - 1) / BK, per = (slabs + p.splits - 1) / p.splits * BK;
    k0 = min(p.K, int(blockIdx.y) * per);
    k1 = min(p.K, k0 + per);
  }
  if constexpr (GROUP == GROUP_ROWS) {
    const int id = xcd_runs(pid, run);
    RowTile t;
    if (!find_row_tile<TM>(p.offsets, p.experts, p.M, id / nt, lane, t)) return false;
    ni = id % nt;
    w.m0 = t.row0;
    w.rows = t.rows;
    if (t.expert < 0) k1 = k0;
    b = static_cast<const E*>(tab.p[max(t.expert, 0)]);
  } else {
    int id, mi;
    if constexpr (GROUP == GROUP_SUM) {
      id = xcd_runs(pid, run);
      const int at = id / (mt * nt);
      if (at >= p.experts) return false;
      id -= at * (mt * nt);
      const int e = expert_of_rank(ranks, at);
      w.c = const_cast<E*>(static_cast<const E*>(tab.p[e]));
      if (!w.c) return false;
      expert_range(p.offsets, e, p.K, lane, k0, k1);
    } else {
      id = xcd_order(pid, mt * nt);
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

// The epilogue of a wave's piece.  Element q of block (i, j) is row 32 i +
// lane % 32, column 32 j + 8 (q / 4) + 4 (lane / 32) + q % 4.  32 rows at a time
// pass through the wave's own part of the ring (free by then) in fp32, so that a
// lane then has 8 consecutive columns of a row, the same columns every time, and
// every access to C, the residual and z is of whole lines.  (Stored from the
// registers in pieces of 32 bytes a row, the weight gradients of 64 experts of
// 1408 x 2048 took 224 us, 75 of them for the stores.)  A lane's vector
// instructions count: with one wave per SIMD nothing else runs meanwhile.  OUT:
// the type stored (E, or float for partial results, which get no epilogue).
// RAGGED: C's columns end inside a group of 8.
template <class C>
struct Staging {
  static constexpr int LD = C::WTN + 4;                // floats of a row: rows 4 banks apart
  static constexpr int BYTES = 32 * LD * 4;            // of a wave
  static constexpr int LPR = C::WTN / 8, RPI = 64 / LPR;  // lanes of a row, rows of a store instruction
};
template <class C, typename E, typename OUT, int ACT, bool EPI, bool RAGGED>
__device__ __forceinline__ void store_piece(const Product& p, OUT* c, int64_t ldc, const Work<E>& o,
                                            const f32x16 (&acc)[C::NBM][C::NBN], float* region, int wm, int wn,
                                            int lane) {
  using S = Staging<C>;
  const E* bias = EPI ? static_cast<const E*>(p.bias) : nullptr;
  const E* res = EPI ? static_cast<const E*>(p.res) : nullptr;
  E* z = EPI ? static_cast<E*>(p.z) : nullptr;
  const int r0 = lane / S::LPR, col = wn + lane % S::LPR * 8;   // this lane's first row of a pass, its columns
  const bool in = col < o.cols;
  const int count = RAGGED ? o.cols - col : 8;                  // columns of the lane's 8 that exist
  float bv[8] = {};
  if (bias && in) load8(bias + o.n0 + col, count, bv);
  const float* from = region + r0 * S::LD + lane % S::LPR * 8;
  float* to = region + (lane & 31) * S::LD + 4 * (lane >> 5);
  const int64_t m = o.m0 + wm + r0, n = o.n0 + col;
  OUT* cp = c + m * ldc + n;
  const E* rp = res + m * p.ldr + n;
  E* zp = z + m * p.ldz + n;
  int left = in ? o.rows - wm - r0 : 0;                         // rows from this lane's on
  static_for<C::NBM>([&](auto it) {
    constexpr int i = decltype(it)::value;
    static_for<4 * C::NBN>([&](auto jg) {
      constexpr int j = decltype(jg)::value / 4, g = decltype(jg)::value % 4;
      *reinterpret_cast<f32x4*>(to + 32 * j + 8 * g) =
          f32x4{acc[i][j][4 * g], acc[i][j][4 * g + 1], acc[i][j][4 * g + 2], acc[i][j][4 * g + 3]};
    });
#pragma unroll 2
    for (int k = 0; k < 32 / S::RPI; ++k) {
      const f32x4 lo = *reinterpret_cast<const f32x4*>(from + k * S::RPI * S::LD);
      const f32x4 hi = *reinterpret_cast<const f32x4*>(from + k * S::RPI * S::LD + 4);
      float v[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
      if (left > 0) {
        if constexpr (EPI) {
#pragma unroll
          for (int e = 0; e < 8; ++e) v[e] += bv[e];
          if (z) store8(zp, count, v);
#pragma unroll
          for (int e = 0; e < 8; ++e) v[e] = act_one<ACT>(v[e]);
          if (res) {
            float rv[8];
            load8(rp, count, rv);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] += rv[e];
          }
        }
        store8(cp, count, v);
      }
      left -= S::RPI;
      cp += S::RPI * ldc;
      if constexpr (EPI) {
        rp += S::RPI * p.ldr;
        zp += S::RPI * p.ldz;
      }
    }
  });
}

template <class C, typename E, bool EPI, bool RAGGED>
__device__ __forceinline__ void store_columns(const Product& p, const Work<E>& o,
                                              const f32x16 (&acc)[C::NBM][C::NBN], float* region, int wm, int wn,
                                              int lane) {
  if (p.splits > 1) {
    store_piece<C, E, float, MUON_ACT_NONE, false, RAGGED>(p, p.part + int64_t(blockIdx.y) * p.M * p.N, p.N, o, acc,
                                                           region, wm, wn, lane);
  } else {
    with_act<EPI>(p.act, [&](auto act) {
      store_piece<C, E, E, decltype(act)::value, EPI, RAGGED>(p, o.c, p.ldc, o, acc, region, wm, wn, lane);
    });
  }
}
template <class C, typename E, bool EPI>
__device__ __forceinline__ void store_tile(const Product& p, const Work<E>& o, const f32x16 (&acc)[C::NBM][C::NBN],
                                           float* region, int wm, int wn, int lane) {
  if (o.cols % 8)
    store_columns<C, E, EPI, true>(p, o, acc, region, wm, wn, lane);
  else
    store_columns<C, E, EPI, false>(p, o, acc, region, wm, wn, lane);
}

template <typename E, int TM, int TN, int U, int FORM, int GROUP>
__global__ __launch_bounds__(256, (Tile<E, TM, TN, U>::RING > 80 * 1024 ? 1 : 2)) void mm_tile_kernel(
    Product p, typename TableOf<GROUP>::T tab, int run, int blocks) {
  using C = Tile<E, TM, TN, U>;
  constexpr bool ATR = FORM == FORM_TT, BTR = FORM != FORM_RR;
  __shared__ __attribute__((aligned(1024))) char lds[C::RING];
  const int lane = threadIdx.x & 63, wid = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // The block's tiles: one of each round of gridDim.x.  Sums by expert take the
  // experts by falling size, and every other round in reverse, so that the blocks'
  // shares come out alike (64 experts of uneven sizes, weight gradients of 1408 x
  // 2048: in order of the experts the largest share was half as large again as
  // the mean).
  Ranks ranks;
  if constexpr (GROUP == GROUP_SUM) rank_experts(p.offsets, p.experts, p.K, lane, ranks);
  auto find = [&](int& round, Work<E>& at) {
    for (; round * int(gridDim.x) < blocks; ++round) {
      const int i = GROUP == GROUP_SUM && (round & 1) ? int(gridDim.x) - 1 - int(blockIdx.x) : int(blockIdx.x);
      const int pid = round * int(gridDim.x) + i;
      if (pid < blocks && locate<E, TM, TN, U, FORM, GROUP>(p, tab, pid, run, lane, ranks, at)) return true;
    }
    return false;
  };
  Work<E> w;
  int round = 0;
  if (!find(round, w)) return;
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
  ra.init(wm, lane);
  rb.init(wn, lane);
  rb.move(C::UA);
  const uint32_t base = lds_addr(lds);
  // The first U units of a tile's slabs.
  auto fill = [&]() {
    la.init(w.a, p.lda, w.rows, w.K, wid, lane);
    lb.init(w.b, p.ldb, w.cols, w.K, wid, lane);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (u & 1) {
#pragma unroll
        for (int i = 0; i < LB::N; ++i) lb.load(i, base + C::at(u), wid);
        lb.next();
      } else {
#pragma unroll
        for (int i = 0; i < LA::N; ++i) la.load(i, base + C::at(u), wid);
        la.next();
      }
    }
  };
  fill();

  for (;;) {
    f32x16 acc[C::NBM][C::NBN];
#pragma unroll
    for (int i = 0; i < C::NBM; ++i)
#pragma unroll
      for (int j = 0; j < C::NBN; ++j)
#pragma unroll
        for (int q = 0; q < 16; ++q) acc[i][j][q] = 0.f;
    // the next tile is looked up while this one's first loads arrive
    Work<E> next;
    ++round;
    const bool more = find(round, next);

    const int nk = (w.K + C::BK - 1) / C::BK;
    // loads of units u0 .. u1 - 1
    auto loads = [](int u0, int u1) constexpr {
      int n = 0;
      for (int u = u0; u < u1; ++u) n += u & 1 ? LB::N : LA::N;
      return n;
    };
    F fa[2][C::NBM], fb[2][C::NBN];
    constexpr int READS = RA::READS + RB::READS;
    constexpr int Q = sizeof(E) == 2 ? 1 : 4;               // MFMAs per block and K step
    constexpr int MFMAS = C::NBM * C::NBN * Q;
    auto read_one = [&](int s, int r, int buf) {
      if (r < RB::READS)
        rb.read(lds, s, r, fb[buf]);
      else
        ra.read(lds, s, r - RB::READS, fa[buf]);
    };
    // MFMAs of a K step (fragments buf) with the reads of step rs spread over the
    // first SPAN of them and the loads l0 .. l1 - 1 of a unit of operand L over
    // all; `mid` runs after MID of them.  No branch surrounds an MFMA: the
    // accumulators would be copied where the paths meet.
    constexpr int SPAN = MFMAS >= 4 ? MFMAS * 3 / 4 : MFMAS, MID = SPAN;
    auto k_step = [&](const auto& L, int l0, int l1, int rs, int buf, uint32_t to, int span, auto mid) {
#pragma unroll
      for (int t = 0; t < MFMAS; ++t) {
#pragma unroll
        for (int r = 0; r < READS; ++r)
          if (r * span / READS == t) read_one(rs, r, buf ^ 1);
#pragma unroll
        for (int i = l0; i < l1; ++i)
          if ((i - l0) * MFMAS / (l1 - l0) == t) L.load(i, to, wid);
        const int q = t / (C::NBM * C::NBN), ij = t % (C::NBM * C::NBN), i = ij / C::NBN, j = ij % C::NBN;
        acc[i][j] = mfma<E>(fb[buf][j], fa[buf][i], acc[i][j], q);
        __builtin_amdgcn_sched_barrier(0);
        if (t + 1 == MID) mid();
      }
    };
    auto nothing = []() {};

    int ua = 0, ub = C::UA;   // the current slab's units
    if (nk > 0) {
      asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"i"(loads(2, U)) : "memory");
      __builtin_amdgcn_sched_barrier(0);
      uint32_t free1 = 0;         // the unit whose loads go out in steps 0 and 1
#pragma unroll
      for (int r = 0; r < READS; ++r) read_one(0, r, 0);
      // The loads that step 3 starts go first, and are A's where U is even.
      auto& first = pick<(U & 1) == 0>(la, lb);
      auto& second = pick<(U & 1) != 0>(la, lb);
      constexpr int L = (U & 1) ? LA::N : LB::N, L1 = L / 2;   // second's loads
      constexpr int L0 = (U & 1) ? LB::N : LA::N;               // first's
      auto wrap = [](int v) { return v >= C::RING ? v - C::RING : v; };
      // Step 2 reads the slab's last fragments early and meets the other waves
      // before its own last MFMAs: this slab is read, the next one has landed;
      // U - 4 units may be in flight.
      constexpr int EARLY = MFMAS >= 4 ? MFMAS / 2 : MFMAS;
      auto publish = [&]() {
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"i"(loads(4, U)) : "memory");
        __builtin_amdgcn_sched_barrier(0);
      };
      auto last_step = [&]() {
        const uint32_t free0 = base + ua;
        free1 = base + ub;
        const int na = wrap(ua + C::UA + C::UB), nb = wrap(ub + C::UA + C::UB);
        ra.move(na - ua);
        rb.move(nb - ub);
        ua = na;
        ub = nb;
        k_step(first, 0, L0, 0, 1, free0, SPAN, nothing);
        first.next();
      };
      // The first slab's steps load nothing: every unit of the ring is taken.
      k_step(la, 0, 0, 1, 0, 0, SPAN, nothing);
      k_step(la, 0, 0, 2, 1, 0, SPAN, nothing);
      k_step(la, 0, 0, 3, 0, 0, EARLY, publish);
      last_step();
      for (int kt = 1; kt < nk; ++kt) {
        k_step(second, 0, L1, 1, 0, free1, SPAN, nothing);
        k_step(second, L1, L, 2, 1, free1, SPAN, nothing);
        second.next();
        k_step(second, 0, 0, 3, 0, 0, EARLY, publish);
        last_step();
      }
    }
    ra.move(-ua);
    rb.move(C::UA - ub);
    // the last slabs' loads (past K) and every wave's reads end here
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    static_assert(4 * Staging<C>::BYTES <= C::RING, "the waves' parts of the ring");
    store_tile<C, E, GROUP == GROUP_NONE && FORM != FORM_TT>(
        p, w, acc, reinterpret_cast<float*>(lds + wid * Staging<C>::BYTES), wm, wn, lane);
    if (!more) break;
    // every wave's part is free again for the next tile's first slabs
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    w = next;
    fill();
  }
}

// Tiles in a row that one XCD takes of a grouped product (xcd_runs), which share
// operands in its L2.  Sums by expert: a whole expert.  Rows by expert: eight rows
// of tiles, an expert or two.  At least four runs per XCD (launch_one), so that
// the XCDs' shares come out alike.
template <int GROUP>
int64_t run_length(int64_t mt, int64_t nt) {
  return GROUP == GROUP_ROWS ? 8 * nt : mt * nt;
}

template <typename E, int TM, int TN, int U, int FORM, int GROUP>
hipError_t launch_one(const Product& p, const Table* t, hipStream_t st) {
  const int64_t nt = (int64_t(p.N) + TN - 1) / TN, mt = (int64_t(p.M) + TM - 1) / TM;
  int64_t blocks = nt * mt;
  int run = 1;
  if constexpr (GROUP == GROUP_ROWS) blocks = nt * row_tiles_bound(p.M, p.experts, TM);
  if constexpr (GROUP == GROUP_SUM) blocks *= p.experts;
  if constexpr (GROUP != GROUP_NONE) {
    const int64_t want = run_length<GROUP>(mt, nt), most = blocks / 32;
    run = int(want < most ? want : most);
    if (run < 1) run = 1;
    blocks = (blocks + 8 * run - 1) / (8 * run) * (8 * run);
  }
  if (blocks >= (int64_t(1) << 24)) return hipErrorInvalidConfiguration;
  if (!blocks) return hipSuccess;
  // A block whose ring fills a CU's LDS has the CU to itself: no more of them than
  // CUs, each with several tiles.  The smaller tiles' blocks share a CU.
  int64_t grid = blocks;
  if (Tile<E, TM, TN, U>::RING > 80 * 1024 && grid > kCUs / p.splits) grid = kCUs / p.splits;
  const dim3 g{unsigned(grid), unsigned(p.splits)}, b{256};
  if constexpr (GROUP == GROUP_NONE)
    hipLaunchKernelGGL((mm_tile_kernel<E, TM, TN, U, FORM, GROUP>), g, b, 0, st, p, NoTable{}, run, int(blocks));
  else
    hipLaunchKernelGGL((mm_tile_kernel<E, TM, TN, U, FORM, GROUP>), g, b, 0, st, p, *t, run, int(blocks));
  return hipGetLastError();
}

// The forms and groupings the layers use.
template <typename E, int TM, int TN, int U>
hipError_t launch_form(int form, int group, const Product& p, const Table* t, hipStream_t st) {
  if (group == GROUP_SUM) return launch_one<E, TM, TN, U, FORM_TT, GROUP_SUM>(p, t, st);
  if (group == GROUP_ROWS)
    return form == FORM_RT ? launch_one<E, TM, TN, U, FORM_RT, GROUP_ROWS>(p, t, st)
                           : launch_one<E, TM, TN, U, FORM_RR, GROUP_ROWS>(p, t, st);
  if (form == FORM_RT) return launch_one<E, TM, TN, U, FORM_RT, GROUP_NONE>(p, t, st);
  if (form == FORM_RR) return launch_one<E, TM, TN, U, FORM_RR, GROUP_NONE>(p, t, st);
  return launch_one<E, TM, TN, U, FORM_TT, GROUP_NONE>(p, t, st);
}

}  // namespace
}  // namespace layers
}  // namespace muon

#endif  // MUON_LAYERS_MM_TILE_H
