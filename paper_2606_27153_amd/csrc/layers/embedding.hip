// Rows of a table by token, scaled, and the table's gradient.
//
//   y[i] = s W[id[i]],   dW[v] = s sum of dy[i] over the i with id[i] = v
//
// Forward: a copy of rows, a thread per 8 columns.
//
// Backward: the tokens are sorted (sort.h), so that a table row's gradient is a sum
// over a run of the sorted list, in the list's order: no atomics, the result does
// not depend on timing.  Every row of dW is written once, by the block that has
// it: the sum of its run, or zeros (most of a large table).  A frequent token's run
// can be a good part of the list: groups of 16 places that lie inside one run are
// summed first, by blocks of their own, and the row adds up the groups.
// Bound by memory: dy read once, dW written once.  32768 tokens (their frequency
// falling with their rank) of a table of 128000 x 4096 in bf16: forward 73 us, 86
// after a backward pass (6.2 TB/s, with what the caches have of frequent rows); backward
// 275 us, of which the sort takes 30 in four launches, the groups 24 and the table's
// rows 222 (1.05 GB written, past the caches' order of use: 243 as ordinary stores).
// A token's groups are added up in one thread for each 8 columns: of 32768 x 4096 gradients
// with one token at half of the places 317 us for 260 without it, of 131072 x 1024 450 for 177.
// With groups of 64, the block of the most frequent token ended last, and each block
// searching its own rows' runs waited for that: 522 us for the table's rows.
#include "sort.h"

namespace muon {
namespace layers {
namespace {

// One digit of the tokens' numbers.  Those outside the table count as `vocab`, the
// largest, and come last.
struct TokenJob {
  const void* ids;         // first digit: the tokens themselves
  const int32_t* keys;     // later ones: as the digit before left them
  const int32_t* index;
  int32_t* keys_out;
  int32_t* index_out;
  int32_t id_bytes, vocab, shift, bins, bits;
  __device__ __forceinline__ int digit(int i, int& key) const {
    if (ids) {
      const int64_t v = id_at(ids, id_bytes, i);
      key = v >= 0 && v < vocab ? int(v) : vocab;
    } else {
      key = keys[i];
    }
    return (key >> shift) & (kSortBins - 1);
  }
  __device__ __forceinline__ void start(int, int) const {}
  __device__ __forceinline__ void put(int i, int key, int, int place) const {
    keys_out[place] = key;
    index_out[place] = ids ? i : index[i];
  }
};

// FAR: stored past the caches' order of use.  32768 x 4096 in bf16 then take 73 us for 92,
// and 194 for 203 with the norm that reads them; of 32 MB the norm finds most in the caches
// (9 for 11, and 27 for 25).  At 64 MB both are alike.
constexpr int64_t kFar = int64_t(1) << 26;   // bytes beyond which the output is stored so
template <typename E, bool WHOLE, bool FAR>
__global__ __launch_bounds__(256) void lookup_kernel(EmbeddingArgs a) {
  const int chunks = (a.cols + 7) / 8;
  const int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x, r = i / chunks;
  if (r >= a.rows) return;
  const int c = int(i - r * chunks) * 8, n = min(8, a.cols - c);
  const int64_t id = id_at(a.ids, a.id_bytes, r);
  const bool live = id >= 0 && id < a.vocab;
  float v[8];
  load_8<WHOLE>(static_cast<const E*>(a.w) + (live ? id : 0) * a.ldw + c, n, v);
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = live ? v[e] * a.scale : 0.f;
  E* to = static_cast<E*>(a.y) + r * a.ldy + c;
  if constexpr (FAR)
    store_8_once<WHOLE>(to, n, v);
  else
    store_8<WHOLE>(to, n, v);
}

constexpr int kRun = 16;    // places of a group
constexpr int kRows = 16;   // table rows of a block

// v[0..7] += the gradients of places lo .. hi - 1, in order, 4 in flight.  ONCE: past the
// caches' order of use (the groups' 25 us for 41; rows of a few places, next to the
// table's stores, lose 3%).
template <typename E, bool WHOLE, bool ONCE>
__device__ __forceinline__ void add_run(const EmbeddingArgs& a, int lo, int hi, int c, int n, float (&v)[8]) {
  const E* dy = static_cast<const E*>(a.dy) + c;
  for (int p = lo; p < hi; p += 4) {
    int64_t row[4];
    float x[4][8];
#pragma unroll
    for (int k = 0; k < 4; ++k) row[k] = a.index[min(p + k, hi - 1)];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if constexpr (ONCE)
        load_8_once<WHOLE>(dy + row[k] * a.lddy, n, x[k]);
      else
        load_8<WHOLE>(dy + row[k] * a.lddy, n, x[k]);
    }
#pragma unroll
    for (int k = 0; k < 4; ++k)
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] += p + k < hi ? x[k][e] : 0.f;
  }
}
// v[0..7] += the sums of groups g0 .. g1 - 1, 8 in flight.
template <bool WHOLE>
__device__ __forceinline__ void add_groups(const EmbeddingArgs& a, int g0, int g1, int c, int n, float (&v)[8]) {
  for (int g = g0; g < g1; g += 8) {
    float x[8][8];
#pragma unroll
    for (int k = 0; k < 8; ++k) load_8<WHOLE>(a.part + int64_t(min(g + k, g1 - 1)) * a.cols + c, n, x[k]);
#pragma unroll
    for (int k = 0; k < 8; ++k)
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] += g + k < g1 ? x[k][e] : 0.f;
  }
}

// Blocks y > 0: the sums of the groups of places inside one run (the others' places
// in `part` stay as they are).  Blocks y = 0: where the tokens' runs begin, the first place
// of at least that token.
template <typename E, bool WHOLE>
__global__ __launch_bounds__(256) void group_kernel(EmbeddingArgs a, int groups) {
  if (blockIdx.y == 0) {
    const int64_t want = int64_t(blockIdx.x) * 256 + threadIdx.x;
    if (want > a.vocab) return;
    int lo = 0, hi = a.rows;
    while (lo < hi) {
      const int mid = (lo + hi) >> 1;
      if (a.keys[mid] < want)
        lo = mid + 1;
      else
        hi = mid;
    }
    a.starts[want] = lo;
    return;
  }
  if (int(blockIdx.x) >= groups) return;
  const int first = blockIdx.x * kRun;
  const int key = a.keys[first];
  if (key >= a.vocab || a.keys[first + kRun - 1] != key) return;
  const int c = ((blockIdx.y - 1) * 256 + threadIdx.x) * 8, n = min(8, a.cols - c);
  if (n <= 0) return;
  float v[8] = {};
  add_run<E, WHOLE, true>(a, first, first + kRun, c, n, v);
  store_8<WHOLE>(a.part + int64_t(blockIdx.x) * a.cols + c, n, v);
}

// A thread has 8 columns of 16 table rows: those of no token first, which wait for
// nothing but where the runs begin, then the others' sums.
template <typename E, bool WHOLE>
__global__ __launch_bounds__(256) void table_grad_kernel(EmbeddingArgs a) {
  const int chunks = (a.cols + 7) / 8;
  const int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x, v0 = i / chunks * kRows;
  if (v0 >= a.vocab) return;
  const int c = int(i % chunks) * 8, n = min(8, a.cols - c);
  E* to = static_cast<E*>(a.dw) + v0 * a.lddw + c;
  int start[kRows + 1];
#pragma unroll
  for (int r = 0; r <= kRows; ++r) start[r] = a.rows ? a.starts[min(v0 + r, int64_t(a.vocab))] : 0;
  const float zero[8] = {};
  uint32_t met = 0;
#pragma unroll
  for (int r = 0; r < kRows; ++r) {
    if (start[r] < start[r + 1])
      met |= 1u << r;
    else if (v0 + r < a.vocab)
      store_8_run<WHOLE>(to + r * a.lddw, n, zero);
  }
  while (met) {
    const int r = __builtin_ctz(met);
    met &= met - 1;
    const int lo = a.starts[v0 + r], hi = a.starts[v0 + r + 1];
    float v[8] = {};
    const int g0 = (lo + kRun - 1) / kRun, g1 = hi / kRun;
    if (g0 < g1) {
      add_run<E, WHOLE, false>(a, lo, g0 * kRun, c, n, v);
      add_groups<WHOLE>(a, g0, g1, c, n, v);
      add_run<E, WHOLE, false>(a, g1 * kRun, hi, c, n, v);
    } else {
      add_run<E, WHOLE, false>(a, lo, hi, c, n, v);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] *= a.scale;
    store_8_run<WHOLE>(to + r * a.lddw, n, v);
  }
}

template <typename E, bool WHOLE>
hipError_t forward(const EmbeddingArgs& a, hipStream_t st) {
  const int64_t blocks = (int64_t(a.rows) * ((a.cols + 7) / 8) + 255) / 256;
  if (blocks >= kMaxGrid) return hipErrorInvalidConfiguration;
  const dim3 g{unsigned(blocks)}, b{256};
  if (int64_t(a.rows) * a.cols * int64_t(sizeof(E)) > kFar)
    hipLaunchKernelGGL((lookup_kernel<E, WHOLE, true>), g, b, 0, st, a);
  else if (blocks)
    hipLaunchKernelGGL((lookup_kernel<E, WHOLE, false>), g, b, 0, st, a);
  return hipGetLastError();
}

template <typename E, bool WHOLE>
hipError_t backward(EmbeddingArgs a, int32_t* const (&keys)[2], int32_t* const (&index)[2], int32_t* counts,
                    hipStream_t st) {
  const int64_t groups = a.rows / kRun, starts = (int64_t(a.vocab) + 256) / 256;
  const int64_t blocks = ((int64_t(a.vocab) + kRows - 1) / kRows * ((a.cols + 7) / 8) + 255) / 256;
  if (blocks >= kMaxGrid || groups >= kMaxGrid) return hipErrorInvalidConfiguration;
  int at = 0;
  for (int shift = 0; a.rows && (shift == 0 || (a.vocab >> shift)); shift += kSortBits, at ^= 1) {
    TokenJob job{};
    if (shift == 0) job.ids = a.ids;
    job.keys = keys[at ^ 1];
    job.index = index[at ^ 1];
    job.keys_out = keys[at];
    job.index_out = index[at];
    job.id_bytes = a.id_bytes;
    job.vocab = a.vocab;
    job.shift = shift;
    for (job.bits = 1; job.bits < kSortBits && (a.vocab >> shift >> job.bits); ++job.bits) {
    }
    job.bins = 1 << job.bits;
    const hipError_t e = launch_sort(job, a.rows, counts, st);
    if (e != hipSuccess) return e;
  }
  a.keys = keys[at ^ 1];
  a.index = index[at ^ 1];
  if (a.rows) {
    const dim3 g{unsigned(groups > starts ? groups : starts), unsigned((a.cols + 2047) / 2048 + 1)};
    hipLaunchKernelGGL((group_kernel<E, WHOLE>), g, dim3{256}, 0, st, a, int(groups));
  }
  hipLaunchKernelGGL((table_grad_kernel<E, WHOLE>), dim3{unsigned(blocks)}, dim3{256}, 0, st, a);
  return hipGetLastError();
}

size_t whole(size_t v) { return (v + 255) / 256 * 256; }

}  // namespace

size_t embedding_bytes(int64_t rows, int64_t vocab, int64_t cols) {
  return 4 * whole(size_t(rows) * 4) + whole(sort_bytes(rows)) + whole((size_t(vocab) + 1) * 4) +
         whole(size_t(rows / kRun) * size_t(cols) * 4);
}

hipError_t launch_embedding_forward(bool bf16, const EmbeddingArgs& a, hipStream_t st) {
  if (a.cols % 8) return bf16 ? forward<__bf16, false>(a, st) : forward<float, false>(a, st);
  return bf16 ? forward<__bf16, true>(a, st) : forward<float, true>(a, st);
}

hipError_t launch_embedding_backward(bool bf16, EmbeddingArgs a, void* workspace, hipStream_t st) {
  char* p = static_cast<char*>(workspace);
  const size_t step = whole(size_t(a.rows) * 4);
  int32_t* const keys[2] = {reinterpret_cast<int32_t*>(p), reinterpret_cast<int32_t*>(p + step)};
  int32_t* const index[2] = {reinterpret_cast<int32_t*>(p + 2 * step), reinterpret_cast<int32_t*>(p + 3 * step)};
  int32_t* counts = reinterpret_cast<int32_t*>(p + 4 * step);
  p += 4 * step + whole(sort_bytes(a.rows));
  a.starts = reinterpret_cast<int32_t*>(p);
  a.part = reinterpret_cast<float*>(p + whole((size_t(a.vocab) + 1) * 4));
  if (a.cols % 8)
    return bf16 ? backward<__bf16, false>(a, keys, index, counts, st)
                : backward<float, false>(a, keys, index, counts, st);
  return bf16 ? backward<__bf16, true>(a, keys, index, counts, st) : backward<float, true>(a, keys, index, counts, st);
}

}  // namespace layers
}  // namespace muon
