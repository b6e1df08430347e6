// A stable counting sort by small digits: experts, or the digits of a token's
// number from the lowest up.
//
// A block places 4096 keys, its wave w the 256 from 256 w on, 64 at a time: the
// lanes that hold the same digit find each other with one ballot per bit, so that
// a key's rank among its wave's earlier ones is a count that the wave keeps plus
// the number of equal lanes before it: no atomics, the order is that of the keys.
// The counts of the waves, of the digits and (count_kernel) of the blocks before are then
// added up.  4096 keys are one launch, more are two: the counts of each block,
// then every block adds up those before its own; beyond 32 blocks a third in
// between does that once.  Latency is all that it costs: a chain of about 100 LDS
// and cross-lane steps, 4 to 5 us for up to 4096 keys, 14 us for 98304 choices among 64
// experts, 15 us for each digit of 32768 tokens.
#ifndef MUON_LAYERS_SORT_H
#define MUON_LAYERS_SORT_H

#include "device.h"

namespace muon {
namespace layers {
namespace {

constexpr int kSortThreads = 1024, kSortWaves = kSortThreads / 64, kSortItems = 4;
constexpr int kSortChunk = kSortThreads * kSortItems;
constexpr int kSortBits = 9, kSortBins = 1 << kSortBits;
constexpr int kSortNear = 32;   // blocks up to which each adds up the counts before its own

inline int sort_blocks(int64_t n) { return int((n + kSortChunk - 1) / kSortChunk); }
// Counts of every block, then the totals.
inline size_t sort_bytes(int64_t n) {
  const int b = sort_blocks(n);
  return b > 1 ? (size_t(b) + 1) * kSortBins * 4 : 0;
}

// Job: what is sorted.  digit(i, key) reads item i and says its digit; put(i, key,
// digit, place) takes its place; start(digit, first) hears, once for each digit up to
// job.bins - 1, where its items begin.
template <class Job>
__global__ __launch_bounds__(kSortThreads) void count_kernel(Job job, int n, int32_t* counts) {
  __shared__ int32_t hist[kSortBins];
  for (int d = threadIdx.x; d < job.bins; d += kSortThreads) hist[d] = 0;
  __syncthreads();
#pragma unroll
  for (int k = 0; k < kSortItems; ++k) {
    const int64_t i = int64_t(blockIdx.x) * kSortChunk + k * kSortThreads + threadIdx.x;
    int key;
    if (i < n) atomicAdd(&hist[job.digit(int(i), key)], 1);
  }
  __syncthreads();
  for (int d = threadIdx.x; d < job.bins; d += kSortThreads) counts[int64_t(blockIdx.x) * kSortBins + d] = hist[d];
}

// Of every digit, each block's count becomes the sum of those before; the totals follow the last.
__global__ __launch_bounds__(64) void prefix_kernel(int32_t* counts, int blocks, int bins) {
  const int d = blockIdx.x * 64 + threadIdx.x;
  if (d >= bins) return;
  int32_t* c = counts + d;
  int sum = 0, b = 0;
  for (; b + 8 <= blocks; b += 8) {
    int v[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = c[int64_t(b + k) * kSortBins];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      c[int64_t(b + k) * kSortBins] = sum;
      sum += v[k];
    }
  }
  for (; b < blocks; ++b) {
    const int v = c[int64_t(b) * kSortBins];
    c[int64_t(b) * kSortBins] = sum;
    sum += v;
  }
  c[int64_t(blocks) * kSortBins] = sum;
}

template <class Job>
__global__ __launch_bounds__(kSortThreads) void place_kernel(Job job, int n, const int32_t* counts, int blocks) {
  __shared__ int32_t count[kSortWaves][kSortBins];
  __shared__ int32_t first[kSortBins];
  __shared__ int32_t wave_sum[kSortBins / 64];
  const int tid = threadIdx.x, lane = tid & 63, wid = tid >> 6;
  for (int d = lane; d < job.bins; d += 64) count[wid][d] = 0;
  const int64_t at = int64_t(blockIdx.x) * kSortChunk + wid * 64 * kSortItems + lane;
  int key[kSortItems], digit[kSortItems], rank[kSortItems];
#pragma unroll
  for (int k = 0; k < kSortItems; ++k) {
    key[k] = 0;
    digit[k] = at + 64 * k < n ? job.digit(int(at + 64 * k), key[k]) : -1;
  }
  __syncthreads();
  const uint64_t below = (uint64_t(1) << lane) - 1;
#pragma unroll
  for (int k = 0; k < kSortItems; ++k) {
    const bool live = digit[k] >= 0;
    uint64_t same = __ballot(live);
    for (int b = 0; b < job.bits; ++b) {
      const uint64_t set = __ballot((digit[k] >> b) & 1);
      same &= (digit[k] >> b) & 1 ? set : ~set;
    }
    // (the wave's own counts: its LDS accesses stay in order)
    volatile int32_t* c = count[wid];
    if (live) {
      const int before = __popcll(same & below), had = c[digit[k]];
      rank[k] = had + before;
      if (before == 0) c[digit[k]] = had + __popcll(same);
    }
  }
  __syncthreads();
  // digit tid: where the block's items of it begin, for each wave
  int total = 0, mine = 0, here = 0;
  if (tid < job.bins) {
#pragma unroll
    for (int w = 0; w < kSortWaves; ++w) {
      const int v = count[w][tid];
      count[w][tid] = here;
      here += v;
    }
    total = here;
    if (blocks > kSortNear) {
      mine = counts[int64_t(blockIdx.x) * kSortBins + tid];
      total = counts[int64_t(blocks) * kSortBins + tid];
    } else if (blocks > 1) {
      total = 0;
      for (int b = 0; b < blocks; b += 8) {
        int v[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = counts[int64_t(min(b + k, blocks - 1)) * kSortBins + tid];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          if (b + k >= blocks) v[k] = 0;
          mine += b + k < int(blockIdx.x) ? v[k] : 0;
          total += v[k];
        }
      }
    }
  }
  int sum = total;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int v = __shfl_up(sum, d);
    if (lane >= d) sum += v;
  }
  if (lane == 63 && wid < kSortBins / 64) wave_sum[wid] = sum;
  __syncthreads();
  if (tid < job.bins) {
    int start = sum - total;
    for (int w = 0; w < wid; ++w) start += wave_sum[w];
    first[tid] = start + mine;
    if (blockIdx.x == 0) job.start(tid, start);
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < kSortItems; ++k)
    if (digit[k] >= 0)
      job.put(int(at + 64 * k), key[k], digit[k], first[digit[k]] + count[wid][digit[k]] + rank[k]);
}

template <class Job>
hipError_t launch_sort(const Job& job, int64_t n, int32_t* counts, hipStream_t st) {
  const int blocks = sort_blocks(n) > 1 ? sort_blocks(n) : 1;
  const dim3 g{unsigned(blocks)}, b{kSortThreads};
  if (blocks > 1) hipLaunchKernelGGL((count_kernel<Job>), g, b, 0, st, job, int(n), counts);
  if (blocks > kSortNear)
    hipLaunchKernelGGL(prefix_kernel, dim3{unsigned(job.bins + 63) / 64}, dim3{64}, 0, st, counts, blocks, job.bins);
  hipLaunchKernelGGL((place_kernel<Job>), g, b, 0, st, job, int(n), counts, blocks);
  return hipGetLastError();
}

}  // namespace
}  // namespace layers
}  // namespace muon

#endif  // MUON_LAYERS_SORT_H
