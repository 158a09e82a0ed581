// group.hip -- gfx950 kernels of the routed rows' order by expert: a stable counting sort of the choices.
//
// Workgroup b takes a run of consecutive entries, each of its waves a run of those, 64 at a time.  Entries of one
// expert among a wave's 64 find each other by ballots over the bits of the expert's number, which ranks them
// without an atomic, and the wave's count for that expert goes up by their number: the order does not depend on
// which wave runs first.  Up to kOneEntries one workgroup does it all in one launch; more are counted by a
// first launch, from whose counts each workgroup of the second finds where its entries of each expert begin.
//
// Nothing here is much data (12 bytes an entry): what counts is the chain of dependent steps.  384 entries of 256
// experts take 3.6 us in one launch, 262144 take 3.0 + 9.6 (a third launch that summed the counts by itself took 81).
// Of the 9.6 some 4.4 are vector instructions, 660 for each of four waves a SIMD on half of the compute units: the
// reading of every workgroup's counts, the counting of the own entries once more, the ranks.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "launch.hpp"
#include "ops.hpp"
#include "vec_device.hpp"

namespace moe {

constexpr int kThreads = 1024;  // a thread for each expert there can be
constexpr int kWaves = kThreads / 64;
constexpr int64_t kOneEntries = 4096;
constexpr int64_t kBlockEntries = 2048;
constexpr int kAhead = 4;  // entries of a lane that are read together
constexpr int64_t kMostBlocks = 128;  // each one reads the counts of all of them

// Entries of a workgroup: a multiple of kThreads.
inline int64_t block_entries(int64_t n) {
  const int64_t even = (n + kMostBlocks - 1) / kMostBlocks;
  return std::max(kBlockEntries, (even + kThreads - 1) / kThreads * kThreads);
}

int64_t group_blocks(int64_t n, int32_t) { return n <= kOneEntries ? 0 : (n + block_entries(n) - 1) / block_entries(n); }

// Lanes of the wave that hold the same id as this one.
__device__ __forceinline__ uint64_t same_id(uint32_t id, int bits) {
  uint64_t m = ~0ull;
  for (int b = 0; b < bits; ++b) {
    const bool on = (id >> b) & 1;
    const uint64_t v = __ballot(on);
    m &= on ? v : ~v;
  }
  return m;
}

__device__ __forceinline__ int rank_below(uint64_t m) {
  return __builtin_amdgcn_mbcnt_hi((uint32_t)(m >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)m, 0));
}

// The expert of entry i; `experts` for an entry that has none.
__device__ __forceinline__ uint32_t id_of(const GroupArgs& a, int64_t i) {
  if (i >= a.n) return a.experts;
  const uint32_t id = (uint32_t)a.ids[i];
  return id < (uint32_t)a.experts ? id : a.experts;
}

// Inclusive sum over the workgroup's threads.
__device__ __forceinline__ int scan(int v, int* part) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int o = __shfl_up(v, d);
    if (lane >= d) v += o;
  }
  if (lane == 63) part[wave] = v;
  __syncthreads();
  for (int w = 0; w < wave; ++w) v += part[w];
  return v;
}

__global__ __launch_bounds__(kThreads) void group_count_kernel(GroupArgs a, int64_t entries) {
  extern __shared__ int cnt[];  // [kWaves][experts]: with few experts all waves would meet at their counts
  const int E = a.experts, tid = threadIdx.x, wave = tid >> 6;
  for (int i = tid; i < kWaves * E; i += kThreads) cnt[i] = 0;
  __syncthreads();
  const int64_t first = blockIdx.x * entries;
#pragma unroll 2
  for (int64_t i = first + tid; i < first + entries; i += kThreads) {
    const uint32_t id = id_of(a, i);
    if (id < (uint32_t)E) atomicAdd(&cnt[wave * E + id], 1);
  }
  __syncthreads();
  for (int e = tid; e < E; e += kThreads) {
    int sum = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) sum += cnt[w * E + e];
    a.counts[(int64_t)blockIdx.x * E + e] = (uint32_t)sum;
  }
}

// kOne: one workgroup, no counts.
template <bool kOne>
__global__ __launch_bounds__(kThreads) void group_place_kernel(GroupArgs a, int64_t entries, int bits) {
  extern __shared__ int cnt[];  // [kWaves][experts], at least 2 * kThreads
  __shared__ int part[kWaves], total;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, E = a.experts;
  const int64_t first = blockIdx.x * entries + wave * (entries / kWaves), end = first + entries / kWaves;
  int before = 0, all = 0;  // thread e: entries of expert e in earlier workgroups, and in all
  if constexpr (!kOne) {
    // Up to 16 threads read each expert's counts, every so-many-th workgroup's, so that the reads are a round trip
    // or two; the sums meet in LDS.
    const int blocks = gridDim.x, me = blockIdx.x, sharers = min(kThreads / E, 16), share = tid / E, e = tid % E;
    if (share < sharers) {
#pragma unroll 16
      for (int b = share; b < blocks; b += sharers) {
        const int v = (int)a.counts[(int64_t)b * E + e];
        all += v;
        before += b < me ? v : 0;
      }
      cnt[tid] = all;
      cnt[kThreads + tid] = before;
    }
    __syncthreads();
    all = before = 0;
    if (tid < E)
      for (int i = tid; i < sharers * E; i += E) {
        all += cnt[i];
        before += cnt[kThreads + i];
      }
    __syncthreads();
  }
  for (int i = tid; i < kWaves * E; i += kThreads) cnt[i] = 0;
  __syncthreads();
  for (int64_t i0 = first + lane; i0 - lane < end; i0 += 64 * kAhead) {
    uint32_t ids[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) ids[u] = i0 + 64 * u < end ? id_of(a, i0 + 64 * u) : E;
#pragma unroll
    for (int u = 0; u < kAhead; ++u)
      if (ids[u] < (uint32_t)E) atomicAdd(&cnt[wave * E + ids[u]], 1);
  }
  __syncthreads();
  if (kOne && tid < E)
    for (int w = 0; w < kWaves; ++w) all += cnt[w * E + tid];
  const int upto = scan(all, part);
  if (tid < E) {
    int at = upto - all + before;  // the first row of each wave's entries of this expert
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const int v = cnt[w * E + tid];
      cnt[w * E + tid] = at;
      at += v;
    }
    if (blockIdx.x == 0) {
      a.offsets[tid + 1] = upto;
      if (tid == 0) a.offsets[0] = 0;
    }
  }
  if (tid == E - 1) total = upto;
  __syncthreads();
  for (int64_t i0 = first + lane; i0 - lane < end && i0 - lane < a.n; i0 += 64 * kAhead) {
    uint32_t ids[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) ids[u] = i0 + 64 * u < end ? id_of(a, i0 + 64 * u) : E;
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int64_t i = i0 + 64 * u;
      if (i - lane >= end) break;
      const uint32_t id = ids[u];
      const uint64_t m = same_id(id, bits);
      const int below = rank_below(m);
      int pos = -1;
      if (id < (uint32_t)E) {
        pos = cnt[wave * E + id] + below;
        // Read by all of them, then raised by the first: a wave's LDS operations happen in their order.
        __builtin_amdgcn_wave_barrier();
        if (below == 0) cnt[wave * E + id] = pos + (int)__popcll(m);
        __builtin_amdgcn_wave_barrier();
        a.row_token[pos] = (int)((uint32_t)i / (uint32_t)a.k);
      }
      if (i < a.n) {
        a.slot[i] = pos;
        if (i >= total) a.row_token[i] = -1;
      }
    }
  }
}

hipError_t launch_group(const GroupArgs& a, hipStream_t s) {
  int bits = 1;  // of the numbers 0 .. experts
  while ((a.experts >> bits) != 0) ++bits;
  const int blocks = (int)group_blocks(a.n, a.experts);
  const uint32_t lds = (uint32_t)(std::max(kWaves * a.experts, 2 * kThreads) * sizeof(int));
  if (blocks == 0) {
    const int64_t entries = ((int64_t)a.n + kThreads - 1) / kThreads * kThreads;
    return launch(group_place_kernel<true>, dim3(1), dim3(kThreads), lds, s, a, entries, bits);
  }
  const int64_t entries = block_entries(a.n);
  if (hipError_t e = launch(group_count_kernel, dim3(blocks), dim3(kThreads), lds, s, a, entries)) return e;
  return launch(group_place_kernel<false>, dim3(blocks), dim3(kThreads), lds, s, a, entries, bits);
}

}  // namespace moe
