// group.hip -- gfx950 kernels of the routed rows' order by expert: a stable counting sort of the choices.
//
// Entries are taken in chunks of 64, one wave at a time: entries of one expert within a chunk find each other
// by ballots over the bits of the expert's number, which gives every entry its rank without an atomic, so the
// order does not depend on which wave runs first.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "ops.hpp"
#include "vec_device.hpp"

namespace moe {

constexpr int kChunk = 64;
constexpr int kBlockThreads = 256;
constexpr int kBlockEntries = 1024;
constexpr int kBlockChunks = kBlockEntries / kChunk;
constexpr int kOneThreads = 1024;       // the single workgroup: a thread per expert
constexpr int kOneBytes = 48 * 1024;    // its counts: chunks x experts x 2 bytes

inline bool one_workgroup(int64_t n, int32_t experts) {
  return n <= 8192 && ((n + kChunk - 1) / kChunk) * experts * 2 <= kOneBytes;
}

int64_t group_blocks(int64_t n, int32_t experts) {
  return one_workgroup(n, experts) ? 0 : (n + kBlockEntries - 1) / kBlockEntries;
}

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
__device__ __forceinline__ uint32_t id_of(const GroupArgs& a, int i) {
  if (i >= a.n) return a.experts;
  const uint32_t id = (uint32_t)a.ids[i];
  return id < (uint32_t)a.experts ? id : a.experts;
}

// Inclusive sum over the workgroup's threads (up to 16 waves).
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

__global__ __launch_bounds__(kOneThreads) void group_one_kernel(GroupArgs a, int bits) {
  __shared__ uint16_t cnt[kOneBytes / 2];
  __shared__ int part[kOneThreads / 64], total;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, E = a.experts;
  const int chunks = (a.n + kChunk - 1) / kChunk;
  for (int i = tid; i < chunks * E; i += kOneThreads) cnt[i] = 0;
  __syncthreads();
  for (int c = wave; c < chunks; c += kOneThreads / 64) {
    const uint32_t id = id_of(a, c * kChunk + lane);
    const uint64_t m = same_id(id, bits);
    if (id < (uint32_t)E && rank_below(m) == 0) cnt[c * E + id] = (uint16_t)__popcll(m);
  }
  __syncthreads();
  int sum = 0;
  if (tid < E)
    for (int c = 0; c < chunks; ++c) sum += cnt[c * E + tid];
  const int end = scan(sum, part);
  if (tid < E) {
    a.offsets[tid + 1] = end;
    int at = end - sum;
    for (int c = 0; c < chunks; ++c) {
      const int v = cnt[c * E + tid];
      cnt[c * E + tid] = (uint16_t)at;
      at += v;
    }
  }
  if (tid == 0) a.offsets[0] = 0;
  if (tid == E - 1) total = end;
  __syncthreads();
  for (int c = wave; c < chunks; c += kOneThreads / 64) {
    const int i = c * kChunk + lane;
    const uint32_t id = id_of(a, i);
    const uint64_t m = same_id(id, bits);
    if (i >= a.n) continue;
    if (id < (uint32_t)E) {
      const int pos = cnt[c * E + id] + rank_below(m);
      a.slot[i] = pos;
      a.row_token[pos] = i / a.k;
    } else {
      a.slot[i] = -1;
    }
  }
  for (int i = total + tid; i < a.n; i += kOneThreads) a.row_token[i] = -1;
}

__global__ __launch_bounds__(kBlockThreads) void group_count_kernel(GroupArgs a) {
  __shared__ uint32_t cnt[1024];
  const int E = a.experts;
  for (int e = threadIdx.x; e < E; e += kBlockThreads) cnt[e] = 0;
  __syncthreads();
  for (int j = threadIdx.x; j < kBlockEntries; j += kBlockThreads) {
    const int64_t i = (int64_t)blockIdx.x * kBlockEntries + j;
    const uint32_t id = i < a.n ? id_of(a, (int)i) : E;
    if (id < (uint32_t)E) atomicAdd(&cnt[id], 1u);
  }
  __syncthreads();
  for (int e = threadIdx.x; e < E; e += kBlockThreads) a.counts[(int64_t)blockIdx.x * E + e] = cnt[e];
}

// counts[b][e] becomes the first row of block b's entries of expert e.
__global__ __launch_bounds__(kOneThreads) void group_scan_kernel(GroupArgs a, int blocks) {
  __shared__ int part[kOneThreads / 64];
  const int e = threadIdx.x, E = a.experts;
  int sum = 0;
  if (e < E)
    for (int b = 0; b < blocks; ++b) sum += a.counts[(int64_t)b * E + e];
  const int end = scan(sum, part);
  if (e == 0) a.offsets[0] = 0;
  if (e >= E) return;
  a.offsets[e + 1] = end;
  int at = end - sum;
  for (int b = 0; b < blocks; ++b) {
    const int v = a.counts[(int64_t)b * E + e];
    a.counts[(int64_t)b * E + e] = at;
    at += v;
  }
}

__global__ __launch_bounds__(kBlockThreads) void group_place_kernel(GroupArgs a, int bits) {
  __shared__ uint16_t cnt[kBlockChunks * 1024];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, E = a.experts;
  const int64_t first = (int64_t)blockIdx.x * kBlockEntries;
  for (int i = tid; i < kBlockChunks * E; i += kBlockThreads) cnt[i] = 0;
  __syncthreads();
  for (int c = wave; c < kBlockChunks; c += kBlockThreads / 64) {
    const int64_t i = first + c * kChunk + lane;
    const uint32_t id = i < a.n ? id_of(a, (int)i) : E;
    const uint64_t m = same_id(id, bits);
    if (id < (uint32_t)E && rank_below(m) == 0) cnt[c * E + id] = (uint16_t)__popcll(m);
  }
  __syncthreads();
  for (int e = tid; e < E; e += kBlockThreads) {
    int at = 0;
    for (int c = 0; c < kBlockChunks; ++c) {
      const int v = cnt[c * E + e];
      cnt[c * E + e] = (uint16_t)at;
      at += v;
    }
  }
  __syncthreads();
  const int total = a.offsets[E];
  for (int c = wave; c < kBlockChunks; c += kBlockThreads / 64) {
    const int64_t i = first + c * kChunk + lane;
    const uint32_t id = i < a.n ? id_of(a, (int)i) : E;
    const uint64_t m = same_id(id, bits);
    if (i >= a.n) continue;
    if (id < (uint32_t)E) {
      const int pos = (int)a.counts[(int64_t)blockIdx.x * E + id] + cnt[c * E + id] + rank_below(m);
      a.slot[i] = pos;
      a.row_token[pos] = (int)i / a.k;
    } else {
      a.slot[i] = -1;
    }
    if (i >= total) a.row_token[i] = -1;
  }
}

hipError_t launch_group(const GroupArgs& a, hipStream_t s) {
  int bits = 1;  // of the numbers 0 .. experts
  while ((a.experts >> bits) != 0) ++bits;
  const int blocks = (int)group_blocks(a.n, a.experts);
  if (blocks == 0) {
    hipLaunchKernelGGL(group_one_kernel, dim3(1), dim3(kOneThreads), 0, s, a, bits);
    return hipGetLastError();
  }
  hipLaunchKernelGGL(group_count_kernel, dim3(blocks), dim3(kBlockThreads), 0, s, a);
  hipLaunchKernelGGL(group_scan_kernel, dim3(1), dim3(kOneThreads), 0, s, a, blocks);
  hipLaunchKernelGGL(group_place_kernel, dim3(blocks), dim3(kBlockThreads), 0, s, a, bits);
  return hipGetLastError();
}

}  // namespace moe
