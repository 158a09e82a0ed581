// combine_backward.hip -- gfx950 kernel of the combine's gradient.
//
//   drecv[slot[t, j]] = bf16( gate[t, j] dout[t] ),   dgate[t, j] = sum_h dout[t, h] recv[slot[t, j], h]
//
// A wave (four, of few choices of long rows) takes one choice of one token: it reads dout's row and recv's, and writes
// drecv's, 16 bytes a lane.  The choices of a token are next to each other, in one workgroup or on one XCD, so that dout's
// row comes from memory once.  Memory bounds it: 8192 tokens, 6 choices of 2048 features, 437 MB in 89 us (4.9 TB/s).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "launch.hpp"
#include "ops.hpp"
#include "plan_types.hpp"
#include "vec_device.hpp"

namespace moe {

namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;

// kParts waves of a workgroup take one choice, 512 features in turn.
template <int kParts>
__global__ __launch_bounds__(kThreads) void combine_backward_kernel(CombineBackwardArgs a, uint32_t per_xcd) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  constexpr int kChoices = kWaves / kParts, kStep = kParts * 512;
  const int part = wave % kParts;
  // Workgroups b, b + 8, ... share an XCD: each XCD takes a run of choices.
  const int64_t choice = (int64_t)((blockIdx.x % kXcds) * per_xcd + blockIdx.x / kXcds) * kChoices + wave / kParts;
  if (blockIdx.x / kXcds >= per_xcd || choice >= a.tokens * a.k) return;
  const int64_t t = choice / a.k;
  const int j = (int)(choice % a.k), H = a.H;
  const int32_t slot = a.slot[choice];
  if (slot < 0 || slot >= a.recv_rows) {
    if (a.dgate && lane == 0 && part == 0) a.dgate[choice] = 0.0f;
    return;
  }
  // A row that a token names more than once takes all of its gates, through the first of them, which does the others' work:
  // their dgate is the same sum, and drecv may be recv, whose row nobody may read when the first has begun to write it.
  float gate = a.gate[choice];
  const bool write = a.drecv != nullptr;
  uint64_t same = 1ull << j;
  if (a.k > 1 && write) {
    same = __ballot(lane < a.k && a.slot[t * a.k + min(lane, a.k - 1)] == slot);
    if (same & ((1ull << j) - 1)) return;
    for (uint64_t more = same & ~(1ull << j); more; more &= more - 1) gate += a.gate[t * a.k + __builtin_ctzll(more)];
  }
  const uint16_t* dout = a.dout + t * H;
  const uint16_t* recv = a.recv + (int64_t)slot * H;
  uint16_t* drecv = a.drecv + (int64_t)slot * H;
  float sum = 0.0f;
  auto piece = [&](const u32x4& dv, const u32x4& rv, int h) {
    float d[8], r[8];
    unpack8(dv, d);
    unpack8(rv, r);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      sum = fmaf(d[i], r[i], sum);
      d[i] *= gate;
    }
    if (write) *(u32x4*)(drecv + h) = pack8(d);
  };
  constexpr int kAhead = 4;  // pieces in flight
  int h = (part * 64 + lane) * 8;
  for (; h + (kAhead - 1) * kStep < H; h += kAhead * kStep) {
    u32x4 d[kAhead], r[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) d[u] = *(const u32x4*)(dout + h + u * kStep), r[u] = *(const u32x4*)(recv + h + u * kStep);
#pragma unroll
    for (int u = 0; u < kAhead; ++u) piece(d[u], r[u], h + u * kStep);
  }
  for (; h < H; h += kStep) piece(*(const u32x4*)(dout + h), *(const u32x4*)(recv + h), h);
  if (a.dgate) {
    sum = wave_reduce(sum, [](float x, float y) { return x + y; });
    if constexpr (kParts > 1) {  // the whole workgroup has one choice
      static_assert(kParts == kWaves);
      __shared__ float sums[kWaves];
      if (lane == 0) sums[wave] = sum;
      __syncthreads();
      sum = sums[0];
#pragma unroll
      for (int w = 1; w < kWaves; ++w) sum += sums[w];
    }
    if (part == 0 && (same >> lane & 1)) a.dgate[t * a.k + lane] = sum;
  }
}

}  // namespace

// With few choices a wave's own turns along a long row are what the call waits for: 512 choices of 7168 features 6.7 us with a
// wave each, 5.4 with four; 64 of 16384 7.4 and 4.1.  At 4096 features that is 5 % less, at 2048 2 % more; from 2048 choices
// on the waves are enough, and four a choice take 7 to 17 % more.
int combine_backward_parts(int64_t choices, int32_t H) { return choices <= 1024 && H >= 4096 ? kWaves : 1; }

hipError_t launch_combine_backward_parts(int parts, const CombineBackwardArgs& a, hipStream_t s) {
  const int choices = kWaves / parts;
  const int64_t blocks = (a.tokens * a.k + choices - 1) / choices, per_xcd = (blocks + kXcds - 1) / kXcds;
  if (!launch_fits(per_xcd * kXcds, kThreads)) return hipErrorInvalidConfiguration;
  return launch(parts > 1 ? combine_backward_kernel<kWaves> : combine_backward_kernel<1>, dim3((uint32_t)(per_xcd * kXcds)), dim3(kThreads), 0,
                s, a, (uint32_t)per_xcd);
}

hipError_t launch_combine_backward(const CombineBackwardArgs& a, hipStream_t s) {
  return launch_combine_backward_parts(combine_backward_parts(a.tokens * a.k, a.H), a, s);
}

}  // namespace moe
