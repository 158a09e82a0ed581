// clip.hip -- gfx950 kernels of the norm of many tensors and of their scaling to at most a given norm.
//
//   total = sum over all tensors of v^2;   v *= max_norm / sqrt(total)  where that is below 1
//
// Squares are taken and added in 64 bits: no gradient is too large or too small for its square, and the order of the
// sum does not show in the 32-bit norm.  Memory bounds both passes: 1.1e9 elements of both types (3.3 GB) are read in 570 us
// (5.8 TB/s), and read and written in 1290 (5.1 TB/s).  Chunks of a 2048th of the whole, as many as there are workgroups,
// took 940 and 1670: the last ones of a launch leave compute units idle, and a thread had one piece in flight.  Now it has
// four where a chunk has as many left: of fp32 always, of bf16 in chunks of 8192 elements or more (a list below 2^28 elements
// has chunks of 4096, two pieces one after another).  The tensors' addresses travel in the kernel's arguments, so nothing is
// copied before a launch and a captured launch keeps them.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "launch.hpp"
#include "ops.hpp"
#include "vec_device.hpp"

namespace moe {

namespace {

constexpr int kThreads = 256;
typedef float f32x4 __attribute__((ext_vector_type(4)));

// A chunk's tensor: first[] of up to 128 tensors, two a lane.
struct Place {
  int tensor;
  int64_t from, n;  // elements
};
template <int kMost>
__device__ __forceinline__ Place place(const TensorTable<kMost>& t, uint32_t chunk, uint32_t first0, uint32_t first1) {
  const int i = __popcll(__ballot(first0 <= chunk)) + __popcll(__ballot(first1 <= chunk)) - 1;
  Place p;
  p.tensor = i;
  p.from = (int64_t)(chunk - t.first[i]) * t.chunk;
  p.n = min((int64_t)t.chunk, t.count[i] - p.from);
  return p;
}
template <int kMost>
__device__ __forceinline__ uint32_t first_of(const TensorTable<kMost>& t, int i) {
  return i < t.n ? t.first[i] : UINT32_MAX;
}

__device__ __forceinline__ float f32_of(uint16_t b) { return __uint_as_float((uint32_t)b << 16); }

// The workgroup's sum, in thread 0 of it.
template <int kWaves>
__device__ __forceinline__ double block_sum(double v) {
  __shared__ double parts[kWaves];
  v = wave_reduce(v, [](double x, double y) { return x + y; });
  if ((threadIdx.x & 63) == 0) parts[threadIdx.x >> 6] = v;
  __syncthreads();
  double s = parts[0];
#pragma unroll
  for (int w = 1; w < kWaves; ++w) s += parts[w];
  return s;
}

// The 16-byte pieces of n elements at p: load(i) of those from element i, kAhead of them in flight, then use(i, piece).
// one(i) takes the elements before the first piece and after the last.
constexpr int kAhead = 4;
template <class T, class Use, class One>
__device__ __forceinline__ void pieces(const T* p, int64_t n, Use&& use, One&& one) {
  constexpr int kLane = 16 / sizeof(T), kStep = kThreads * kLane;
  const int head = (int)min(n, (int64_t)((16 - ((uintptr_t)p & 15)) & 15) / (int64_t)sizeof(T));
  const int64_t end = head + (n - head) / kLane * kLane;
  for (int64_t i = threadIdx.x; i < head; i += kThreads) one(i);
  int64_t i = head + (int)threadIdx.x * kLane;
  for (; i + (kAhead - 1) * kStep < end; i += kAhead * kStep) {
    u32x4 v[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) v[u] = *(const u32x4*)(p + i + u * kStep);
#pragma unroll
    for (int u = 0; u < kAhead; ++u) use(i + u * kStep, v[u]);
  }
  for (; i < end; i += kStep) use(i, *(const u32x4*)(p + i));
  for (int64_t k = end + threadIdx.x; k < n; k += kThreads) one(k);
}

template <int kMost>
__global__ __launch_bounds__(kThreads) void squares_kernel(TensorTable<kMost> t, double* parts) {
  const int lane = threadIdx.x & 63;
  const uint32_t first0 = first_of(t, lane), first1 = first_of(t, lane + 64);
  double s0 = 0, s1 = 0;
  for (uint32_t c = blockIdx.x; c < t.chunks; c += gridDim.x) {
    const Place p = place(t, c, first0, first1);
    const uint64_t at = t.in[p.tensor];
    auto add2 = [&](float a, float b) {
      s0 = fma((double)a, (double)a, s0);
      s1 = fma((double)b, (double)b, s1);
    };
    if (at >> 63) {
      const uint16_t* v = (const uint16_t*)(at << 1 >> 1) + p.from;
      pieces(v, p.n, [&](int64_t, const u32x4& piece) {
        float f[8];
        unpack8(piece, f);
#pragma unroll
        for (int q = 0; q < 8; q += 2) add2(f[q], f[q + 1]);
      }, [&](int64_t i) { add2(f32_of(v[i]), 0.0f); });
    } else {
      const float* v = (const float*)at + p.from;
      pieces(v, p.n, [&](int64_t, const u32x4& piece) {
        const f32x4 f = __builtin_bit_cast(f32x4, piece);
        add2(f[0], f[1]);
        add2(f[2], f[3]);
      }, [&](int64_t i) { add2(v[i], 0.0f); });
    }
  }
  const double s = block_sum<kThreads / 64>(s0 + s1);
  if (threadIdx.x == 0) parts[blockIdx.x] = s;
}

__global__ __launch_bounds__(1024) void squares_sum_kernel(const double* parts, int n, double* total) {
  double s = 0;
  for (int i = threadIdx.x; i < n; i += 1024) s += parts[i];
  s = block_sum<16>(s);
  if (threadIdx.x == 0) *total = s;
}

// Chunks from the last to the first: what the sum of squares has read last is nearest.
template <int kMost>
__global__ __launch_bounds__(kThreads) void clip_kernel(TensorTable<kMost> t, const double* total, float max_norm, float* norm) {
  const double root = sqrt(*total);
  if (norm && blockIdx.x == 0 && threadIdx.x == 0) *norm = (float)root;
  // A norm that is not finite, or not as the caller sees it in 32 bits, leaves the gradients as they are.
  const double ratio = root > (double)max_norm && (float)root < __builtin_huge_valf() ? (double)max_norm / root : 1.0;
  // In 32 bits a ratio below 2^-126 would lose bits of its own (it may be as small as 2^-277).  It goes in two steps then, a
  // power of two that leaves 2^-100 or so of it: exact for every value that the ratio does not take below 2^-150, half of
  // the smallest one, as those are 2^-74 or more after it.
  const int shift = ratio > 0 && ratio < 0x1p-126 ? ilogb(ratio) + 100 : 0;
  const float scale = (float)ldexp(ratio, -shift);
  auto scaled = [&](float f) { return ldexpf(f, shift) * scale; };
  const int lane = threadIdx.x & 63;
  const uint32_t first0 = first_of(t, lane), first1 = first_of(t, lane + 64);
  for (uint32_t c = blockIdx.x; c < t.chunks; c += gridDim.x) {
    const Place p = place(t, t.chunks - 1 - c, first0, first1);
    const uint64_t at = t.in[p.tensor];
    const bool bf16 = at >> 63;
    const uint64_t in = at << 1 >> 1, to = t.out[p.tensor];
    if (in == to && scale == 1.0f) continue;
    const bool alike = ((in ^ to) & 15) == 0;  // pieces of 16 bytes in both
    if (bf16) {
      const uint16_t* v = (const uint16_t*)in + p.from;
      uint16_t* o = (uint16_t*)to + p.from;
      auto one = [&](int64_t i) { o[i] = (uint16_t)bf16x2_of(scaled(f32_of(v[i])), 0.0f); };
      if (alike)
        pieces(v, p.n, [&](int64_t i, const u32x4& piece) {
          float f[8];
          unpack8(piece, f);
#pragma unroll
          for (int q = 0; q < 8; ++q) f[q] = scaled(f[q]);
          *(u32x4*)(o + i) = pack8(f);
        }, one);
      else
        for (int64_t i = threadIdx.x; i < p.n; i += kThreads) one(i);
    } else {
      const float* v = (const float*)in + p.from;
      float* o = (float*)to + p.from;
      auto one = [&](int64_t i) { o[i] = scaled(v[i]); };
      if (alike)
        pieces(v, p.n, [&](int64_t i, const u32x4& piece) {
          f32x4 f = __builtin_bit_cast(f32x4, piece);
#pragma unroll
          for (int q = 0; q < 4; ++q) f[q] = scaled(f[q]);
          *(f32x4*)(o + i) = f;
        }, one);
      else
        for (int64_t i = threadIdx.x; i < p.n; i += kThreads) one(i);
    }
  }
}

}  // namespace

template <int kMost>
hipError_t launch_squares(const TensorTable<kMost>& t, double* parts, int blocks, hipStream_t s) {
  return launch(squares_kernel<kMost>, dim3((uint32_t)blocks), dim3(kThreads), 0, s, t, parts);
}
hipError_t launch_squares_sum(const double* parts, int n, double* total, hipStream_t s) {
  return launch(squares_sum_kernel, dim3(1), dim3(1024), 0, s, parts, n, total);
}
template <int kMost>
hipError_t launch_clip(const TensorTable<kMost>& t, const double* total, float max_norm, float* norm, int blocks, hipStream_t s) {
  return launch(clip_kernel<kMost>, dim3((uint32_t)blocks), dim3(kThreads), 0, s, t, total, max_norm, norm);
}
template hipError_t launch_squares(const TensorTable<kShortTable>&, double*, int, hipStream_t);
template hipError_t launch_squares(const TensorTable<kTableTensors>&, double*, int, hipStream_t);
template hipError_t launch_clip(const TensorTable<kShortTable>&, const double*, float, float*, int, hipStream_t);
template hipError_t launch_clip(const TensorTable<kTableTensors>&, const double*, float, float*, int, hipStream_t);

}  // namespace moe
