// norm.hip -- gfx950 kernels of the root-mean-square norm with the residual's addition and an output in
// 8 bits, of its gradients, and of rows in 8 bits.
//
//   h = bf16(x + residual),  r = 1 / sqrt(mean(h^2) + eps),  y = h r w
//   8 bits: scale = max|y| / 127, q = rne(y 127 / max|y|)
//   gradients: g = dy w,  dx = r (g - h r^2 mean(g h)) + dsum,  dw = sum_rows dy h r
//
// Each row is read once, held in registers, and each output is written once; memory bounds them all.
// Sums are fp32; h is rounded to bf16 before it is normed, so that the gradients, which start from the
// stored h, are those of the very function that was computed.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "ops.hpp"
#include "vec_device.hpp"

namespace moe {

constexpr float kTinyRow = 0x1p-100f;  // rows of less than this are zeros in 8 bits: 127 / max would overflow
constexpr int kThreads = 256;

template <class T, class F>
__device__ __forceinline__ T block_reduce(T v, F&& f) {
  __shared__ T part[kThreads / 64];
  v = wave_reduce(v, f);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
  __syncthreads();
  v = part[0];
  for (int i = 1; i < kThreads / 64; ++i) v = f(v, part[i]);
  __syncthreads();
  return v;
}

__global__ __launch_bounds__(kThreads) void norm_kernel(NormArgs a) {
  const int nvec = a.H / 8;
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const u32x4* x = (const u32x4*)(a.x + row * a.H);
    const u32x4* res = a.residual ? (const u32x4*)(a.residual + row * a.H) : nullptr;
    auto load_h = [&](int v, float (&h)[8]) {
      unpack8(x[v], h);
      if (res) {
        float t[8];
        unpack8(res[v], t);
        for (int e = 0; e < 8; ++e) h[e] += t[e];
        unpack8(pack8(h), h);
      }
    };
    float ss = 0.0f;
    for (int v = threadIdx.x; v < nvec; v += kThreads) {
      float h[8];
      load_h(v, h);
      for (int e = 0; e < 8; ++e) ss += h[e] * h[e];
    }
    ss = block_reduce(ss, [](float p, float q) { return p + q; });
    const float r = a.weight ? 1.0f / sqrtf(ss / (float)a.H + a.eps) : 1.0f;
    auto load_y = [&](int v, float (&y)[8]) {
      load_h(v, y);
      if (!a.weight) return;
      float w[8];
      unpack8(((const u32x4*)a.weight)[v], w);
      for (int e = 0; e < 8; ++e) y[e] = y[e] * r * w[e];
    };
    if (a.out_q) {
      uint32_t top = 0;
      for (int v = threadIdx.x; v < nvec; v += kThreads) {
        float y[8];
        load_y(v, y);
        for (int e = 0; e < 8; ++e) top = max(top, magnitude(y[e]));
      }
      top = block_reduce(top, [](uint32_t p, uint32_t q) { return max(p, q); });
      const float amax = __uint_as_float(top);
      const bool finite = top < 0x7F800000u;
      const float inv = finite && amax >= kTinyRow ? 127.0f / amax : 0.0f;
      if (threadIdx.x == 0) a.scale[row] = !finite ? __uint_as_float(0x7FC00000u) : amax >= kTinyRow ? amax / 127.0f : 0.0f;
      for (int v = threadIdx.x; v < nvec; v += kThreads) {
        float y[8];
        load_y(v, y);
        uint32_t q[2] = {0, 0};
        if (inv > 0.0f)
          for (int e = 0; e < 8; ++e) q[e / 4] |= ((uint32_t)(int)rintf(y[e] * inv) & 0xFFu) << (8 * (e % 4));
        ((u32x2*)(a.out_q + row * a.H))[v] = u32x2{q[0], q[1]};
      }
    }
    if (a.rstd && threadIdx.x == 0) a.rstd[row] = r;
    if (a.sum_out || a.out) {
      for (int v = threadIdx.x; v < nvec; v += kThreads) {
        float h[8], y[8];
        load_h(v, h);
        load_y(v, y);
        if (a.sum_out) ((u32x4*)(a.sum_out + row * a.H))[v] = pack8(h);
        if (a.out) ((u32x4*)(a.out + row * a.H))[v] = pack8(y);
      }
    }
  }
}

hipError_t launch_norm(const NormArgs& a, hipStream_t s) {
  const uint32_t grid = (uint32_t)std::min<int64_t>(a.rows, 1 << 20);
  hipLaunchKernelGGL(norm_kernel, dim3(grid), dim3(kThreads), 0, s, a);
  return hipGetLastError();
}

// Part p holds the sums of rows p, p + parts, ...
int64_t norm_backward_parts(int64_t rows, int32_t) { return std::min<int64_t>(rows, 256); }

__global__ __launch_bounds__(kThreads) void norm_backward_kernel(NormBackwardArgs a) {
  const int nvec = a.H / 8;
  const u32x4* wv = (const u32x4*)a.weight;
  float* mine = a.parts + (int64_t)blockIdx.x * a.H;
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const u32x4* dyv = (const u32x4*)(a.dy + row * a.H);
    const u32x4* hv = (const u32x4*)(a.h + row * a.H);
    const u32x4* dsv = a.dsum ? (const u32x4*)(a.dsum + row * a.H) : nullptr;
    float dot = 0.0f;
    for (int v = threadIdx.x; v < nvec; v += kThreads) {
      float dy[8], h[8], w[8];
      unpack8(dyv[v], dy);
      unpack8(hv[v], h);
      unpack8(wv[v], w);
      for (int e = 0; e < 8; ++e) dot += dy[e] * w[e] * h[e];
    }
    dot = block_reduce(dot, [](float p, float q) { return p + q; });
    const float r = a.rstd[row];
    const float c = dot / (float)a.H * r * r;
    for (int v = threadIdx.x; v < nvec; v += kThreads) {
      float dy[8], h[8], w[8], ds[8] = {}, dx[8];
      unpack8(dyv[v], dy);
      unpack8(hv[v], h);
      unpack8(wv[v], w);
      if (dsv) unpack8(dsv[v], ds);
      for (int e = 0; e < 8; ++e) {
        dx[e] = r * (dy[e] * w[e] - h[e] * c) + ds[e];
        const float d = dy[e] * h[e] * r;
        mine[v * 8 + e] = row == blockIdx.x ? d : mine[v * 8 + e] + d;
      }
      ((u32x4*)(a.dx + row * a.H))[v] = pack8(dx);
    }
  }
}

__global__ __launch_bounds__(kThreads) void norm_weight_kernel(const float* parts, int64_t n, int32_t H, float* dweight) {
  const int c = blockIdx.x * kThreads + threadIdx.x;
  if (c >= H) return;
  float s = 0.0f;
  for (int64_t p = 0; p < n; ++p) s += parts[p * H + c];
  dweight[c] = s;
}

hipError_t launch_norm_backward(const NormBackwardArgs& a, hipStream_t s) {
  const int64_t parts = norm_backward_parts(a.rows, a.H);
  if (parts > 0) {
    hipLaunchKernelGGL(norm_backward_kernel, dim3((uint32_t)parts), dim3(kThreads), 0, s, a);
    if (hipError_t e = hipGetLastError()) return e;
  }
  hipLaunchKernelGGL(norm_weight_kernel, dim3((a.H + kThreads - 1) / kThreads), dim3(kThreads), 0, s, a.parts, parts, a.H,
                     a.dweight);
  return hipGetLastError();
}

__global__ __launch_bounds__(kThreads) void restore_kernel(RestoreArgs a) {
  const int nvec = a.H / 8;
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const float s = a.scale[row];
    for (int v = threadIdx.x; v < nvec; v += kThreads) {
      const u32x2 q = ((const u32x2*)(a.q + row * a.H))[v];
      float f[8];
      for (int e = 0; e < 8; ++e) f[e] = (float)(int8_t)(q[e / 4] >> (8 * (e % 4))) * s;
      ((u32x4*)(a.out + row * a.H))[v] = pack8(f);
    }
  }
}

hipError_t launch_restore(const RestoreArgs& a, hipStream_t s) {
  const uint32_t grid = (uint32_t)std::min<int64_t>(a.rows, 1 << 20);
  hipLaunchKernelGGL(restore_kernel, dim3(grid), dim3(kThreads), 0, s, a);
  return hipGetLastError();
}

}  // namespace moe
