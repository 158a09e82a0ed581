// norm.hip -- gfx950 kernels of the root-mean-square norm with the residual's addition and an output in
// 8 bits, of its gradients, and of rows in 8 bits.
//
//   h = bf16(x + residual),  r = 1 / sqrt(mean(h^2) + eps),  y = h r w
//   8 bits: scale = max|y| / 127, q = rne(y 127 / max|y|)
//   gradients: g = dy w,  dx = r (g - h r^2 mean(g h)) + dsum,  dw = sum_rows dy h r
//
// Each row is read once, held in registers as its packed bf16, and each output is written once; memory bounds
// them all: 4096 rows of 7168 with the sum and 8 bits out 40 us (205 MB, 5.2 TB/s), 8192 rows of 14336 to 8 bits
// 55 us (352 MB, 6.4 TB/s), back to bf16 4096 of 7168 14 us (88 MB, 6.3 TB/s), the gradients of 8192 rows of 2048
// 24 + 5 us (135 MB).  Read three times over from memory, as a first version did, the first took 88 us.  A few rows
// are bound by their chain (loads, one or two reductions, stores): 16 of 4096 take 3.4 us.
// Sums are fp32; h is rounded to bf16 before it is normed, so that the gradients, which start from the stored h,
// are those of the very function that was computed.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <type_traits>

#include "launch.hpp"
#include "ops.hpp"
#include "vec_device.hpp"

namespace moe {

constexpr float kTinyRow = 0x1p-100f;  // rows of less than this are zeros in 8 bits: 127 / max would overflow

__device__ __forceinline__ float add(float a, float b) { return a + b; }
__device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t b) { return max(a, b); }

// f over the kLanes threads that hold a row, in all of them.  `part` is this reduction's own LDS.
template <int kLanes, class T, class F>
__device__ __forceinline__ T row_reduce(T v, T* part, F&& f) {
  v = wave_reduce(v, f);
  if constexpr (kLanes > 64) {
    const int wave = threadIdx.x >> 6;
    if ((threadIdx.x & 63) == 0) part[wave] = v;
    __syncthreads();
    const T* mine = part + (int)(threadIdx.x / kLanes) * (kLanes / 64);
    v = mine[0];
#pragma unroll
    for (int i = 1; i < kLanes / 64; ++i) v = f(v, mine[i]);
  }
  return v;
}

// How a row's values become int8: rne(y 127 / amax).  The quotient is a product with 1 / amax and a correction by
// its remainder, which gives the fp32 nearest to it: with a product alone, values that fall half way between two
// steps (bf16 rows have many) go up or down as 1 / amax happens to be rounded.
struct Quantiser {
  float times, top, inv;
  explicit __device__ __forceinline__ Quantiser(float amax) {
    const float down = amax > 0x1p100f ? 0x1p-64f : 1.0f;  // or 127 y might overflow
    times = 127.0f * down;
    top = amax * down;
    inv = 1.0f / top;
  }
  // The step in the lowest byte: adding 1.5 * 2^23 rounds to the nearest even whole number.
  __device__ __forceinline__ uint32_t step(float y) const {
    const float t = __fmul_rn(y, times), p = __fmul_rn(t, inv);
    return __float_as_uint(__fadd_rn(fmaf(fmaf(-p, top, t), inv, p), 12582912.0f));
  }
  __device__ __forceinline__ uint32_t four(float a, float b, float c, float d) const {
    return __builtin_amdgcn_perm(step(b), step(a), 0x0C0C0400u) | __builtin_amdgcn_perm(step(d), step(c), 0x04000C0Cu);
  }
};

constexpr int row_threads(int lanes) { return std::max(lanes, 256); }

// kLanes threads hold a row, kV vectors of 8 values each; kNorm: the norm, else rows are quantised as they are.
template <int kLanes, int kV, bool kNorm>
__global__ __launch_bounds__(row_threads(kLanes)) void norm_kernel(NormArgs a) {
  constexpr int kRows = row_threads(kLanes) / kLanes;
  __shared__ float part_sum[row_threads(kLanes) / 64];
  __shared__ uint32_t part_max[row_threads(kLanes) / 64];
  const int sub = __builtin_amdgcn_readfirstlane(threadIdx.x / kLanes), lane = threadIdx.x % kLanes;
  const int64_t row = (int64_t)blockIdx.x * kRows + sub;
  if (kLanes <= 64 && row >= a.rows) return;  // wider rows take a workgroup each: none is left over
  const int nvec = a.H / 8;
  const u32x4* x = (const u32x4*)(a.x + row * a.H);
  u32x4 h[kV], w[kV];
#pragma unroll
  for (int i = 0; i < kV; ++i) {
    const int v = lane + i * kLanes;
    h[i] = w[i] = u32x4{};
    if (v < nvec) {
      h[i] = x[v];
      if constexpr (kNorm) w[i] = ((const u32x4*)a.weight)[v];
    }
  }
  float r = 1.0f;
  if constexpr (kNorm) {
    if (a.residual) {
      const u32x4* res = (const u32x4*)(a.residual + row * a.H);
      u32x4 t[kV];
#pragma unroll
      for (int i = 0; i < kV; ++i) {
        const int v = lane + i * kLanes;
        t[i] = u32x4{};
        if (v < nvec) t[i] = res[v];
      }
#pragma unroll
      for (int i = 0; i < kV; ++i) {
        float p[8], q[8];
        unpack8(h[i], p);
        unpack8(t[i], q);
#pragma unroll
        for (int e = 0; e < 8; ++e) p[e] += q[e];
        h[i] = pack8(p);
      }
    }
    if (a.sum_out) {
#pragma unroll
      for (int i = 0; i < kV; ++i) {
        const int v = lane + i * kLanes;
        if (v < nvec) ((u32x4*)(a.sum_out + row * a.H))[v] = h[i];
      }
    }
    float ss = 0.0f;
#pragma unroll
    for (int i = 0; i < kV; ++i) {
      float f[8];
      unpack8(h[i], f);
#pragma unroll
      for (int e = 0; e < 8; ++e) ss += f[e] * f[e];
    }
    ss = row_reduce<kLanes>(ss, part_sum, add);
    r = 1.0f / sqrtf(ss / (float)a.H + a.eps);
    if (a.rstd && lane == 0) a.rstd[row] = r;
  }
  auto normed = [&](int i, float (&y)[8]) {
    unpack8(h[i], y);
    if constexpr (kNorm) {
      float f[8];
      unpack8(w[i], f);
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] = y[e] * r * f[e];
    }
  };
  if (kNorm && a.out) {
#pragma unroll
    for (int i = 0; i < kV; ++i) {
      const int v = lane + i * kLanes;
      float y[8];
      normed(i, y);
      if (v < nvec) ((u32x4*)(a.out + row * a.H))[v] = pack8(y);
    }
  }
  if (kNorm && !a.out_q) return;
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < kV; ++i) {
    float y[8];
    normed(i, y);
    if (lane + i * kLanes < nvec) {  // past the row's end h and w are 0, but r may be infinite
#pragma unroll
      for (int e = 0; e < 8; ++e) top = max(top, magnitude(y[e]));
    }
  }
  top = row_reduce<kLanes>(top, part_max, larger);
  const float amax = __uint_as_float(top);
  const bool finite = top < 0x7F800000u;
  const bool zero = !finite || amax < kTinyRow;
  const Quantiser to8(zero ? 1.0f : amax);
  if (lane == 0) a.scale[row] = !finite ? __uint_as_float(0x7FC00000u) : zero ? 0.0f : amax / 127.0f;
#pragma unroll
  for (int i = 0; i < kV; ++i) {
    const int v = lane + i * kLanes;
    float y[8];
    normed(i, y);
    u32x2 q = {to8.four(y[0], y[1], y[2], y[3]), to8.four(y[4], y[5], y[6], y[7])};
    if (zero) q = u32x2{};
    if (v < nvec) ((u32x2*)(a.out_q + row * a.H))[v] = q;
  }
}

// Calls f(threads per row, vectors per thread) as compile-time numbers.
template <class F>
void by_row(int64_t rows, int32_t H, F&& f) {
  const int nvec = H / 8;
  auto with = [&](auto lanes) {
    constexpr int L = decltype(lanes)::value;
    if (nvec <= L)
      f(lanes, std::integral_constant<int, 1>{});
    else if (nvec <= 2 * L)
      f(lanes, std::integral_constant<int, 2>{});
    else if (nvec <= 4 * L)
      f(lanes, std::integral_constant<int, 4>{});
    else
      f(lanes, std::integral_constant<int, 8>{});
  };
  // Many rows: a wave takes a whole one of up to 4096 values, which needs no barrier (8192 rows of 2048 23.6 us,
  // with 256 threads a row 29.9).  Few rows: threads enough for one or two vectors each, so that the row's loads
  // are one round trip (16 rows of 4096 3.4 us, with 4 to 8 vectors a thread in turn 7.0).
  const bool few = rows <= 512;
  if (nvec <= (few ? 128 : 512))
    with(std::integral_constant<int, 64>{});
  else if (nvec <= (few ? 512 : 2048))
    with(std::integral_constant<int, 256>{});
  else
    with(std::integral_constant<int, 1024>{});
}

hipError_t launch_norm(const NormArgs& a, hipStream_t s) {
  hipError_t e = hipErrorInvalidConfiguration;
  by_row(a.rows, a.H, [&](auto lanes, auto vecs) {
    constexpr int L = decltype(lanes)::value, V = decltype(vecs)::value, kRows = row_threads(L) / L;
    const int64_t blocks = (a.rows + kRows - 1) / kRows;
    if (!launch_fits(blocks, row_threads(L))) return;
    e = launch(a.weight ? norm_kernel<L, V, true> : norm_kernel<L, V, false>, dim3((uint32_t)blocks), dim3(row_threads(L)), 0, s, a);
  });
  return e;
}

// ------------------------------------------------------------------------------------ gradients

constexpr int kBackThreads = 512;
constexpr int kMaxParts = 256;
constexpr int kWideRow = 4 * 8 * kBackThreads;  // longer rows do not fit the registers

// Threads that hold a row, at most 4 vectors each: with their sums, the weights and a row's operands those take
// 190 to 220 registers, two waves per SIMD (8 vectors would spill).
constexpr int back_lanes(int32_t H) { return H <= 2048 ? 64 : H <= 4096 ? 128 : H <= 8192 ? 256 : kBackThreads; }
constexpr int back_rows(int32_t H) { return kBackThreads / back_lanes(H); }

// Up to two turns of rows go to one workgroup, whose sums are the gradient: a launch less (4 rows of 4072, forward
// and backward, 11.7 -> 9.8 us).
int64_t norm_backward_parts(int64_t rows, int32_t H) {
  return rows <= 2 * back_rows(H) ? 1 : std::min<int64_t>((rows + back_rows(H) - 1) / back_rows(H), kMaxParts);
}

// Workgroup p takes rows p * kRows + its row groups, then every parts * kRows rows on: the order of a column's
// sum depends on the sizes alone.  Each thread keeps its columns' sums of dy h r in registers over all its rows.
template <int kLanes, int kV>
__global__ __launch_bounds__(kBackThreads) void norm_backward_kernel(NormBackwardArgs a) {
  constexpr int kRows = kBackThreads / kLanes;
  __shared__ float part[2][kBackThreads / 64];
  __shared__ float sums[kRows > 1 ? kBackThreads * 8 : 1];
  const int sub = __builtin_amdgcn_readfirstlane(threadIdx.x / kLanes), lane = threadIdx.x % kLanes;
  const int nvec = a.H / 8;
  u32x4 w[kV];
  float dw[kV][8];
#pragma unroll
  for (int i = 0; i < kV; ++i) {
    const int v = lane + i * kLanes;
    w[i] = u32x4{};
    if (v < nvec) w[i] = ((const u32x4*)a.weight)[v];
#pragma unroll
    for (int e = 0; e < 8; ++e) dw[i][e] = 0.0f;
  }
  int turn = 0;
  for (int64_t row0 = (int64_t)blockIdx.x * kRows; row0 < a.rows; row0 += (int64_t)gridDim.x * kRows) {
    const int64_t row = row0 + sub;
    const bool have = row < a.rows;  // the others of the workgroup may have one: its barriers are everybody's
    u32x4 dy[kV], h[kV], ds[kV];
    const float r = have ? a.rstd[row] : 0.0f;
#pragma unroll
    for (int i = 0; i < kV; ++i) {
      const int v = lane + i * kLanes;
      dy[i] = h[i] = ds[i] = u32x4{};
      if (have && v < nvec) {
        dy[i] = ((const u32x4*)(a.dy + row * a.H))[v];
        h[i] = ((const u32x4*)(a.h + row * a.H))[v];
        if (a.dsum) ds[i] = ((const u32x4*)(a.dsum + row * a.H))[v];
      }
    }
    float dot = 0.0f;
#pragma unroll
    for (int i = 0; i < kV; ++i) {
      float fy[8], fh[8], fw[8];
      unpack8(dy[i], fy);
      unpack8(h[i], fh);
      unpack8(w[i], fw);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        dot += fy[e] * fw[e] * fh[e];
        dw[i][e] += fy[e] * (fh[e] * r);
      }
    }
    dot = row_reduce<kLanes>(dot, part[turn], add);
    turn ^= 1;  // the next row's partial sums do not meet this one's readers
    const float c = dot / (float)a.H * r * r;
#pragma unroll
    for (int i = 0; i < kV; ++i) {
      const int v = lane + i * kLanes;
      float fy[8], fh[8], fw[8], fs[8];
      unpack8(dy[i], fy);
      unpack8(h[i], fh);
      unpack8(w[i], fw);
      unpack8(ds[i], fs);
#pragma unroll
      for (int e = 0; e < 8; ++e) fy[e] = r * (fy[e] * fw[e] - fh[e] * c) + fs[e];
      if (have && v < nvec) ((u32x4*)(a.dx + row * a.H))[v] = pack8(fy);
    }
  }
  // The row groups' sums in their order, a vector of each thread at a time.
  float* mine = a.parts + (int64_t)blockIdx.x * a.H;
#pragma unroll
  for (int i = 0; i < kV; ++i) {
    const int v = lane + i * kLanes;
    if constexpr (kRows > 1) {
      __syncthreads();
#pragma unroll
      for (int e = 0; e < 8; ++e) sums[(sub * 8 + e) * kLanes + lane] = dw[i][e];
      __syncthreads();
      // The row groups share the elements of each lane's vector out among them.
#pragma unroll
      for (int e0 = 0; e0 < 8; e0 += kRows) {
        float s = 0.0f;
#pragma unroll
        for (int g = 0; g < kRows; ++g) s += sums[(g * 8 + e0 + sub) * kLanes + lane];
        if (v < nvec) mine[v * 8 + e0 + sub] = s;
      }
    } else if (v < nvec) {
#pragma unroll
      for (int e = 0; e < 8; ++e) mine[v * 8 + e] = dw[i][e];
    }
  }
}

typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));  // the gradient itself may be the sums

// Rows too long for registers: read twice, the sums kept in the workspace.
__global__ __launch_bounds__(kBackThreads) void norm_backward_wide_kernel(NormBackwardArgs a) {
  __shared__ float part[2][kBackThreads / 64];
  const int nvec = a.H / 8;
  float* mine = a.parts + (int64_t)blockIdx.x * a.H;
  int turn = 0;
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const u32x4* dyv = (const u32x4*)(a.dy + row * a.H);
    const u32x4* hv = (const u32x4*)(a.h + row * a.H);
    const u32x4* wv = (const u32x4*)a.weight;
    float dot = 0.0f;
    for (int v = threadIdx.x; v < nvec; v += kBackThreads) {
      float fy[8], fh[8], fw[8];
      unpack8(dyv[v], fy);
      unpack8(hv[v], fh);
      unpack8(wv[v], fw);
#pragma unroll
      for (int e = 0; e < 8; ++e) dot += fy[e] * fw[e] * fh[e];
    }
    dot = row_reduce<kBackThreads>(dot, part[turn], add);
    turn ^= 1;
    const float r = a.rstd[row];
    const float c = dot / (float)a.H * r * r;
    for (int v = threadIdx.x; v < nvec; v += kBackThreads) {
      float fy[8], fh[8], fw[8], fs[8] = {}, dw[8];
      unpack8(dyv[v], fy);
      unpack8(hv[v], fh);
      unpack8(wv[v], fw);
      if (a.dsum) unpack8(((const u32x4*)(a.dsum + row * a.H))[v], fs);
      f32x4_any* sum = (f32x4_any*)(mine + v * 8);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        dw[e] = fy[e] * (fh[e] * r);
        fy[e] = r * (fy[e] * fw[e] - fh[e] * c) + fs[e];
      }
      f32x4_any s0{}, s1{};
      if (row != blockIdx.x) s0 = sum[0], s1 = sum[1];
      sum[0] = f32x4_any{s0[0] + dw[0], s0[1] + dw[1], s0[2] + dw[2], s0[3] + dw[3]};
      sum[1] = f32x4_any{s1[0] + dw[4], s1[1] + dw[5], s1[2] + dw[6], s1[3] + dw[7]};
      ((u32x4*)(a.dx + row * a.H))[v] = pack8(fy);
    }
  }
}

// dweight[c] = the parts' sums: 32 columns a workgroup, 32 threads down each, joined in their order.
constexpr int kSumCols = 32, kSumRows = 32;
__global__ __launch_bounds__(kSumCols* kSumRows) void norm_weight_kernel(const float* parts, int n, int32_t H, float* dweight) {
  __shared__ float sums[kSumRows][kSumCols + 1];
  const int col = threadIdx.x % kSumCols, down = threadIdx.x / kSumCols, c = blockIdx.x * kSumCols + col;
  float s = 0.0f;
  if (c < H) {
#pragma unroll 8
    for (int p = down; p < n; p += kSumRows) s += parts[(int64_t)p * H + c];
  }
  sums[down][col] = s;
  __syncthreads();
  if (down == 0 && c < H) {
#pragma unroll
    for (int i = 1; i < kSumRows; ++i) s += sums[i][col];
    dweight[c] = s;
  }
}

hipError_t launch_norm_backward(const NormBackwardArgs& args, hipStream_t s) {
  NormBackwardArgs a = args;
  const int64_t parts = a.rows > 0 ? norm_backward_parts(a.rows, a.H) : 0;
  if (parts == 1) a.parts = a.dweight;
  const int nvec = a.H / 8;
  auto kernel = norm_backward_kernel<kBackThreads, 4>;
  if (a.H > kWideRow)
    kernel = norm_backward_wide_kernel;
  else if (nvec <= 64)
    kernel = norm_backward_kernel<64, 1>;
  else if (nvec <= 128)
    kernel = norm_backward_kernel<64, 2>;
  else if (back_lanes(a.H) == 64)
    kernel = norm_backward_kernel<64, 4>;
  else if (back_lanes(a.H) == 128)
    kernel = norm_backward_kernel<128, 4>;
  else if (back_lanes(a.H) == 256)
    kernel = norm_backward_kernel<256, 4>;
  if (parts > 0)  // no rows: dweight becomes zeros below
    if (hipError_t e = launch(kernel, dim3((uint32_t)parts), dim3(kBackThreads), 0, s, a)) return e;
  if (parts == 1) return hipSuccess;
  return launch(norm_weight_kernel, dim3((a.H + kSumCols - 1) / kSumCols), dim3(kSumCols * kSumRows), 0, s, a.parts,
                (int)parts, a.H, a.dweight);
}

// ------------------------------------------------------------------------------------ back to bf16

template <int kLanes>
__global__ __launch_bounds__(256) void restore_kernel(RestoreArgs a) {
  const int nvec = a.H / 8;
  const int64_t row = (int64_t)blockIdx.x * (256 / kLanes) + threadIdx.x / kLanes;
  if (row >= a.rows) return;
  const float s = a.scale[row];
#pragma unroll 4
  for (int v = threadIdx.x % kLanes; v < nvec; v += kLanes) {
    const u32x2 q = ((const u32x2*)(a.q + row * a.H))[v];
    float f[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = (float)(int8_t)(q[e / 4] >> (8 * (e % 4))) * s;
    ((u32x4*)(a.out + row * a.H))[v] = pack8(f);
  }
}

hipError_t launch_restore(const RestoreArgs& a, hipStream_t s) {
  const bool wave = a.H <= 2048;
  const int64_t blocks = wave ? (a.rows + 3) / 4 : a.rows;
  if (!launch_fits(blocks, 256)) return hipErrorInvalidConfiguration;
  return launch(wave ? restore_kernel<64> : restore_kernel<256>, dim3((uint32_t)blocks), dim3(256), 0, s, a);
}

}  // namespace moe
