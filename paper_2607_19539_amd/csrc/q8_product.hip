// q8_product.hip -- gfx950 kernels of the experts' products in 8 bits.
//
//   out[i, n] = bf16( float(sum_k x[r_i, k] w[e, n, k]) * (xs[r_i] ws[e, n]) ),  or silu(g) * u of two of them
//
// v_mfma_i32_16x16x64_i8, 32-bit integer sums (exact).  The weights are the A operand, so a lane ends up with
// 4 consecutive features of one row and stores them together.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "ops.hpp"
#include "vec_device.hpp"

namespace moe {

typedef int32_t i32x4 __attribute__((ext_vector_type(4)));

constexpr int kThreads = 256;
constexpr int kRows = 64, kCols = 64;  // rows and features of a workgroup's tile; a wave takes 16 features

struct Tile {
  int expert;    // -1: none
  int64_t row0;  // first row
  int rows;      // valid rows
};

// Tile t of the experts' rows cut into runs of kRows: every thread walks the offsets.
__device__ __forceinline__ Tile find_tile(const Q8Args& a, int t) {
  if (!a.offsets) {
    const int64_t r0 = (int64_t)t * kRows;
    return r0 < a.rows ? Tile{0, r0, (int)min((int64_t)kRows, a.rows - r0)} : Tile{-1, 0, 0};
  }
  int64_t lo = min(max((int64_t)a.offsets[0], (int64_t)0), a.rows);
  for (int e = 0; e < a.experts; ++e) {
    const int64_t hi = min(max((int64_t)a.offsets[e + 1], lo), a.rows);
    const int n = (int)((hi - lo + kRows - 1) / kRows);
    if (t < n) return Tile{e, lo + (int64_t)t * kRows, (int)min((int64_t)kRows, hi - lo - (int64_t)t * kRows)};
    t -= n;
    lo = hi;
  }
  return Tile{-1, 0, 0};
}

__device__ __forceinline__ float silu_mul(float g, float u) { return g / (1.0f + expf(-g)) * u; }

template <bool gated>
__global__ __launch_bounds__(kThreads) void q8_kernel(Q8Args a) {
  const Tile tile = find_tile(a, blockIdx.y);
  if (tile.expert < 0) return;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, lr = lane & 15, lk = lane >> 4;
  const int n0 = blockIdx.x * kCols + wave * 16;
  const int K = a.K, N = a.N;
  const int wrow = min(n0 + lr, N - 1);
  const int8_t* w = a.w + ((int64_t)tile.expert * N + wrow) * K;
  const int8_t* w3 = gated ? a.w3 + ((int64_t)tile.expert * N + wrow) * K : nullptr;
  const int8_t* x[kRows / 16];
  float xs[kRows / 16];
  for (int j = 0; j < kRows / 16; ++j) {
    const int64_t i = tile.row0 + min(j * 16 + lr, tile.rows - 1);
    int64_t r = a.index ? a.index[i] : i;
    const bool ok = r >= 0 && r < a.x_rows;
    if (!ok) r = 0;
    x[j] = a.x_rows > 0 ? a.x + r * K : nullptr;
    xs[j] = ok ? a.xs[r] : __uint_as_float(0x7FC00000u);
  }
  i32x4 acc[kRows / 16] = {}, acc3[kRows / 16] = {};
  for (int k0 = 0; k0 < K; k0 += 64) {
    const int k = k0 + lk * 16;
    i32x4 fa = {}, fa3 = {};
    if (k < K) {
      fa = *(const i32x4*)(w + k);
      if (gated) fa3 = *(const i32x4*)(w3 + k);
    }
    for (int j = 0; j < kRows / 16; ++j) {
      i32x4 fb = {};
      if (k < K && x[j]) fb = *(const i32x4*)(x[j] + k);
      acc[j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fa, fb, acc[j], 0, 0, 0);
      if (gated) acc3[j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fa3, fb, acc3[j], 0, 0, 0);
    }
  }
  // Lane: features n0 + 4 lk + 0..3 of row lr of each 16.
  const int n = n0 + 4 * lk;
  if (n >= N) return;  // N is a multiple of 8: four features are all inside or all outside
  for (int j = 0; j < kRows / 16; ++j) {
    const int m = j * 16 + lr;
    if (m >= tile.rows) continue;
    float v[4];
    for (int q = 0; q < 4; ++q) {
      v[q] = (float)acc[j][q] * (xs[j] * a.ws[(int64_t)tile.expert * N + n + q]);
      if (gated) v[q] = silu_mul(v[q], (float)acc3[j][q] * (xs[j] * a.ws3[(int64_t)tile.expert * N + n + q]));
    }
    *(u32x2*)(a.out + (tile.row0 + m) * N + n) = u32x2{bf16x2_of(v[0], v[1]), bf16x2_of(v[2], v[3])};
  }
}

hipError_t launch_q8(const Q8Args& a, bool gated, hipStream_t s) {
  // Tiles there can be: every expert may end in a partly filled one.
  const int64_t tiles = (a.rows + kRows - 1) / kRows + (a.offsets ? std::min<int64_t>(a.experts, a.rows) : 0);
  if (tiles > 65535) return hipErrorInvalidConfiguration;
  const dim3 grid((a.N + kCols - 1) / kCols, (uint32_t)tiles);
  if (gated)
    hipLaunchKernelGGL(q8_kernel<true>, grid, dim3(kThreads), 0, s, a);
  else
    hipLaunchKernelGGL(q8_kernel<false>, grid, dim3(kThreads), 0, s, a);
  return hipGetLastError();
}

}  // namespace moe
