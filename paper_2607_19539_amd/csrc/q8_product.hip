// q8_product.hip -- gfx950 kernels of the experts' products in 8 bits.
//
//   out[i, n] = bf16( float(sum_k x[r_i, k] w[e, n, k]) * (xs[r_i] ws[e, n]) ),  or silu(g) * u of two of them
//
// v_mfma_i32_16x16x64_i8, 32-bit integer sums (exact).  The weights are the A operand, so a lane ends up with
// 4 consecutive features of one row and stores them together.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "mma_tile.hpp"
#include "ops.hpp"
#include "vec_device.hpp"

namespace moe {

constexpr int kThreads = 256;
constexpr int kRowsTile = kTileM;  // 256 rows of one expert
constexpr int kWTile = 256;        // weight rows of a tile: features, or 128 gate and 128 up features
constexpr int kBand = 4;           // tile rows that take turns on one weight tile
constexpr int kDeal = 32;          // consecutive items that one XCD's compute units run at a time

// Epilogue: the finished tile goes through LDS, rows padded by 16 bytes, the scales behind it.
__host__ __device__ constexpr int out_cols(bool gated) { return gated ? kWTile / 2 : kWTile; }
__host__ __device__ constexpr int out_stride(bool gated) { return out_cols(gated) * 2 + 16; }
constexpr int kScales = kRowsTile * out_stride(false);  // kWTile weight scales, then kRowsTile row scales
static_assert(kScales + (kWTile + kRowsTile) * 4 <= kLdsBytes, "scales behind the staged tile");

// silu(g) * u with the hardware exponential and reciprocal, each within about one fp32 ulp (the bf16
// rounding that follows is 2^-9); a large negative g gives e^-g = inf, a reciprocal of 0 and a result of 0.
__device__ __forceinline__ float silu_mul(float g, float u) {
  return (g * u) * __builtin_amdgcn_rcpf(1.0f + __expf(-g));
}

// Rows [lo, hi) of expert e from the caller's offsets, which the host cannot check: cut to the rows there
// are, and never falling (`prev`: where the experts before it end).
__device__ __forceinline__ void expert_rows(const Q8Args& a, int e, int64_t& lo, int64_t& hi) {
  lo = min(max((int64_t)a.offsets[e], (int64_t)0), a.rows);
  hi = min(max((int64_t)a.offsets[e + 1], (int64_t)0), a.rows);
}

struct Item {
  int expert, col, rows;  // rows: valid rows of the tile, 0: no item
  int64_t row0;
};

template <class T>
__device__ __forceinline__ T shfl_up_max(T v, int lane) {
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const T o = __shfl_up(v, d);
    if (lane >= d) v = max(v, o);
  }
  return v;
}

// Workgroup b's item.  An expert's items are bands of kBand tile rows by all columns, the rows of a band
// next to each other; items are dealt to the XCDs (workgroups b, b + 8, ... share one) in runs of kDeal, so
// that the compute units of an XCD read the same few weight and row tiles through its L2.  Every wave finds
// the item by itself: 64 experts at a time, a lane each.
__device__ __forceinline__ Item find_item(const Q8Args& a, uint32_t b, int cols) {
  const int lane = threadIdx.x & 63;
  const uint32_t xcd = b % kXcds, j = b / kXcds;
  if (!a.offsets) {
    const int64_t tiles = (a.rows + kRowsTile - 1) / kRowsTile;
    const uint32_t total = (uint32_t)(tiles * cols);
    const uint32_t run = min((uint32_t)kDeal, (total + kXcds - 1) / kXcds);
    const uint32_t it = ((j / run) * kXcds + xcd) * run + j % run;
    if (it >= total) return Item{0, 0, 0, 0};
    const uint32_t band = it / (uint32_t)(kBand * cols), q = it % (uint32_t)(kBand * cols);
    const int64_t t0 = (int64_t)band * kBand;
    const uint32_t nb = (uint32_t)min((int64_t)kBand, tiles - t0);
    const int64_t row0 = (t0 + q % nb) * kRowsTile;
    return Item{0, (int)(q / nb), (int)min((int64_t)kRowsTile, a.rows - row0), row0};
  }
  // Tile rows of every expert: a running sum, twice (the deal needs the total first).
  int64_t seen = 0;
  uint32_t before = 0;
  auto chunk = [&](int e0, int64_t& lo, int64_t& hi, uint32_t& end) {
    const int e = e0 + lane;
    lo = hi = 0;
    if (e < a.experts) expert_rows(a, e, lo, hi);
    hi = max(shfl_up_max(max(lo, hi), lane), seen);
    const int64_t ends = __shfl_up(hi, 1);
    lo = max(lo, lane == 0 ? seen : max(ends, seen));
    if (e >= a.experts) lo = hi;
    const uint32_t n = (uint32_t)((hi - lo + kRowsTile - 1) / kRowsTile);
    end = n;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const uint32_t o = __shfl_up(end, d);
      if (lane >= d) end += o;
    }
    end += before;
  };
  for (int e0 = 0; e0 < a.experts; e0 += 64) {
    int64_t lo, hi;
    uint32_t end;
    chunk(e0, lo, hi, end);
    seen = __shfl(hi, 63);
    before = __shfl(end, 63);
  }
  const uint32_t total = before * (uint32_t)cols;
  if (total == 0) return Item{0, 0, 0, 0};
  const uint32_t run = min((uint32_t)kDeal, (total + kXcds - 1) / kXcds);
  const uint32_t it = ((j / run) * kXcds + xcd) * run + j % run;
  if (it >= total) return Item{0, 0, 0, 0};
  seen = 0;
  before = 0;
  for (int e0 = 0; e0 < a.experts; e0 += 64) {
    int64_t lo, hi;
    uint32_t end;
    chunk(e0, lo, hi, end);
    const uint64_t past = __ballot(it < end * (uint32_t)cols);
    if (past != 0) {
      const int l = __builtin_ctzll(past);
      const uint32_t prev = __shfl_up(end, 1);
      const uint32_t first = __builtin_amdgcn_readfirstlane(l == 0 ? before : __shfl(prev, l));
      const uint32_t tiles = __builtin_amdgcn_readfirstlane(__shfl(end, l)) - first;
      const int64_t elo = __shfl(lo, l), ehi = __shfl(hi, l);
      const uint32_t local = it - first * (uint32_t)cols;
      const uint32_t band = local / (uint32_t)(kBand * cols), q = local % (uint32_t)(kBand * cols);
      const uint32_t nb = min((uint32_t)kBand, tiles - band * kBand);
      const int64_t row0 = elo + (int64_t)(band * kBand + q % nb) * kRowsTile;
      return Item{e0 + l, (int)(q / nb), (int)min((int64_t)kRowsTile, ehi - row0), row0};
    }
    seen = __shfl(hi, 63);
    before = __shfl(end, 63);
  }
  return Item{0, 0, 0, 0};
}

// The item in scalar registers: it is the same in every lane.
__device__ __forceinline__ Item uniform(const Item& it) {
  return Item{__builtin_amdgcn_readfirstlane(it.expert), __builtin_amdgcn_readfirstlane(it.col),
              __builtin_amdgcn_readfirstlane(it.rows),
              (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(it.row0 >> 32)) << 32 |
                        (uint32_t)__builtin_amdgcn_readfirstlane((int)it.row0))};
}

// One tile of kRows rows (of which it.rows are valid) by kWTile weight rows.
template <bool gated, int kRows>
__device__ __forceinline__ void q8_item(const Q8Args& a, const Item& it, uint8_t* lds) {
  constexpr bool kNarrow = kRows <= 64;
  constexpr int kNI = kNarrow ? 4 : 8;
  constexpr int kNJ = kNarrow ? kRows / 16 : kRows / 32;
  constexpr int kDmaX = kRows / 32;
  const int tid = item_thread(), lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lr = lane & 15, lk = lane >> 4;
  const int K = a.K, N = a.N;
  auto quad_n = [&](int i) {
    return kNarrow ? (wave >> 1) * 128 + (i >> 1) * 64 + (wave & 1) * 32 + (i & 1) * 16 + 4 * lk
                   : (wave & 1) * 128 + i * 16 + 4 * lk;
  };
  auto quad_m = [&](int j) { return (kNarrow ? 0 : (wave >> 1) * (kRows / 2)) + j * 16 + lr; };
  // Tile row n is feature first + n, or, gated, rows 0..63 and 128..191 are gate features and the 64 rows
  // after each the up rows of the same features: a wave holds both of a feature.
  const int first = it.col * out_cols(gated);
  auto feature = [&](int n) { return gated ? first + (n >> 7) * 64 + (n & 63) : first + n; };
  const uint32_t r8 = (uint32_t)lane >> 3;
  const int cmax = min(K / 16, 8) - 1;
  DmaRows<kDmaPerThread> w;
  DmaRows<kDmaX> x;
  w.step = x.step = kRowBytes;
  const int64_t wofs = (int64_t)it.expert * N;
  {
    const int f0 = min(feature(wave * 64), N - 1);
    w.base = (const uint8_t*)(gated && (wave & 1) ? a.w3 : a.w) + (wofs + f0) * K;
#pragma unroll
    for (int i = 0; i < kDmaPerThread; ++i) {
      const uint32_t n = (uint32_t)(8 * i) + r8;
      const uint32_t c = min(((uint32_t)lane & 7) ^ swz(n), (uint32_t)cmax);
      w.off[i] = (uint32_t)(min(feature(wave * 64 + (int)n), N - 1) - f0) * (uint32_t)K + (c << 4);
    }
  }
  // A row that row_index does not name takes row 0 (any readable one) and a scale of NaN.
  auto source = [&](int m, bool& ok) {
    const int64_t i = it.row0 + min(m, it.rows - 1);
    const int64_t r = a.index ? (int64_t)a.index[i] : i;
    ok = r >= 0 && r < a.x_rows;
    return ok ? r : (int64_t)0;
  };
  const int64_t xrow0 = a.index ? 0 : it.row0;
  x.base = a.x_rows > 0 ? (const uint8_t*)a.x + xrow0 * K : (const uint8_t*)a.w;
#pragma unroll
  for (int i = 0; i < kDmaX; ++i) {
    const uint32_t n = (uint32_t)(wave * kDmaX + i) * kRowsPerDma + r8;
    const uint32_t c = min(((uint32_t)lane & 7) ^ swz(n), (uint32_t)cmax);
    bool ok;
    const int64_t r = source((int)n, ok);
    x.off[i] = (ok ? (uint32_t)(r - xrow0) * (uint32_t)K : 0u) + (c << 4);
  }
  float my_xs, my_ws;
  {
    bool ok;
    const int64_t r = source(tid, ok);
    my_xs = ok ? a.xs[r] : __uint_as_float(0x7FC00000u);
    const int f = min(feature(tid), N - 1);
    my_ws = (gated && ((tid >> 6) & 1) ? a.ws3 : a.ws)[wofs + f];
  }
  // Offsets and scales are complete before the first operand DMA, which the compiler does not count.
#pragma unroll
  for (int i = 0; i < kDmaX; ++i) asm volatile("" ::"v"(x.off[i]));
  asm volatile("" ::"v"(my_xs), "v"(my_ws));

  i32x4 acc[kNI][kNJ];
  const ChunkTail tail(K);
  auto nothing = [] {};
  if constexpr (kNarrow)
    narrow_mma<I8Mma, kNJ>(lds, w, x, K, tail, acc, nothing);
  else
    tile_mma<I8Mma, kNJ>(lds, w, x, K, tail, acc, nothing);

  float* scales = (float*)(lds + kScales);
  scales[tid] = my_ws;
  scales[kWTile + tid] = my_xs;
  __syncthreads();
  constexpr int kStride = out_stride(gated);
  float xs[kNJ];
#pragma unroll
  for (int j = 0; j < kNJ; ++j) xs[j] = scales[kWTile + quad_m(j)];
#pragma unroll
  for (int i = 0; i < (gated ? kNI / 2 : kNI); ++i) {
    const int n = quad_n(i);
    const f32x4 ws = *(const f32x4*)(scales + n);
    f32x4 ws3 = {};
    if constexpr (gated) ws3 = *(const f32x4*)(scales + n + 64);
#pragma unroll
    for (int j = 0; j < kNJ; ++j) {
      float v[4];
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        v[q] = (float)acc[i][j][q] * (xs[j] * ws[q]);
        if constexpr (gated) v[q] = silu_mul(v[q], (float)acc[i + kNI / 2][j][q] * (xs[j] * ws3[q]));
      }
      const int fl = gated ? (n >> 7) * 64 + (n & 63) : n;
      *(u32x2*)(lds + quad_m(j) * kStride + fl * 2) = u32x2{bf16x2_of(v[0], v[1]), bf16x2_of(v[2], v[3])};
      __builtin_amdgcn_sched_barrier(0);  // block by block, or the accumulators are all read at once
    }
  }
  __syncthreads();
  constexpr int kLanes = out_cols(gated) / 8;  // threads that store one row
  const int c8 = tid % kLanes;
  const int f = first + c8 * 8;
  if (f < N) {
#pragma unroll 4
    for (int p = 0; p < kRows * kLanes / kThreads; ++p) {
      const int m = p * (kThreads / kLanes) + tid / kLanes;
      if (m < it.rows) *(u32x4*)(a.out + (it.row0 + m) * N + f) = *(const u32x4*)(lds + m * kStride + c8 * 16);
    }
  }
}

template <bool gated>
__global__ __launch_bounds__(kThreads, 1) void q8_tile_kernel(Q8Args a, int cols) {
  __shared__ __attribute__((aligned(1024))) uint8_t lds[kLdsBytes];
  const Item it = uniform(find_item(a, blockIdx.x, cols));
  const int rows = it.rows;
  if (rows <= 0) return;
  if (rows <= 32)
    q8_item<gated, 32>(a, it, lds);
  else if (rows <= 64)
    q8_item<gated, 64>(a, it, lds);
  else if (rows <= 128)
    q8_item<gated, 128>(a, it, lds);
  else if (rows <= 192)
    q8_item<gated, 192>(a, it, lds);
  else
    q8_item<gated, 256>(a, it, lds);
}

hipError_t launch_q8(const Q8Args& a, bool gated, hipStream_t s) {
  // Tiles there can be: every expert may end in a partly filled one.
  const int64_t tiles = (a.rows + kRowsTile - 1) / kRowsTile + (a.offsets ? std::min<int64_t>(a.experts, a.rows) : 0);
  const int cols = (a.N + out_cols(gated) - 1) / out_cols(gated);
  const int64_t grid = (tiles * cols + kXcds * kDeal - 1) / (kXcds * kDeal) * (kXcds * kDeal);
  if (grid > INT32_MAX) return hipErrorInvalidConfiguration;
  if (gated)
    hipLaunchKernelGGL(q8_tile_kernel<true>, dim3((uint32_t)grid), dim3(kThreads), 0, s, a, cols);
  else
    hipLaunchKernelGGL(q8_tile_kernel<false>, dim3((uint32_t)grid), dim3(kThreads), 0, s, a, cols);
  return hipGetLastError();
}

}  // namespace moe
