// product.hip -- gfx950 kernels of the experts' 16-bit products and of the gradient by their rows.
//
//   moe_product     out[i, n] = bf16( sum_k x[r_i, k] w[e, n, k] )
//   moe_product_dx  dx[i, k]  = bf16( sum_n dy[i, n] w[e, n, k] )
//
// Both are out[i, n] = sum_k x[r_i, k] W[n, k], with W's rows in memory (ByRow) or its columns (ByK: the LDS read turns
// them round, so the weights are needed once and in one layout).  v_mfma_f32_16x16x32_bf16, sums in fp32.  The weights
// are the A operand, so a lane ends up with 4 consecutive features of one row and stores them together.
//
// Three kinds of kernel, chosen by an estimate of each one's time (product_kind):
//  * whole tiles of 256 features by up to 256 rows, one workgroup a compute unit that stays; tall tiles follow one
//    another in the ring.  Their K steps bound them: 8192 rows by 4096 x 14336 take 630 us (1.53 PFLOP/s; the library's
//    product 613), ByK 616 (1.56; 689).  Ragged experts cost what their short last tiles and the last round leave idle:
//    64 of some 768 rows by 2816 x 2048 480 us (1.18), 8 of some 1024 by 4096 x 14336 770 (1.25).
//  * tiles of 128 features by 128 or 64 rows, or of 64 each way, bound by their loads, where whole tiles would leave compute
//    units idle.
//  * 16 rows by 16, 32 or (ByK) 64 features, K divided among the waves, for a few rows of each expert: bound by the
//    reading of the weights (32 experts of 4096 x 7168, 8 rows each: 1.88 GB in 310 us, 6.1 TB/s; tiles of 64
//    take 302 there), or by its latency.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <cmath>

#include "expert_tiles.hpp"
#include "launch.hpp"
#include "mma_tile.hpp"
#include "ops.hpp"
#include "vec_device.hpp"

namespace moe {

namespace {

template <bool by_k>
using WeightLayout = std::conditional_t<by_k, ByK, ByRow>;

constexpr float kNan = __builtin_nanf("");

// Where a K loop over a.K ends: rows of a.K elements are not read past their end.
template <bool by_k>
__device__ __forceinline__ ElementTail tail_of(const ProductArgs& a) {
  return ElementTail(a.K, true, by_k ? (uint32_t)a.N * 2 : 2u, 2u);
}

// The weights of a tile as a DMA source: kDma instructions a wave, the tile's features from `first` on.
template <bool by_k, int kDma>
__device__ __forceinline__ void weight_rows(const ProductArgs& a, int expert, int first, int lane, int wave, DmaRows<kDma>& w) {
  const int K = a.K, N = a.N;
  const uint32_t r8 = (uint32_t)lane >> 3;
  if constexpr (by_k) {
    // Block rows of the wave's DMAs: panel by panel, 64 k each.
    const int panel = wave * kDma / 8, k0 = wave * kDma % 8 * 8;
    w.step = (uint32_t)kTileK * (uint32_t)N * 2;
    w.base = (const uint8_t*)(a.w + (int64_t)expert * K * N + first);
#pragma unroll
    for (int i = 0; i < kDma; ++i) {
      const uint32_t k = (uint32_t)(k0 + 8 * i) + r8;
      const int col = min(first + panel * 64 + (int)((((uint32_t)lane & 7) ^ swz_k(k)) << 3), N - 8) - first;
      w.off[i] = (min(k, (uint32_t)K - 1) * (uint32_t)N + (uint32_t)col) * 2;
    }
  } else {
    const int cmax = min(K / 8, 8) - 1;
    auto feature = [&](int n) { return min(first + n, N - 1); };
    const int f0 = feature(wave * kDma * 8);
    w.step = kRowBytes;
    w.base = (const uint8_t*)(a.w + ((int64_t)expert * N + f0) * K);
#pragma unroll
    for (int i = 0; i < kDma; ++i) {
      const uint32_t n = (uint32_t)((wave * kDma + i) * 8) + r8;
      const uint32_t c = min(((uint32_t)lane & 7) ^ swz(n), (uint32_t)cmax);
      w.off[i] = (uint32_t)(feature((int)n) - f0) * (uint32_t)K * 2 + (c << 4);
    }
  }
}

// Whether row i of out has a row of x, and which; a row that row_index does not name takes row 0 (any readable one).
__device__ __forceinline__ bool named(const ProductArgs& a, uint32_t r) { return (int64_t)r < a.x_rows; }

// ------------------------------------------------------------------------------------ small tiles

// K steps in a small tile's ring.  Four, of which a compute unit holds two workgroups with tiles of 64 and one with
// tiles of 128.  With weights ByK two workgroups of tiles of 128 with two steps each are 5 % faster (290 products of over
// 40 us; 3 % slower ByRow), since one's reads fill the other's waits, except where every compute unit has one tile at most:
// three steps for it alone take 10 % less there (16 experts of some 180 rows, 1408 x 1024: 22.7 -> 19.6 us).  Tiles of 64
// with two steps: 20 to 40 % slower.  128 features by 64 rows have three, two workgroups a compute unit.
template <bool by_k, int kW, int kX>
constexpr int kStages = kW != kX ? 3 : by_k && kW == 128 ? 2 : 4;

template <int kW, int kX>
struct SmallShape {
  static constexpr int kStride = kW * 2 + 16;  // of a finished row in LDS
  static constexpr int kOutBytes = kX * kStride;
};

// One tile of kW features by kX rows, of which it.rows are valid.
template <bool by_k, int kW, int kX, int kSteps>
__device__ __forceinline__ void small_item(const ProductArgs& a, const Item& it, uint8_t* lds) {
  using S = SmallShape<kW, kX>;
  constexpr int kNI = kW / 32, kNJ = kX / 32;
  const int tid = item_thread(), lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lr = lane & 15, lk = lane >> 4;
  const int K = a.K, N = a.N, first = it.col * kW;
  const uint32_t cmax = (uint32_t)min(K / 8, 8) - 1;
  DmaRows<kNI> w;
  DmaRows<kNJ> x;
  weight_rows<by_k>(a, it.expert, first, lane, wave, w);
  auto source = [&](int m) {
    const int i = it.row0 + min(m, it.rows - 1);
    return (uint32_t)(a.index ? a.index[i] : i);
  };
  const int row0 = a.index ? 0 : it.row0;
  x.step = kRowBytes;
  x.base = a.x_rows > 0 ? (const uint8_t*)(a.x + (int64_t)row0 * K) : (const uint8_t*)a.w;
#pragma unroll
  for (int i = 0; i < kNJ; ++i) {
    const uint32_t n = (uint32_t)((wave * kNJ + i) * kRowsPerDma) + ((uint32_t)lane >> 3), r = source((int)n);
    const uint32_t c = min(((uint32_t)lane & 7) ^ swz(n), cmax);
    x.off[i] = (named(a, r) ? (r - (uint32_t)row0) * (uint32_t)K * 2 : 0u) + (c << 4);
  }
  bool ok[kNJ];
#pragma unroll
  for (int j = 0; j < kNJ; ++j) ok[j] = !a.index || named(a, source((wave >> 1) * (kX / 2) + j * 16 + lr));
  // Offsets are complete before the first operand DMA, which the compiler does not count.
#pragma unroll
  for (int i = 0; i < kNJ; ++i) asm volatile("" ::"v"(x.off[i]));
#pragma unroll
  for (int j = 0; j < kNJ; ++j) asm volatile("" ::"v"((int)ok[j]));

  f32x4 acc[kNI][kNJ];
  small_mma<Bf16Mma, kW, kX, kSteps, WeightLayout<by_k>>(lds, w, x, K, tail_of<by_k>(a), acc);

#pragma unroll
  for (int i = 0; i < kNI; ++i)
#pragma unroll
    for (int j = 0; j < kNJ; ++j) {
      f32x4 v = acc[i][j];
      if (!ok[j]) v = f32x4{kNan, kNan, kNan, kNan};
      const int m = (wave >> 1) * (kX / 2) + j * 16 + lr, n = (wave & 1) * (kW / 2) + i * 16 + 4 * lk;
      *(u32x2*)(lds + m * S::kStride + n * 2) = u32x2{bf16x2_of(v[0], v[1]), bf16x2_of(v[2], v[3])};
    }
  __syncthreads();
  constexpr int kLanes = kW / 8;  // threads that store one row
  const int c8 = tid % kLanes, f = first + c8 * 8;
  if (f < N) {
#pragma unroll 4
    for (int p = 0; p < kX * kLanes / kThreads; ++p) {
      const int m = p * (kThreads / kLanes) + tid / kLanes;
      if (m < it.rows) *(u32x4*)(a.out + (int64_t)(it.row0 + m) * N + f) = *(const u32x4*)(lds + m * S::kStride + c8 * 16);
    }
  }
}

template <bool by_k, int kW, int kX, int kSteps = kStages<by_k, kW, kX>>
__global__ __launch_bounds__(kThreads, 2 * kSteps * (kW + kX) * kRowBytes <= kLdsBytes ? 2 : 1) void product_small_kernel(ProductArgs a, int cols) {
  constexpr int kRing = kSteps * (kW + kX) * kRowBytes, kOut = SmallShape<kW, kX>::kOutBytes;
  __shared__ __attribute__((aligned(1024))) uint8_t lds[kRing > kOut ? kRing : kOut];
  const Item it = uniform(Items<kX>(a, cols).find(a, blockIdx.x % kXcds, blockIdx.x / kXcds));
  if (it.rows <= 0) return;
  small_item<by_k, kW, kX, kSteps>(a, it, lds);
}

// ------------------------------------------------------------------------------------ whole tiles

// What a tile's DMAs read.
template <bool by_k>
struct ProductSource {
  DmaRows<kDmaPerThread> w;
  DmaRows<8> x;
  uint32_t row[8];  // of x, for the tile whose addresses come next
  // First the rows, which may have to be looked up ...
  __device__ __forceinline__ void rows(const ProductArgs& a, const Item& it) {
    const int lane = item_thread() & 63, wave = __builtin_amdgcn_readfirstlane(item_thread() >> 6);
    const int dx = row_dmas(it.rows);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int n = (wave * dx + i) * kRowsPerDma + (lane >> 3), m = it.row0 + min(n, it.rows - 1);
      row[i] = (uint32_t)(a.index ? a.index[m] : m);
    }
  }
  // ... then the addresses.
  __device__ __forceinline__ void addresses(const ProductArgs& a, const Item& it) {
    const int lane = item_thread() & 63, wave = __builtin_amdgcn_readfirstlane(item_thread() >> 6);
    const int K = a.K, dx = row_dmas(it.rows);
    const uint32_t cmax = (uint32_t)min(K / 8, 8) - 1;
    weight_rows<by_k>(a, it.expert, it.col * 256, lane, wave, w);
    const int row0 = a.index ? 0 : it.row0;
    x.step = kRowBytes;
    x.base = a.x_rows > 0 ? (const uint8_t*)(a.x + (int64_t)row0 * K) : (const uint8_t*)a.w;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t n = (uint32_t)((wave * dx + i) * kRowsPerDma) + ((uint32_t)lane >> 3);
      const uint32_t c = min(((uint32_t)lane & 7) ^ swz(n), cmax);
      x.off[i] = (named(a, row[i]) ? (row[i] - (uint32_t)row0) * (uint32_t)K * 2 : 0u) + (c << 4);
      asm volatile("" ::"v"(x.off[i]));  // complete before the first DMA, which the compiler does not count
    }
  }
  template <int kDma>
  __device__ __forceinline__ DmaRows<kDma> first_rows() const {
    DmaRows<kDma> r{x.base, kRowBytes, {}};
#pragma unroll
    for (int i = 0; i < kDma; ++i) r.off[i] = x.off[i];
    return r;
  }
  // The first K steps on their way, the bases at the step after them.
  __device__ __forceinline__ void start(const ProductArgs& a, const Item& it, uint8_t* lds) {
    const ElementTail tail = tail_of<by_k>(a);
    auto narrow = [&](auto dma) {
      auto r = first_rows<decltype(dma)::value>();
      narrow_start<2 * decltype(dma)::value>(lds, w, r, a.K, tail);
      x.base = r.base;
    };
    auto tall = [&](auto dma) {
      auto r = first_rows<decltype(dma)::value>();
      tile_start<decltype(dma)::value>(lds, w, r, a.K, tail);
      x.base = r.base;
    };
    using std::integral_constant;
    switch (row_dmas(it.rows)) {
      case 1: return narrow(integral_constant<int, 1>{});
      case 2: return narrow(integral_constant<int, 2>{});
      case 4: return tall(integral_constant<int, 4>{});
      case 6: return tall(integral_constant<int, 6>{});
      default: return tall(integral_constant<int, 8>{});
    }
  }
};

// The finished tile: acc[i][j] holds features quad_n(i) + 4 lk on of row quad_m(j) + lr, r[j] that row's of x.
// A lane has 4 consecutive features of a row in each of two fragments; the lanes 16 apart exchange quads, so that
// each stores 8 consecutive features of one.  A tall tile that is full, of rows that are there, is stored without a question.
template <bool tall, int kNI, int kNJ, class QuadN, class QuadM>
__device__ __forceinline__ void store_tile(const ProductArgs& a, const Item& it, f32x4 (&acc)[kNI][kNJ], const uint32_t (&r)[kNJ],
                                           QuadN&& quad_n, QuadM&& quad_m) {
  const int lane = item_thread() & 63, lk = lane >> 4, N = a.N, first = it.col * 256;
  auto store = [&](auto whole) {
    constexpr bool kWhole = decltype(whole)::value;
#pragma unroll
    for (int j = 0; j < kNJ; ++j) {
      const bool ok = named(a, r[j]);
      const int m = quad_m(j, lane), f = first + (lk & 1) * 16 + (lk >> 1) * 8;
      uint16_t* row = a.out + (int64_t)(it.row0 + m) * N + f;
#pragma unroll
      for (int i = 0; i < kNI; i += 2) {
        uint32_t h[2][2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          float v[4];
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            v[q] = acc_read(acc[i + u][j][q]);
            if (!kWhole && !ok) v[q] = kNan;
          }
          h[u][0] = bf16x2_of(v[0], v[1]);
          h[u][1] = bf16x2_of(v[2], v[3]);
        }
        const auto lo = __builtin_amdgcn_permlane16_swap(h[0][0], h[1][0], false, false);
        const auto hi = __builtin_amdgcn_permlane16_swap(h[0][1], h[1][1], false, false);
        if (kWhole || (m < it.rows && f + quad_n(i) < N)) *(u32x4*)(row + quad_n(i)) = u32x4{lo[0], hi[0], lo[1], hi[1]};
        __builtin_amdgcn_sched_barrier(0);  // block by block, or the accumulators are all read at once
      }
    }
  };
  if constexpr (tall) {
    bool all = it.rows == 32 * kNJ && first + 256 <= N;
#pragma unroll
    for (int j = 0; j < kNJ; ++j) all = all && named(a, r[j]);
    if (__all(all)) return store(std::true_type{});
  }
  store(std::false_type{});
}

// Which rows of x a lane's columns of a tile are.
template <int kNJ, class QuadM>
__device__ __forceinline__ void lane_rows(const ProductArgs& a, const Item& it, uint32_t (&r)[kNJ], QuadM&& quad_m) {
  const int lane = item_thread() & 63;
#pragma unroll
  for (int j = 0; j < kNJ; ++j) {
    const int m = it.row0 + min(quad_m(j, lane), it.rows - 1);
    r[j] = (uint32_t)(a.index ? a.index[m] : m);
  }
}
template <int n>
__device__ __forceinline__ void arrived(const uint32_t (&r)[n]) {  // the compiler waits for them here, not under later DMAs
#pragma unroll
  for (int j = 0; j < n; ++j) asm volatile("" ::"v"(r[j]));
}

// Tiles of up to 64 rows, whose first K steps `src` has started: the K loop, the next item's start, which find() gives,
// and under it the epilogue.  Leaves the next item in `it`.
template <bool by_k, int kDma, class Find>
__device__ __forceinline__ void narrow_item(const ProductArgs& a, Item& it, ProductSource<by_k>& src, uint8_t* lds, Find&& find) {
  constexpr int kNJ = 2 * kDma;
  const int wave = __builtin_amdgcn_readfirstlane(item_thread() >> 6);
  auto quad_n = [&](int i) { return (wave >> 1) * 128 + (i >> 1) * 64 + (wave & 1) * 32 + (i & 1) * 16; };
  auto quad_m = [&](int j, int lane) { return j * 16 + (lane & 15); };
  DmaRows<kDma> x = src.template first_rows<kDma>();
  f32x4 acc[4][kNJ];
  uint32_t r[kNJ];
  const Item next = find();
  // Which rows there are, and the next item's, are asked for near the loop's end: all are there when it ends.
  auto late = [&] {
    lane_rows(a, it, r, quad_m);
    if (next.rows > 0) src.rows(a, next);
  };
  narrow_run<Bf16MmaBuiltin, WeightLayout<by_k>>(lds, src.w, x, a.K, tail_of<by_k>(a), acc, late, [] {});
  arrived(r);
  if (next.rows > 0) {
    src.addresses(a, next);
    src.start(a, next, lds);
  }
  store_tile<false>(a, it, acc, r, quad_n, quad_m);
  it = next;
}

// Tiles of 32 kDma rows one after another, as long as the next item is as high.  The first is started by `src`, or
// (`running`) by the tile before it, in its ring.  Leaves the next item in `it`, started; true: in the ring.
template <bool by_k, int kDma, class Find>
__device__ __forceinline__ bool tall_items(const ProductArgs& a, Item& it, ProductSource<by_k>& src, uint8_t* lds, Ring& ring, bool running,
                                           Find&& find) {
  const int wave = __builtin_amdgcn_readfirstlane(item_thread() >> 6);
  auto quad_n = [&](int i) { return (wave & 1) * 128 + i * 16; };
  auto quad_m = [&](int j, int lane) { return (wave >> 1) * (16 * kDma) + j * 16 + (lane & 15); };
  const ElementTail tail = tail_of<by_k>(a);
  const int nk = ElementTail::steps(a.K);
  TileStream<Bf16Mma, WeightLayout<by_k>, ByRow, kDma> stream;
  if (running)
    stream.resume(lds, ring);
  else
    stream.begin(lds, nk);
  uint32_t follows;
  do {
    f32x4 acc[8][kDma];
    uint32_t r[kDma];
    Item next;
    auto early = [&] {
      lane_rows(a, it, r, quad_m);
      next = find();
      if (next.rows > 0) src.rows(a, next);
    };
    // Another tall tile may follow in the ring.
    auto late = [&] {
      arrived(r);
      const int dma = nk > 1 && next.rows > 64 ? row_dmas(next.rows) : 0;
      if (dma > 0) {
        src.addresses(a, next);
        advance_to(src.w, src.x, 0, nk, tail);
      }
      return Following<ElementTail>{(uint32_t)dma, nk, tail};
    };
    follows = stream.run(src.w, src.x, nk, tail, acc, early, late);
    if (follows == 0) {
      stream.end();
      if (next.rows > 0) {
        src.addresses(a, next);
        src.start(a, next, lds);
      }
    }
    store_tile<true>(a, it, acc, r, quad_n, quad_m);
    it = next;
  } while (follows == kDma);
  ring = stream.o;
  return follows > 0;
}

// Workgroups that stay: b takes item (b / 8 + 7 n) mod (workgroups of its XCD) of the n-th set that its XCD's
// workgroups take together.  (Rotating keeps a workgroup from meeting the short last tile of one expert after
// another.)
template <bool by_k>
__global__ __launch_bounds__(kThreads, 1) void product_tile_kernel(ProductArgs a, int cols) {
  __shared__ __attribute__((aligned(1024))) uint8_t lds[kLdsBytes];
  const Items<256> items(a, cols);
  const uint32_t xcd = blockIdx.x % kXcds, mine = blockIdx.x / kXcds, set = gridDim.x / kXcds;
  uint32_t n = 0;
  auto find = [&] {
    const uint32_t j = n * set + (mine + 7 * n) % set;
    ++n;
    return uniform(items.find(a, xcd, j));
  };
  Item it = find();
  if (it.rows <= 0) return;
  ProductSource<by_k> src;
  src.rows(a, it);
  src.addresses(a, it);
  src.start(a, it, lds);
  Ring ring{};
  bool running = false;
  while (it.rows > 0) {
    switch (row_dmas(it.rows)) {
      case 1: narrow_item<by_k, 1>(a, it, src, lds, find); break;
      case 2: narrow_item<by_k, 2>(a, it, src, lds, find); break;
      case 4: running = tall_items<by_k, 4>(a, it, src, lds, ring, running, find); break;
      case 6: running = tall_items<by_k, 6>(a, it, src, lds, ring, running, find); break;
      default: running = tall_items<by_k, 8>(a, it, src, lds, ring, running, find); break;
    }
  }
}

// ------------------------------------------------------------------------------------ few rows

// A tile of 16 rows by 16 kN features: the four waves take every fourth 128 bytes of K each, straight from memory
// into registers, so nothing in the loop waits for another wave, and add their sums up in LDS at the end.
template <int kN>
__global__ __launch_bounds__(kThreads) void product_slim_kernel(ProductArgs a) {
  constexpr int kWaves = kThreads / 64, kStep = 64;  // k of a wave's turn: two of the matrix instruction
  __shared__ f32x4 sums[kWaves][kN][64];
  const Item it = uniform(find_rows<16>(a, blockIdx.y));
  if (it.rows <= 0) return;
  const int lane = threadIdx.x & 63, lr = lane & 15, lk = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int K = a.K, N = a.N, n0 = blockIdx.x * 16 * kN;
  const uint16_t* wp[kN];
#pragma unroll
  for (int i = 0; i < kN; ++i) wp[i] = a.w + ((int64_t)it.expert * N + min(n0 + i * 16 + lr, N - 1)) * K + lk * 8;
  const int mine = it.row0 + min(lr, it.rows - 1);
  const uint32_t r = (uint32_t)(a.index ? a.index[mine] : mine);
  const bool ok = named(a, r);
  const uint16_t* xp = (ok ? a.x + (int64_t)r * K : a.w) + lk * 8;
  f32x4 acc[kN];
#pragma unroll
  for (int i = 0; i < kN; ++i) acc[i] = f32x4{};
  struct Chunk {
    bf16x8 w[2][kN], x[2];
  };
  auto load = [&](Chunk& c, int k) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
#pragma unroll
      for (int i = 0; i < kN; ++i) c.w[h][i] = *(const bf16x8*)(wp[i] + k + h * 32);
      c.x[h] = *(const bf16x8*)(xp + k + h * 32);
    }
  };
  auto multiply = [&](const Chunk& c) {
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int i = 0; i < kN; ++i) acc[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(c.w[h][i], c.x[h], acc[i], 0, 0, 0);
  };
  const int nfull = K / kStep;
  Chunk c0, c1;
  int c = wave;
  if (c < nfull) load(c0, c * kStep);
  while (c < nfull) {
    if (c + kWaves < nfull) load(c1, (c + kWaves) * kStep);
    multiply(c0);
    c += kWaves;
    if (c >= nfull) break;
    if (c + kWaves < nfull) load(c0, (c + kWaves) * kStep);
    multiply(c1);
    c += kWaves;
  }
  if (K % kStep && wave == nfull % kWaves) {  // the last chunks of 8
    const int k = nfull * kStep;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const bool in = k + h * 32 + lk * 8 < K;
#pragma unroll
      for (int i = 0; i < kN; ++i) {
        c0.w[h][i] = bf16x8{};
        if (in) c0.w[h][i] = *(const bf16x8*)(wp[i] + k + h * 32);
      }
      c0.x[h] = bf16x8{};
      if (in) c0.x[h] = *(const bf16x8*)(xp + k + h * 32);
    }
    multiply(c0);
  }
#pragma unroll
  for (int i = 0; i < kN; ++i) sums[wave][i][lane] = acc[i];
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kN; ++i) {
    if (i % kWaves != wave) continue;
    const int n = n0 + i * 16 + 4 * lk;
    if (n >= N || lr >= it.rows) continue;
    f32x4 s = sums[0][i][lane];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) s += sums[w][i][lane];
    if (!ok) s = f32x4{kNan, kNan, kNan, kNan};
    *(u32x2*)(a.out + (int64_t)(it.row0 + lr) * N + n) = u32x2{bf16x2_of(s[0], s[1]), bf16x2_of(s[2], s[3])};
  }
}

// The same with the weights ByK, 64 features by 16 rows: a wave fetches every fourth K step into a ring of its own, and
// waits for its own loads alone.  A few rows of up to 64 MB of weights take 20 to 25 % less than with tiles of 64 (10.5
// us at the median of 72 products of one row or two an expert).  Two steps in the ring leave room for two workgroups a
// compute unit; three and one took 7 % longer, 32 rows at a time mostly longer too.
__global__ __launch_bounds__(kThreads, 2) void product_thin_kernel(ProductArgs a) {
  constexpr int kWaves = kThreads / 64, kStages = 2, kDmaX = 2;
  constexpr uint32_t kPanel = 64 * kRowBytes, kStage = kPanel + 16 * kRowBytes, kWave = kStages * kStage;
  static_assert(kWave >= 4 * 64 * sizeof(f32x4), "the sums take the rings' place");
  __shared__ __attribute__((aligned(1024))) uint8_t lds[kWaves * kWave];
  const Item it = uniform(find_rows<16>(a, blockIdx.y));
  if (it.rows <= 0) return;
  const int tid = item_thread(), lane = tid & 63, lr = lane & 15, lk = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int K = a.K, N = a.N, first = blockIdx.x * 64, nk = ElementTail::steps(K);
  const uint32_t r8 = (uint32_t)lane >> 3, cmax = (uint32_t)min(K / 8, 8) - 1;
  const ElementTail tail = tail_of<true>(a);
  DmaRows<8> w;
  w.step = (uint32_t)kTileK * (uint32_t)N * 2;
  w.base = (const uint8_t*)(a.w + (int64_t)it.expert * K * N + first);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t k = (uint32_t)(8 * i) + r8;
    const int col = min(first + (int)((((uint32_t)lane & 7) ^ swz_k(k)) << 3), N - 8) - first;
    w.off[i] = (min(k, (uint32_t)K - 1) * (uint32_t)N + (uint32_t)col) * 2;
  }
  auto source = [&](int m) {
    const int i = it.row0 + min(m, it.rows - 1);
    return (uint32_t)(a.index ? a.index[i] : i);
  };
  const int row0 = a.index ? 0 : it.row0;
  DmaRows<kDmaX> x;
  x.step = kRowBytes;
  x.base = a.x_rows > 0 ? (const uint8_t*)(a.x + (int64_t)row0 * K) : (const uint8_t*)a.w;
#pragma unroll
  for (int i = 0; i < kDmaX; ++i) {
    const uint32_t n = (uint32_t)(8 * i) + r8, r = source((int)n);
    x.off[i] = (named(a, r) ? (r - (uint32_t)row0) * (uint32_t)K * 2 : 0u) + (min(((uint32_t)lane & 7) ^ swz(n), cmax) << 4);
  }
  const bool ok = !a.index || named(a, source(lr));
#pragma unroll
  for (int i = 0; i < kDmaX; ++i) asm volatile("" ::"v"(x.off[i]));  // complete before the first DMA, which the compiler does not count
  asm volatile("" ::"v"((int)ok));

  // K step `wave` first, then every fourth.
  const uint32_t mine = (uint32_t)wave * kWave, to = lds_addr(lds) + mine;
  auto fetch = [&](int step, uint32_t slot) {
    if (step >= nk) return;
    const int64_t back = step == nk - 1 ? 1 : 0;
    const uint8_t* wb = w.base + (int64_t)step * w.step - back * tail.back_w();
    const uint8_t* xb = x.base + (int64_t)step * x.step - back * tail.back_x();
    static_for<8>([&](auto q) { dma16<decltype(q)::value * 1024>(wb, w.off[decltype(q)::value], to + slot); });
    static_for<kDmaX>([&](auto q) { dma16<decltype(q)::value * 1024>(xb, x.off[decltype(q)::value], to + slot + kPanel); });
  };
  const Fragments<ByK, bf16x8> a_lane(0u, lane);
  const Fragments<ByRow, bf16x8> b_lane(0u, lane);
  f32x4 acc[4] = {};
  auto multiply = [&](uint32_t slot, bool last) {
    bf16x8 fa[2][4], fb[2][1];
#pragma unroll
    for (int kk = 0; kk < 2; ++kk) {
      fb[kk][0] = b_lane.read(lds + mine, slot + kPanel, kk, 0);
#pragma unroll
      for (int i = 0; i < 4; ++i) fa[kk][i] = a_lane.read(lds + mine, slot, kk, i * 16);
    }
    if (last) {
#pragma unroll
      for (int kk = 0; kk < 2; ++kk) {
        mask_elements(tail, kk, lk, fa[kk], 0, 4);
        mask_elements(tail, kk, lk, fb[kk], 0, 1);
      }
    }
#pragma unroll
    for (int kk = 0; kk < 2; ++kk)
#pragma unroll
      for (int i = 0; i < 4; ++i) acc[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fa[kk][i], fb[kk][0], acc[i], 0, 0, 0);
  };
  uint32_t slot = 0;
  static_for<kStages - 1>([&](auto s) { fetch(wave + kWaves * decltype(s)::value, decltype(s)::value * kStage); });
  uint32_t free_slot = (kStages - 1) * kStage;
  for (int step = wave; step < nk; step += kWaves) {
    const int ahead = step + kWaves * (kStages - 1);
    fetch(ahead, free_slot);
    // The steps after this one that are on their way: each is kDmaX + 8 loads.
    static_for<kStages>([&](auto s) {
      constexpr int n = kStages - 1 - decltype(s)::value;
      const bool exact = n == kStages - 1 ? step + kWaves * n < nk : step + kWaves * n < nk && step + kWaves * (n + 1) >= nk;
      if (exact) wait_vm<n * (8 + kDmaX)>();
    });
    multiply(slot, step == nk - 1);
    wait_vm<63>();  // the reads have returned before the slot is filled again
    free_slot = slot;
    slot = slot == (kStages - 1) * kStage ? 0 : slot + kStage;
  }
  __syncthreads();
  f32x4* sums = (f32x4*)lds;
#pragma unroll
  for (int i = 0; i < 4; ++i) sums[(wave * 4 + i) * 64 + lane] = acc[i];
  __syncthreads();
  const int n = first + wave * 16 + 4 * lk;  // wave i adds up fragments i
  if (n >= N || lr >= it.rows) return;
  f32x4 s = sums[wave * 64 + lane];
#pragma unroll
  for (int v = 1; v < kWaves; ++v) s += sums[(v * 4 + wave) * 64 + lane];
  if (!ok) s = f32x4{kNan, kNan, kNan, kNan};
  *(u32x2*)(a.out + (int64_t)(it.row0 + lr) * N + n) = u32x2{bf16x2_of(s[0], s[1]), bf16x2_of(s[2], s[3])};
}

// ------------------------------------------------------------------------------------ host side

hipError_t launch_thin(const ProductArgs& a, hipStream_t s) {
  const int64_t tiles = most_tiles(a.rows, a.offsets != nullptr, a.experts, 16), cols = ((int64_t)a.N + 63) / 64;
  if (tiles > kSlimTiles || !launch_fits(cols, kThreads)) return hipErrorInvalidConfiguration;
  return launch(product_thin_kernel, dim3((uint32_t)cols, (uint32_t)tiles), dim3(kThreads), 0, s, a);
}

template <int kN>
hipError_t launch_slim(const ProductArgs& a, hipStream_t s) {
  const int64_t tiles = most_tiles(a.rows, a.offsets != nullptr, a.experts, 16), cols = ((int64_t)a.N + 16 * kN - 1) / (16 * kN);
  if (tiles > kSlimTiles || !launch_fits(cols, kThreads)) return hipErrorInvalidConfiguration;
  return launch(product_slim_kernel<kN>, dim3((uint32_t)cols, (uint32_t)tiles), dim3(kThreads), 0, s, a);
}

template <bool by_k, int kW, int kX, int kSteps = kStages<by_k, kW, kX>>
hipError_t launch_tiles(const ProductArgs& a, hipStream_t s) {
  const int64_t tiles = most_tiles(a.rows, a.offsets != nullptr, a.experts, kX);
  const int cols = (a.N + kW - 1) / kW;
  const int64_t grid = dealt(tiles, cols);
  if (kW == 256 ? grid > INT32_MAX : !launch_fits(grid, kThreads)) return hipErrorInvalidConfiguration;
  if constexpr (kW == 256)
    return launch(product_tile_kernel<by_k>, dim3((uint32_t)std::min<int64_t>(grid, kStaying)), dim3(kThreads), 0, s, a, cols);
  else
    return launch(product_small_kernel<by_k, kW, kX, kSteps>, dim3((uint32_t)grid), dim3(kThreads), 0, s, a, cols);
}

}  // namespace

ProductKind product_kind(int64_t rows, bool grouped, int32_t experts, int32_t K, int32_t N, bool by_k) {
  // What each kernel would take, in microseconds, from the rows an expert has on average (the host does not know
  // the offsets): the rounds of tiles over 256 compute units, each so many K steps and something for its start and end;
  // and the reading of every weight, at the rate in TB/s that the kernel reached where that is all.  Fitted to 15675 measured
  // products (1 to 49152 rows, 1 to 128 experts): the kernel chosen takes 2.6 % longer than the best one, 18 % in one of twenty,
  // 97 % at most; by k 1.4, 12 and 91 %.  The tiles of 128 x 64 and the deep ring were worth 1.1 % at the mean of 2000 problems by
  // row and 2.3 by k.
  const double nk = (K + kTileK - 1) / kTileK;
  const double busy = grouped ? experts * (1.0 - std::pow(1.0 - 1.0 / experts, (double)rows)) : 1.0;
  const double per = rows / busy, megabytes = busy * N * (2e-6 * K);
  auto tiles = [&](double x) { return grouped ? busy * (1.0 + std::max(0.0, (per - x / 2) / x)) : std::ceil(rows / x); };
  auto items = [&](double w, double x) { return tiles(x) * std::ceil(N / w) / 256.0; };
  auto by = [&](double row, double k) { return by_k ? k : row; };
  auto cost = [&](double work, double rate) { return std::max(work, megabytes / rate) + 0.35 * work; };
  auto step = [](double h) {
    return h < 64 ? 0.41 + 0.25 * (h - 32) / 32 : h < 128 ? 0.66 + 0.11 * (h - 64) / 64 : 0.77 + 0.615 * (h - 128) / 128;
  };
  const double whole = items(256, 256), half = items(128, 128), quarter = items(64, 64);
  const double height = std::min(256.0, std::max(32.0, per)), rest = whole - std::floor(whole);
  const double pace = by(0.701, 0.94);
  double tall = std::floor(whole) * (nk * pace * step(height) + by(4.73, 5.56));
  if (rest > 0) {
    const int parts = parts_of((uint32_t)std::ceil(rest * kStaying / kXcds));
    tall += nk * pace * step(std::max(32.0, std::min(height, 256.0 / parts))) + by(5.19, 4.15);
  }
  ProductKind best = kProductTiles256;
  double least = cost(by(2.62, 1.52) + tall, by(4.99, 5.18));
  auto consider = [&](ProductKind kind, double c) {
    if (c < least) best = kind, least = c;
  };
  // The small tiles and the slim kernels have a workgroup for each item, and can be too many for one launch.
  auto launches = [&](int w, int x) { return launch_fits(dealt(most_tiles(rows, grouped, experts, x), (N + w - 1) / w), kThreads); };
  if (launches(128, 128))
    consider(kProductTiles128, cost(1.16 + std::ceil(half) * (nk * by(0.449, 0.466) + by(2.97, 2.8)), by(5.14, 4.8)));
  if (by_k && launches(128, 128)) consider(kProductDeep128, cost(0.24 + std::ceil(half) * (nk * 0.46 + 3.75), 5.36));
  if (launches(128, 64))
    consider(kProductTiles128x64, cost(by(2.16, 1.2) + std::ceil(items(128, 64)) * (nk * by(0.263, 0.313) + by(1.32, 1.11)), by(5.24, 5.2)));
  if (launches(64, 64))
    consider(kProductTiles64, cost(by(2.23, 1.68) + std::max(1.0, quarter) * (nk * by(0.231, 0.282) + by(0.894, 0.627)), by(6.84, 5.1)));
  if (most_tiles(rows, grouped, experts, 16) > kSlimTiles || !launch_fits(((int64_t)N + 15) / 16, kThreads)) return best;
  if (by_k) {
    consider(kProductSlim1, cost(2.21 + nk * std::max(0.075, 0.279 * items(64, 16)), 3.72));
  } else {
    consider(kProductSlim1, cost(1.4 + nk * std::max(0.12, 0.163 * items(16, 16)), 6.9));
    consider(kProductSlim2, cost(2.4 + nk * 0.16 * std::max(1.0, items(32, 16)), 6.9));
  }
  return best;
}

hipError_t launch_product_kind(ProductKind kind, const ProductArgs& a, bool by_k, hipStream_t s) {
  switch (kind) {
    case kProductSlim1:
      return by_k ? launch_thin(a, s) : launch_slim<1>(a, s);
    case kProductSlim2:  // by k there is one of them
      return by_k ? launch_thin(a, s) : launch_slim<2>(a, s);
    case kProductTiles64:
      return by_k ? launch_tiles<true, 64, 64>(a, s) : launch_tiles<false, 64, 64>(a, s);
    case kProductTiles128:
      return by_k ? launch_tiles<true, 128, 128>(a, s) : launch_tiles<false, 128, 128>(a, s);
    case kProductTiles128x64:
      return by_k ? launch_tiles<true, 128, 64>(a, s) : launch_tiles<false, 128, 64>(a, s);
    case kProductDeep128:  // by row the tiles of 128 have as many steps
      return by_k ? launch_tiles<true, 128, 128, 3>(a, s) : launch_tiles<false, 128, 128>(a, s);
    case kProductTiles256:
      return by_k ? launch_tiles<true, 256, 256>(a, s) : launch_tiles<false, 256, 256>(a, s);
  }
  return hipErrorInvalidValue;
}

hipError_t launch_product(const ProductArgs& a, bool by_k, hipStream_t s) {
  return launch_product_kind(product_kind(a.rows, a.offsets != nullptr, a.experts, a.K, a.N, by_k), a, by_k, s);
}

}  // namespace moe
