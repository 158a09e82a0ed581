// product_dw.hip -- gfx950 kernels of the gradient of the experts' 16-bit products by their weights.
//
//   dw[e, n, k] = sum over rows i of e: dy[i, n] x[r_i, k]      (added to what dw holds, on request)
//
// The rows are what is summed over, and both operands have them as rows in memory: both lie ByK in LDS, x as the A
// operand, so that a lane ends up with 4 consecutive k of one n.  v_mfma_f32_16x16x32_bf16, sums in fp32.  Each expert
// has as many rows as it has: a K step that is not full starts early, or, with fewer than 64 rows, repeats the last.
//
// The sums' writing bounds it as much as the products do: 8 experts of some 1024 rows by 4096 x 14336 (1.88 GB of fp32) take
// 940 us, 720 without the stores, and 64 of some 768 by 2816 x 2048 (1.48 GB) 670 and 496; one matrix of 8192 x 8192 x
// 8192 755 us (1.46 PFLOP/s; into bf16 733, the library's product 939).  Tried without gain: stores past the
// caches (2 to 15 % slower), stores whose lanes lie next to each other (the same, though one compute unit alone then
// stores three times as fast), workgroups out of step with one another by a part of a tile (0 to 5 % slower: their
// reads no longer meet in L2), waits that let the stores pass (the same).
//
// Added to what dw holds, whole tiles read it 16 bytes a lane at a time behind the products: 64 experts of some 768 rows by
// 2816 x 2048 take 1207 us (704 without, on one box), 8 of some 1024 by 4096 x 14336 1649 (986).
//
// Where there are fewer tiles than compute units each expert's rows are split into parts, which leave fp32 sums in the
// workspace, added up in their order by a second launch: the result does not depend on who came first.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <cmath>

#include "expert_tiles.hpp"
#include "launch.hpp"
#include "mma_tile.hpp"
#include "ops.hpp"
#include "row_parts.hpp"
#include "vec_device.hpp"

namespace moe {

namespace {

constexpr float kNan = __builtin_nanf("");
constexpr int kBandTiles = 4;  // tiles of n that take turns on a tile of k

struct DwItem {
  int expert, part, n0, k0;  // the first feature of dy and of x; expert < 0: no item
  int row0, rows;            // of the part
};

// The rows of one expert at a time, from its 64 experts' table.
struct ExpertRows {
  Experts<256> table;
  Before past;
  int e0 = 0;
  __device__ __forceinline__ explicit ExpertRows(const ProductDwArgs& a) {
    if (a.offsets) table = Experts<256>(a, 0, past);
  }
  __device__ __forceinline__ void of(const ProductDwArgs& a, int e, int& lo, int& hi) {
    if (!a.offsets) {
      lo = 0, hi = (int)a.rows;
      return;
    }
    while (e >= e0 + 64) {  // items come in the experts' order
      past = table.after(a, e0);
      e0 += 64;
      table = Experts<256>(a, e0, past);
    }
    lo = __builtin_amdgcn_readlane(table.lo, e - e0);
    hi = __builtin_amdgcn_readlane(table.hi, e - e0);
  }
};

// Item `it` of a launch: the experts one after another, in each the parts, in each bands of kBandTiles tiles of n by
// all tiles of k, the tiles of a band next to each other.
template <int kTile>
__device__ __forceinline__ DwItem dw_item(const ProductDwArgs& a, ExpertRows& experts, int split, uint32_t it) {
  const uint32_t tn = (uint32_t)(a.N + kTile - 1) / kTile, tk = (uint32_t)(a.K + kTile - 1) / kTile, tiles = tn * tk;
  const uint32_t slice = it / tiles, q = it % tiles;
  const int e = (int)(slice / (uint32_t)split), part = (int)(slice % (uint32_t)split);
  if (e >= a.experts) return DwItem{-1, 0, 0, 0, 0, 0};
  const uint32_t band = q / (kBandTiles * tk), in = q % (kBandTiles * tk), nb = min((uint32_t)kBandTiles, tn - band * kBandTiles);
  int lo, hi;
  experts.of(a, e, lo, hi);
  const RowPart rows = row_part(lo, hi, split, part);
  return DwItem{e, part, (int)(band * kBandTiles + in % nb) * kTile, (int)(in / nb) * kTile, rows.row0, rows.rows};
}

__device__ __forceinline__ DwItem uniform(const DwItem& it) {
  auto u = [](int v) { return __builtin_amdgcn_readfirstlane(v); };
  return DwItem{u(it.expert), u(it.part), u(it.n0), u(it.k0), u(it.row0), u(it.rows)};
}

// kDma instructions a wave of the rows `it` has in a matrix of `width` columns, from column `first` on.
template <int kDma>
__device__ __forceinline__ void rows_by_k(const uint16_t* m, int width, const DwItem& it, int first, int lane, int wave, DmaRows<kDma>& d) {
  const uint32_t r8 = (uint32_t)lane >> 3;
  const int panel = wave * kDma / 8, k0 = wave * kDma % 8 * 8;
  d.step = (uint32_t)kTileK * (uint32_t)width * 2;
  d.base = (const uint8_t*)(m + (int64_t)it.row0 * width + first);
#pragma unroll
  for (int i = 0; i < kDma; ++i) {
    const uint32_t k = (uint32_t)(k0 + 8 * i) + r8;
    const int col = min(first + panel * 64 + (int)((((uint32_t)lane & 7) ^ swz_k(k)) << 3), width - 8) - first;
    d.off[i] = (min(k, (uint32_t)it.rows - 1) * (uint32_t)width + (uint32_t)col) * 2;
    asm volatile("" ::"v"(d.off[i]));
  }
}

// x as the A operand: its rows as they lie, or through row_index.
template <bool indexed, int kDma>
using XRows = std::conditional_t<indexed, IndexedRows<kDma>, DmaRows<kDma>>;

template <int kDma>
__device__ __forceinline__ void x_rows(const ProductDwArgs& a, const DwItem& it, int lane, int wave, const IndexAhead&, DmaRows<kDma>& d) {
  rows_by_k(a.x, a.K, it, it.k0, lane, wave, d);
}
template <int kDma>
__device__ __forceinline__ void x_rows(const ProductDwArgs& a, const DwItem& it, int lane, int wave, const IndexAhead& ahead, IndexedRows<kDma>& d) {
  const int panel = wave * kDma / 8;
  d.base = a.x_rows > 0 ? (const uint8_t*)(a.x + it.k0) : (const uint8_t*)a.dw;  // which has a row of K as well
  d.index = a.index + it.row0;
  d.n = it.rows;
  d.limit = (uint32_t)a.x_rows;
  d.stride = (uint32_t)a.K * 2;
  d.first = wave * kDma % 8 * 8 + (lane >> 3);
  d.bad = false;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const uint32_t k = (uint32_t)(d.first + 8 * h);
    const int col = min(it.k0 + panel * 64 + (int)((((uint32_t)lane & 7) ^ swz_k(k)) << 3), a.K - 8) - it.k0;
    d.chunk[h] = (uint32_t)col * 2;
  }
  d.ahead = ahead;
  d.ahead.arrived();
  d.ask(0);
  d.take();
#pragma unroll
  for (int i = 0; i < kDma; ++i) asm volatile("" ::"v"(d.off[i]));  // complete before the first DMA
}
// What x_rows needs from memory.
template <bool indexed>
__device__ __forceinline__ void x_ahead(const ProductDwArgs& a, const DwItem& it, IndexAhead& ahead) {
  if constexpr (indexed) ahead.load(a.index + it.row0, it.rows, 0);
}

// Where the sum over an item's rows ends.  An index starts its last step early by itself.
template <bool indexed>
__device__ __forceinline__ ElementTail tail_of(const ProductDwArgs& a, int rows) {
  return ElementTail(rows, true, indexed ? 0u : (uint32_t)a.K * 2, (uint32_t)a.N * 2);
}

template <int kDma>
__device__ __forceinline__ bool any_bad(const DmaRows<kDma>&) { return false; }
template <int kDma>
__device__ __forceinline__ bool any_bad(const IndexedRows<kDma>& d) { return __any(d.bad); }

// Whether sums leave as bf16: not where they are parts.
__device__ __forceinline__ bool as_bf16(const ProductDwArgs& a, int split) { return a.bf16 && split == 1; }

// Element `at` of dw in fp32 and the three after it, or of a part of it.
template <bool add>
__device__ __forceinline__ void store4(const ProductDwArgs& a, const DwItem& it, int split, int64_t at, f32x4 v) {
  if (split > 1) {
    *(f32x4*)(a.parts + (int64_t)it.part * a.experts * a.N * a.K + at) = v;
  } else {
    f32x4* out = (f32x4*)((float*)a.dw + at);
    if constexpr (add) v += *out;
    *out = v;
  }
}
// Four consecutive k of dw[e, n, :], if they are inside.
__device__ __forceinline__ void store_inside(const ProductDwArgs& a, const DwItem& it, int split, int n, int k, f32x4 v) {
  if (n >= a.N || k >= a.K) return;
  const int64_t at = ((int64_t)it.expert * a.N + n) * a.K + k;
  if (a.accumulate)
    store4<true>(a, it, split, at, v);
  else
    store4<false>(a, it, split, at, v);
}

// The same of dw in bf16, k0 the first of 32 consecutive k: v[u] holds four of the 16 from k0 + 16 u on.  Lanes 16 apart
// exchange quads, so that each stores 8 consecutive k and four of them 64 bytes of a row.  (Quads stored as they come, 32 bytes
// of a row: 64 experts of some 768 rows by 2816 x 2048 675 us, so 620; 8 of some 1024 by 4096 x 14336 935 and 856.)
template <bool inside>
__device__ __forceinline__ void store_bf16(const ProductDwArgs& a, const DwItem& it, int n, int k0, int lk, const f32x4 (&v)[2]) {
  uint32_t h[2][2];
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    h[u][0] = bf16x2_of(v[u][0], v[u][1]);
    h[u][1] = bf16x2_of(v[u][2], v[u][3]);
  }
  const auto lo = __builtin_amdgcn_permlane16_swap(h[0][0], h[1][0], false, false);
  const auto hi = __builtin_amdgcn_permlane16_swap(h[0][1], h[1][1], false, false);
  const int k = k0 + (lk & 1) * 16 + (lk >> 1) * 8;
  if (inside || (n < a.N && k < a.K))
    *(u32x4*)((uint16_t*)a.dw + ((int64_t)it.expert * a.N + n) * a.K + k) = u32x4{lo[0], hi[0], lo[1], hi[1]};
}

// ------------------------------------------------------------------------------------ small tiles

// K steps in a small tile's ring: two, so that a compute unit holds two workgroups with tiles of 128 and four with tiles
// of 64, and one's start and stores run under another's products.  With rings of four and half as many workgroups the
// same sums took 20 to 28 % longer (of 570 of over 10 us).
constexpr int kStages = 2;

template <bool indexed, int kTile>
__global__ __launch_bounds__(kThreads, kTile <= 64 ? 4 : 2) void dw_small_kernel(ProductDwArgs a, int split) {
  constexpr int kN = kTile / 32;
  __shared__ __attribute__((aligned(1024))) uint8_t lds[2 * kStages * kTile * kRowBytes];
  ExpertRows experts(a);
  const DwItem it = uniform(dw_item<kTile>(a, experts, split, blockIdx.x));
  if (it.expert < 0) return;
  const int tid = item_thread(), lane = tid & 63, lr = lane & 15, lk = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  f32x4 acc[kN][kN];
  bool bad = false;
  if (it.rows > 0) {
    XRows<indexed, kN> x;
    DmaRows<kN> y;
    IndexAhead ahead;
    x_ahead<indexed>(a, it, ahead);
    x_rows(a, it, lane, wave, ahead, x);
    rows_by_k(a.dy, a.N, it, it.n0, lane, wave, y);
    small_mma<Bf16Mma, kTile, kTile, kStages, ByK, ByK>(lds, x, y, it.rows, tail_of<indexed>(a, it.rows), acc);
    bad = any_bad(x);  // every wave has asked for all rows of the item
  } else {
#pragma unroll
    for (int i = 0; i < kN; ++i)
#pragma unroll
      for (int j = 0; j < kN; ++j) acc[i][j] = f32x4{};
  }
  // The sums pass through LDS, where the ring was, so that a wave stores whole rows of the tile: as they lie in registers,
  // four lanes to a row, tiles take 3 % longer at the mean of 600 problems, in fp32 as in bf16.
  const int wave_n = (wave >> 1) * (kTile / 2), wave_k = (wave & 1) * (kTile / 2);
  if (as_bf16(a, split)) {
    constexpr int kLanes = kTile / 8, kStride = kTile * 2 + 16;  // threads, and bytes in LDS, of a row
    static_assert(kTile * kStride <= (int)sizeof(lds));
#pragma unroll
    for (int i = 0; i < kN; ++i)
#pragma unroll
      for (int j = 0; j < kN; ++j) {
        f32x4 v = acc[i][j];
        if (bad) v = f32x4{kNan, kNan, kNan, kNan};
        *(u32x2*)(lds + (wave_n + j * 16 + lr) * kStride + (wave_k + i * 16 + 4 * lk) * 2) = u32x2{bf16x2_of(v[0], v[1]), bf16x2_of(v[2], v[3])};
      }
    __syncthreads();
    const int c = tid % kLanes, k = it.k0 + c * 8;
    if (k >= a.K) return;
#pragma unroll 4
    for (int p = 0; p < kTile * kLanes / kThreads; ++p) {
      const int m = p * (kThreads / kLanes) + tid / kLanes, n = it.n0 + m;
      if (n < a.N) *(u32x4*)((uint16_t*)a.dw + ((int64_t)it.expert * a.N + n) * a.K + k) = *(const u32x4*)(lds + m * kStride + c * 16);
    }
    return;
  }
  constexpr int kLanes = kTile / 4, kStride = kTile * 4 + 16, kRows = kTile / 2;  // half of the tile at a time
  static_assert(kRows * kStride <= (int)sizeof(lds));
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    if (half > 0) __syncthreads();
    if (wave >> 1 == half) {
#pragma unroll
      for (int i = 0; i < kN; ++i)
#pragma unroll
        for (int j = 0; j < kN; ++j) {
          f32x4 v = acc[i][j];
          if (bad) v = f32x4{kNan, kNan, kNan, kNan};
          *(f32x4*)(lds + (j * 16 + lr) * kStride + (wave_k + i * 16 + 4 * lk) * 4) = v;
        }
    }
    __syncthreads();
    const int c = tid % kLanes;
#pragma unroll 4
    for (int p = 0; p < kRows * kLanes / kThreads; ++p) {
      const int m = p * (kThreads / kLanes) + tid / kLanes;
      store_inside(a, it, split, it.n0 + half * kRows + m, it.k0 + c * 4, *(const f32x4*)(lds + m * kStride + c * 16));
    }
  }
}

// ------------------------------------------------------------------------------------ whole tiles

template <bool indexed>
struct DwSource {
  XRows<indexed, kDmaPerThread> x;
  DmaRows<8> y;
  IndexAhead ahead;  // of the tile whose addresses come next
  __device__ __forceinline__ void rows(const ProductDwArgs& a, const DwItem& it) { x_ahead<indexed>(a, it, ahead); }
  // 8 or 4 token DMAs: tiles of 256 n, and of the 128 or fewer that are left.
  static __device__ __forceinline__ int dmas(const ProductDwArgs& a, const DwItem& it) { return a.N - it.n0 > 128 ? 8 : 4; }
  __device__ __forceinline__ void addresses(const ProductDwArgs& a, const DwItem& it) {
    const int lane = item_thread() & 63, wave = __builtin_amdgcn_readfirstlane(item_thread() >> 6);
    x_rows(a, it, lane, wave, ahead, x);
    if (dmas(a, it) == 8) {
      rows_by_k(a.dy, a.N, it, it.n0, lane, wave, y);
    } else {
      const auto half = first_dmas<4>();
      DmaRows<4> h = half;
      rows_by_k(a.dy, a.N, it, it.n0, lane, wave, h);
      y.base = h.base;
#pragma unroll
      for (int i = 0; i < 4; ++i) y.off[i] = h.off[i];
    }
    y.step = (uint32_t)kTileK * (uint32_t)a.N * 2;
  }
  template <int kDma>
  __device__ __forceinline__ DmaRows<kDma> first_dmas() const {
    DmaRows<kDma> r{y.base, y.step, {}};
#pragma unroll
    for (int i = 0; i < kDma; ++i) r.off[i] = y.off[i];
    return r;
  }
  // The first K steps on their way, the bases at the step after them.
  __device__ __forceinline__ void start(const ProductDwArgs& a, const DwItem& it, uint8_t* lds) {
    const ElementTail tail = tail_of<indexed>(a, it.rows);
    if (dmas(a, it) == 8) {
      tile_start<8>(lds, x, y, it.rows, tail);
    } else {
      auto half = first_dmas<4>();
      tile_start<4>(lds, x, half, it.rows, tail);
      y.base = half.base;
    }
  }
};

// The finished tile.  One that lies within dw, and replaces it, is stored without a question.
template <int kDma>
__device__ __forceinline__ void store_dw_tile(const ProductDwArgs& a, int split, const DwItem& it, f32x4 (&acc)[8][kDma], bool bad) {
  const int wave = __builtin_amdgcn_readfirstlane(item_thread() >> 6);
  const int lane = item_thread() & 63, lr = lane & 15, lk = lane >> 4;
  auto store = [&](auto plain, auto wide) {
    constexpr bool kPlain = decltype(plain)::value;
#pragma unroll
    for (int j = 0; j < kDma; ++j) {
      const int n = it.n0 + (wave >> 1) * (16 * kDma) + j * 16 + lr, k = it.k0 + (wave & 1) * 128;
      const int64_t row = ((int64_t)it.expert * a.N + n) * a.K + k + 4 * lk;
#pragma unroll
      for (int i = 0; i < 8; i += 2) {
        f32x4 v[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            v[u][q] = acc_read(acc[i + u][j][q]);
            if (!kPlain && bad) v[u][q] = kNan;
          }
          if constexpr (decltype(wide)::value) continue;
          if constexpr (kPlain)
            store4<false>(a, it, split, row + (i + u) * 16, v[u]);
          else
            store_inside(a, it, split, n, k + (i + u) * 16 + 4 * lk, v[u]);
          __builtin_amdgcn_sched_barrier(0);  // block by block, or the accumulators are all read at once
        }
        if constexpr (decltype(wide)::value) {
          store_bf16<kPlain>(a, it, n, k + i * 16, lk, v);
          __builtin_amdgcn_sched_barrier(0);
        }
      }
    }
  };
  const bool inside = !bad && !a.accumulate && it.n0 + 32 * kDma <= a.N && it.k0 + 256 <= a.K;
  using std::false_type;
  using std::true_type;
  if (as_bf16(a, split))
    inside ? store(true_type{}, true_type{}) : store(false_type{}, true_type{});
  else
    inside ? store(true_type{}, false_type{}) : store(false_type{}, false_type{});
}

// An item without rows: zeros.
__device__ __forceinline__ void no_rows(const ProductDwArgs& a, int split, const DwItem& it) {
  const int tid = item_thread();
  const bool wide = as_bf16(a, split);
  for (int i = tid; i < 256 * 64; i += kThreads) {
    const int n = it.n0 + i / 64, k = it.k0 + i % 64 * 4;
    if (!wide)
      store_inside(a, it, split, n, k, f32x4{});
    else if (n < a.N && k < a.K)
      *(u32x2*)((uint16_t*)a.dw + ((int64_t)it.expert * a.N + n) * a.K + k) = u32x2{};
  }
}

// Tiles of 256 k by 32 kDma n one after another, as long as the next item has rows and is as wide.  The first is started
// by `src`, or (`running`) by the tile before it, in its ring.  Leaves the next item in `it`, started if it has rows;
// true: in the ring.
template <bool indexed, int kDma, class Find>
__device__ __forceinline__ bool dw_tiles(const ProductDwArgs& a, int split, DwItem& it, DwSource<indexed>& src, uint8_t* lds, Ring& ring,
                                         bool running, Find&& find) {
  TileStream<Bf16Mma, ByK, ByK, kDma> stream;
  if (running)
    stream.resume(lds, ring);
  else
    stream.begin(lds, ElementTail::steps(it.rows));
  uint32_t follows;
  do {
    f32x4 acc[8][kDma];
    const int nk = ElementTail::steps(it.rows);
    DwItem next;
    bool bad = false;
    auto early = [&] {
      next = find();
      if (next.rows > 0) src.rows(a, next);
    };
    auto late = [&] {
      bad = any_bad(src.x);  // every wave has asked for the rows of every step by now (and of one past the last)
      const bool fits = nk > 1 && next.rows > kTileK;
      if (fits) src.addresses(a, next);
      return Following<ElementTail>{fits ? (uint32_t)src.dmas(a, next) : 0u, ElementTail::steps(next.rows), tail_of<indexed>(a, next.rows)};
    };
    follows = stream.run(src.x, src.y, nk, tail_of<indexed>(a, it.rows), acc, early, late);
    if (follows == 0) {
      stream.end();
      if (next.rows > 0) {
        src.addresses(a, next);
        src.start(a, next, lds);
      }
    }
    store_dw_tile(a, split, it, acc, bad);
    it = next;
  } while (follows == kDma);
  ring = stream.o;
  return follows > 0;
}

// Workgroups that stay, a compute unit each; the 32 of an XCD take runs of consecutive items.
template <bool indexed>
__global__ __launch_bounds__(kThreads, 1) void dw_tile_kernel(ProductDwArgs a, int split) {
  __shared__ __attribute__((aligned(1024))) uint8_t lds[kLdsBytes];
  ExpertRows experts(a);
  const uint32_t xcd = blockIdx.x % kXcds, mine = blockIdx.x / kXcds, set = gridDim.x / kXcds;
  uint32_t n = 0;
  auto find = [&] {
    const uint32_t at = (n * kXcds + xcd) * set + (mine + 7 * n) % set;
    ++n;
    return uniform(dw_item<256>(a, experts, split, at));
  };
  DwItem it = find();
  DwSource<indexed> src;
  Ring ring{};
  bool running = false, started = false;
  while (it.expert >= 0) {
    if (it.rows <= 0) {
      no_rows(a, split, it);
      it = find();
      started = false;
      continue;
    }
    if (!started) {
      src.rows(a, it);
      src.addresses(a, it);
      src.start(a, it, lds);
    }
    started = true;  // what follows a tile is started by it
    if (src.dmas(a, it) == 8)
      running = dw_tiles<indexed, 8>(a, split, it, src, lds, ring, running, find);
    else
      running = dw_tiles<indexed, 4>(a, split, it, src, lds, ring, running, find);
  }
}

// ------------------------------------------------------------------------------------ parts

// dw from the parts, in their order: four elements a thread.
__global__ __launch_bounds__(kThreads) void dw_sum_kernel(ProductDwArgs a, int split, int64_t quads) {
  const int64_t q = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  if (q >= quads) return;
  f32x4 v = ((const f32x4*)a.parts)[q];
  for (int p = 1; p < split; ++p) v += ((const f32x4*)a.parts)[p * quads + q];
  if (a.bf16) {
    ((u32x2*)a.dw)[q] = u32x2{bf16x2_of(v[0], v[1]), bf16x2_of(v[2], v[3])};
  } else {
    f32x4* out = (f32x4*)a.dw + q;
    if (a.accumulate) v += *out;
    *out = v;
  }
}

int64_t dw_items(const DwPlan& p, const ProductDwArgs& a) {
  return (int64_t)a.experts * p.split * ((a.N + p.tile - 1) / p.tile) * ((a.K + p.tile - 1) / p.tile);
}

template <bool indexed>
hipError_t launch_dw(const DwPlan& plan, const ProductDwArgs& a, hipStream_t s) {
  const int64_t items = dw_items(plan, a);
  if (items > INT32_MAX - 2 * kStaying || (plan.tile != 256 && !launch_fits(items, kThreads))) return hipErrorInvalidConfiguration;
  if (plan.tile == 64) return launch(dw_small_kernel<indexed, 64>, dim3((uint32_t)items), dim3(kThreads), 0, s, a, plan.split);
  if (plan.tile == 128) return launch(dw_small_kernel<indexed, 128>, dim3((uint32_t)items), dim3(kThreads), 0, s, a, plan.split);
  return launch(dw_tile_kernel<indexed>, dim3((uint32_t)std::min<int64_t>((items + kXcds - 1) / kXcds * kXcds, kStaying)), dim3(kThreads), 0, s,
                a, plan.split);
}

}  // namespace

DwPlan product_dw_plan(int64_t rows, int32_t experts, int32_t K, int32_t N) {
  // What each way would take, in microseconds, from the rows an expert has on average: one tile alone, or as many as a
  // compute unit has one after another, whichever is longer; the writing of the sums; and the second launch that adds up
  // parts.  Fitted to 12441 problems (1 to 49152 rows, 1 to 128 experts, both types): the way chosen takes 1.8 % longer than
  // the best one, 13 % in one of twenty, 71 % at most.
  const double nk = std::ceil((double)rows / experts / kTileK), megabytes = (double)experts * N * K * 4e-6;
  DwPlan best{256, 1};
  double least = 1e30;
  struct Cost {
    double step_alone, alone, step, each, waste, write, start, join, second;
  };
  auto consider = [&](int tile, const Cost& c) {
    const double tiles = (double)experts * std::ceil((double)N / tile) * std::ceil((double)K / tile) / 256;
    for (int split = 1; split <= 32; split *= 2) {
      if (tile != 256 && tiles * split * 256 * kThreads > UINT32_MAX) break;  // more than one launch takes
      if (split > 1 && (nk < split || split * megabytes > 1024)) break;
      const double items = tiles * split, rounds = items + c.waste * (std::ceil(items) - items), steps = std::ceil(nk / split);
      const double cost = c.start + std::max(steps * c.step_alone + c.alone, rounds * (steps * c.step + c.each)) + megabytes * split * c.write +
                          (split > 1 ? c.second + megabytes * split * c.join : 0);
      if (cost < least) best = DwPlan{tile, split}, least = cost;
    }
  };
  consider(256, {0.505, 1.7, 1.191, 9.198, 0.599, 0.052, 4.411, 0.153, 1.497});
  consider(128, {0.658, 0.735, 0.578, 0.489, 0.492, 0.143, 4.184, 0.257, 1.455});
  consider(64, {0.349, 0, 0.227, 0.55, 0.91, 0.1, 3.2, 0.177, 2.568});
  return best;
}

hipError_t launch_product_dw_plan(const DwPlan& plan, const ProductDwArgs& a, hipStream_t s) {
  if (hipError_t e = a.index ? launch_dw<true>(plan, a, s) : launch_dw<false>(plan, a, s)) return e;
  if (plan.split == 1) return hipSuccess;
  const int64_t quads = (int64_t)a.experts * a.N * a.K / 4, blocks = (quads + kThreads - 1) / kThreads;
  if (!launch_fits(blocks, kThreads)) return hipErrorInvalidConfiguration;
  return launch(dw_sum_kernel, dim3((uint32_t)blocks), dim3(kThreads), 0, s, a, plan.split, quads);
}

}  // namespace moe
