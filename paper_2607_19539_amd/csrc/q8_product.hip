// q8_product.hip -- gfx950 kernels of the experts' products in 8 bits.
//
//   out[i, n] = bf16( float(sum_k x[r_i, k] w[e, n, k]) * (xs[r_i] ws[e, n]) ),  or silu(g) * u of two of them
//
// v_mfma_i32_16x16x64_i8, 32-bit integer sums (exact).  The weights are the A operand, so a lane ends up with
// 4 consecutive features of one row and stores them together.
//
// Three kinds of kernel, chosen by an estimate of each one's time (q8_kind):
//  * whole tiles of 256 weight rows by up to 256 rows on the K loops of mma_tile.hpp, one workgroup a compute unit
//    that stays and starts its next tile's loads under the epilogue.  Their K steps bound them: 8192 rows by
//    14336 x 4096 take 322 us (2.99 POP/s), 8192 x 8192 x 8192 384 (2.86; the library's product takes 542).  A step
//    takes 1.5 us with random operands, whether they come from L2 or from memory, which at the clock it then runs at
//    (1.96 GHz) is 2900 cycles for 2048 of matrix instructions, and 1.04 us with zeros (4.1 POP/s): power counts, but
//    what the other third of the cycles waits for has not been taken apart.
//    A tile costs some 8 us besides its K steps, which is a quarter of the time at K 2048.
//    The last, partly filled round cuts its tiles by rows into 2, 4 or 8 for the units that would idle: 8192 rows by
//    4608 x 14336 446 -> 390 us, 2048 by 4096 x 14336 131 -> 92.
//  * tiles of 128 or 64, whose loads bound them, where even so whole tiles would leave compute units idle: 256 rows by
//    3000 x 2000 7.9 us with tiles of 64, 14.4 with whole ones; 1024 by 4096 x 4096 24.4 with tiles of 128, 28.6.
//  * 16 rows by 16 or 32 features straight from memory into registers, K divided among the waves, for a few rows of
//    each expert: bound by the reading of the weights (32 experts of 7168 x 2048, 8 rows each: 470 MB in 83 us, 5.7
//    TB/s) or, in small matrices, by its latency (one row by 4096 x 4096 7.0 us, 10.9 with tiles of 64).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <cmath>

#include "launch.hpp"
#include "mma_tile.hpp"
#include "ops.hpp"
#include "vec_device.hpp"

namespace moe {

constexpr int kThreads = 256;
constexpr int kBandRows = 1024;  // rows of the tiles that take turns on one weight tile
constexpr int kStaying = 256;    // workgroups of the whole tiles' kernel: one takes all of a compute unit's LDS
constexpr int kDeal = 32;        // consecutive items that one XCD's compute units run at a time

// A workgroup's tile: kW weight rows (features, or as many gate and up features in turn) by up to kX rows.
// Quarter q of the weight rows is gate (q even) or up (q odd) of the same features, so that a wave, which
// multiplies a half of them, holds both of a feature; and a wave fetches a quarter, of one matrix.
template <bool gated, int kW, int kX>
struct Shape {
  static constexpr int kCols = gated ? kW / 2 : kW;  // features
  // Epilogue: the finished tile goes through LDS, rows padded by 16 bytes, the scales behind it.
  static constexpr int kStride = kCols * 2 + 16;
  static constexpr int kScales = kX * kStride;
  static constexpr int kOutBytes = kScales + (kW + kX) * 4;
  static __device__ __forceinline__ int feature(int n) {
    return gated ? n / (kW / 2) * (kW / 4) + n % (kW / 4) : n;
  }
  static __device__ __forceinline__ bool up(int n) { return gated && (n / (kW / 4)) & 1; }
};

// silu(g) * u = (g / (1 + e^-g)) u, from a quarter of g, with the hardware's exponential and reciprocal, each within
// one fp32 ulp.  The exponent t = -g log2(e) is rounded, which would cost e^-g an error of |g| 2^-24; the rounding r is
// made good in the first order (e^-g (1 + r ln 2)), as a bf16 result that falls the other way may change the row's
// 8-bit scale after it.  With a quarter of 1 + e^-g, too, the reciprocal is never a subnormal, which the hardware
// would flush: it is 2^-126 or more, and 0 from t = 128 on, where e^-g is infinite in fp32.  Where t itself overflows
// r is infinite; its factor is kept near a quarter.  u comes last, as g u may overflow where silu(g) u does not.
constexpr float kGateShare = 0.25f;
__device__ __forceinline__ float silu_mul(float quarter_g, float u) {
  constexpr float kLog2e = 4 * 1.44269504f, kLog2eRest = 4 * 1.92596303e-8f, kLn2 = 0.693147181f;
  constexpr float kLow = 0.15915494f, kHigh = 0.5f;  // constants that an instruction holds
  const float t = -quarter_g * kLog2e;
  const float r = fmaf(-quarter_g, kLog2eRest, fmaf(-quarter_g, kLog2e, -t));
  const float factor = __builtin_amdgcn_fmed3f(fmaf(r, kLn2 / 4, 0.25f), kLow, kHigh);
  return quarter_g * __builtin_amdgcn_rcpf(fmaf(__builtin_amdgcn_exp2f(t), factor, 0.25f)) * u;
}

// The parts by rows that each of the last round's tiles is cut into, with `per` of them for the kDeal compute units
// of an XCD: as many as there are units for, down to 32 rows.
__host__ __device__ __forceinline__ uint32_t parts_of(uint32_t per) {
  return per * 8 <= kDeal ? 8 : per * 4 <= kDeal ? 4 : per * 2 <= kDeal ? 2 : 1;
}

struct Item {
  int expert, col, rows;  // rows: valid rows of the tile, 0: no item
  int row0;
};

// v of the lanes up to each, summed.
__device__ __forceinline__ uint32_t scan_add(uint32_t v) {
  auto from = [&](auto ctrl, auto rows) {
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, decltype(ctrl)::value, decltype(rows)::value, 0xF, false);
  };
  using std::integral_constant;
  v += from(integral_constant<int, 0x111>{}, integral_constant<int, 0xF>{});  // 1, 2, 4, 8 lanes down within 16
  v += from(integral_constant<int, 0x112>{}, integral_constant<int, 0xF>{});
  v += from(integral_constant<int, 0x114>{}, integral_constant<int, 0xF>{});
  v += from(integral_constant<int, 0x118>{}, integral_constant<int, 0xF>{});
  v += from(integral_constant<int, 0x142>{}, integral_constant<int, 0xA>{});  // lane 15 of a row to the next
  v += from(integral_constant<int, 0x143>{}, integral_constant<int, 0xC>{});  // lane 31 to the upper half
  return v;
}

// The rows [lo, hi) of 64 experts from e0 on, an expert a lane, and where the tiles of kTile rows of each end in
// the running count.  The host cannot check the caller's offsets: they are cut to the rows there are and never
// fall (`seen`: where the experts before e0 end).
struct Before {
  int seen = 0;             // where the experts before these end
  uint32_t tiles = 0;       // and how many tiles they have
};
template <int kTile>
struct Experts {
  int lo, hi;
  uint32_t end;
  Experts() = default;
  __device__ __forceinline__ Experts(const Q8Args& a, int e0, const Before& b) {
    const int seen = b.seen;
    const int lane = threadIdx.x & 63, e = e0 + lane, rows = (int)a.rows;
    const bool have = e < a.experts;
    lo = have ? a.offsets[e] : 0;
    hi = have ? a.offsets[e + 1] : 0;
    if (__any(have && (lo < seen || hi < lo || hi > rows))) {
      int m = have ? min(max(max(lo, hi), seen), rows) : seen;
#pragma unroll
      for (int d = 1; d < 64; d <<= 1) {
        const int o = __shfl_up(m, d);
        if (lane >= d) m = max(m, o);
      }
      const int start = __shfl_up(m, 1);
      lo = lane == 0 ? min(max(lo, seen), m) : max(start, min(lo, m));
      hi = m;
      if (!have) lo = hi;
    }
    end = b.tiles + scan_add((uint32_t)(hi - lo + kTile - 1) / kTile);
  }
  __device__ __forceinline__ Before after(const Q8Args& a, int e0) const {
    return Before{__builtin_amdgcn_readlane(hi, min(a.experts - e0, 64) - 1), (uint32_t)__builtin_amdgcn_readlane((int)end, 63)};
  }
};

// The items of a launch.  An expert's are bands of kBandRows rows by all columns, the tiles of a band next to
// each other; they are dealt to the XCDs (workgroups b, b + 8, ... share one) in runs of kDeal, so that the
// compute units of an XCD read the same few weight and row tiles through its L2 (as the parts of one tile do).
// Every wave finds an item by itself, 64 experts at a time, a lane each.
template <int kTile>
struct Items {
  using X = Experts<kTile>;
  X table;  // of up to 64 experts
  uint32_t total = 0, cols;
  __device__ __forceinline__ Items(const Q8Args& a, int cols_) : cols((uint32_t)cols_) {
    if (!a.offsets) {
      total = (uint32_t)((a.rows + kTile - 1) / kTile) * cols;
    } else {
      Before all;  // the tiles of all experts are counted first: the deal goes by their number
      for (int e0 = 0; e0 < a.experts; e0 += 64) {
        table = X(a, e0, all);
        all = table.after(a, e0);
      }
      total = all.tiles * cols;
    }
  }
  // Item j of XCD xcd's.  It grows with j, so that an XCD without an item j has none after it.
  __device__ __forceinline__ Item find(const Q8Args& a, uint32_t xcd, uint32_t j) const {
    const Item none{0, 0, 0, 0};
    if constexpr (kTile != 256) {
      const uint32_t run = min((uint32_t)kDeal, (total + kXcds - 1) / kXcds);
      const uint32_t it = run ? ((j / run) * kXcds + xcd) * run + j % run : 0;
      return it < total ? at(a, it) : none;
    } else {
      const uint32_t whole = total / kStaying * kStaying;
      if (j < whole / kXcds) return at(a, ((j / kDeal) * kXcds + xcd) * kDeal + j % kDeal);
      // The last, partly filled round: its tiles are cut into as many parts by rows as there are compute units for.
      const uint32_t per = (total - whole + kXcds - 1) / kXcds, in = j - whole / kXcds;
      const uint32_t parts = parts_of(per);
      const uint32_t it = whole + xcd * per + in / parts;
      if (in >= per * parts || it >= total) return none;
      Item found = at(a, it);
      const int height = kTile / (int)parts, skip = (int)(in % parts) * height;
      found.row0 += skip;
      found.rows = min(found.rows - skip, height);
      return found;
    }
  }

 private:
  __device__ __forceinline__ Item at(const Q8Args& a, uint32_t it) const {
    if (!a.offsets) return place(0, 0, (int)a.rows, total / cols, it);
    Item found{0, 0, 0, 0};
    if (a.experts <= 64) {
      pick(table, 0, Before{}, it, found);
      return found;
    }
    Before past;
    for (int e0 = 0; e0 < a.experts; e0 += 64) {
      const X x(a, e0, past);
      if (pick(x, e0, past, it, found)) return found;
      past = x.after(a, e0);
    }
    return found;
  }

  // Item q of an expert with rows [lo, hi) in `tiles` tiles.
  __device__ __forceinline__ Item place(int expert, int lo, int hi, uint32_t tiles, uint32_t q) const {
    constexpr uint32_t kBand = kBandRows / kTile;
    const uint32_t band = q / (kBand * cols), in = q % (kBand * cols);
    const uint32_t nb = min(kBand, tiles - band * kBand);
    const int row0 = lo + (int)(band * kBand + in % nb) * kTile;
    return Item{expert, (int)(in / nb), min(kTile, hi - row0), row0};
  }
  __device__ __forceinline__ bool pick(const X& x, int e0, const Before& b, uint32_t it, Item& found) const {
    const uint64_t past = __ballot(it < x.end * cols);
    if (past == 0) return false;
    const int l = __builtin_ctzll(past);
    const uint32_t first = l == 0 ? b.tiles : (uint32_t)__builtin_amdgcn_readlane((int)x.end, l - 1);
    const uint32_t tiles = (uint32_t)__builtin_amdgcn_readlane((int)x.end, l) - first;
    found = place(e0 + l, __builtin_amdgcn_readlane(x.lo, l), __builtin_amdgcn_readlane(x.hi, l), tiles, it - first * cols);
    return true;
  }
};

// The item in scalar registers: it is the same in every lane.
__device__ __forceinline__ Item uniform(const Item& it) {
  return Item{__builtin_amdgcn_readfirstlane(it.expert), __builtin_amdgcn_readfirstlane(it.col),
              __builtin_amdgcn_readfirstlane(it.rows), __builtin_amdgcn_readfirstlane(it.row0)};
}

// kW weight rows by kX rows in two by two waves, for products too small for whole tiles: a ring of four K steps.
// A step's second half of fragments is read under the products of the first; the barrier between the two ends
// every wave's reads of the step, whose slot is filled again at once, and the next step's first half is read under
// the products of the second.
template <int kW, int kX>
__device__ __forceinline__ void small_mma(uint8_t* __restrict__ lds, DmaRows<kW / 32>& w, DmaRows<kX / 32>& x, int K,
                                          const ChunkTail& tail, i32x4 (&acc)[kW / 32][kX / 32]) {
  constexpr int kStages = 4, kNI = kW / 32, kNJ = kX / 32;
  constexpr uint32_t kStageBytes = (kW + kX) * kRowBytes;
  constexpr int kDmaStage = kNI + kNJ;
  const int tid = item_thread(), lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lr = lane & 15, lk = lane >> 4;
  const uint32_t lane_chunk = (uint32_t)lr * kRowBytes + (((uint32_t)lk ^ swz(lr)) << 4);
  const uint32_t a_lane = (uint32_t)((wave & 1) * (kW / 2)) * kRowBytes + lane_chunk;
  const uint32_t b_lane = (uint32_t)(kW + (wave >> 1) * (kX / 2)) * kRowBytes + lane_chunk;
#pragma unroll
  for (int i = 0; i < kNI; ++i)
#pragma unroll
    for (int j = 0; j < kNJ; ++j) acc[i][j] = i32x4{};
  const int nk = ChunkTail::steps(K);
  const uint32_t lds_w = lds_addr(lds) + (uint32_t)wave * kNI * 1024;
  const uint32_t lds_x = lds_addr(lds) + kW * kRowBytes + (uint32_t)wave * kNJ * 1024;
  int loaded = 0;
  uint32_t st_load = 0, st_use = 0;
  auto next = [](uint32_t st) { return st == (kStages - 1) * kStageBytes ? 0u : st + kStageBytes; };
  auto load = [&]() {
    static_for<kNI>([&](auto q) {
      dma16<decltype(q)::value * 1024>(w.base, w.off[decltype(q)::value], lds_w + st_load);
    });
    static_for<kNJ>([&](auto q) {
      dma16<decltype(q)::value * 1024>(x.base, x.off[decltype(q)::value], lds_x + st_load);
    });
    advance_to(w, x, ++loaded, nk, tail);
    st_load = next(st_load);
  };
  i32x4 fa[2][kNI], fb[2][kNJ];
  auto read = [&](int kk) {
#pragma unroll
    for (int j = 0; j < kNJ; ++j) fb[kk][j] = *(const i32x4*)(lds + ((b_lane ^ ((uint32_t)kk << 6)) + st_use + j * 16 * kRowBytes));
#pragma unroll
    for (int i = 0; i < kNI; ++i) fa[kk][i] = *(const i32x4*)(lds + ((a_lane ^ ((uint32_t)kk << 6)) + st_use + i * 16 * kRowBytes));
  };
  auto multiply = [&](int kk) {
#pragma unroll
    for (int i = 0; i < kNI; ++i)
#pragma unroll
      for (int j = 0; j < kNJ; ++j) I8Mma::mma(acc[i][j], fa[kk][i], fb[kk][j]);
  };
  // ahead: K steps behind the next one that may still be in flight; -1: there is no next step.
  auto step = [&](auto ahead, auto fetch) {
    constexpr int n = decltype(ahead)::value;
    read(1);
    if constexpr (n < 0) {
      mask_chunks(tail, 0, lk, fa[0]);
      mask_chunks(tail, 1, lk, fa[1]);
    }
    multiply(0);
    if constexpr (n >= 0) {
      wait_vm_and_barrier<n * kDmaStage>();
      st_use = next(st_use);
      if constexpr (decltype(fetch)::value) load();
      read(0);
    }
    multiply(1);
  };
  using std::false_type;
  advance_to(w, x, 0, nk, tail);
  for (int ks = 0; ks < min(nk, kStages); ++ks) load();
  if (nk >= 4)
    wait_vm_and_barrier<3 * kDmaStage>();
  else if (nk == 3)
    wait_vm_and_barrier<2 * kDmaStage>();
  else if (nk == 2)
    wait_vm_and_barrier<kDmaStage>();
  else
    wait_vm_and_barrier<0>();
  read(0);
  for (int ks = 0; ks + kStages < nk; ++ks) step(std::integral_constant<int, 2>{}, std::true_type{});
  if (nk >= 4) step(std::integral_constant<int, 2>{}, false_type{});
  if (nk >= 3) step(std::integral_constant<int, 1>{}, false_type{});
  if (nk >= 2) step(std::integral_constant<int, 0>{}, false_type{});
  step(std::integral_constant<int, -1>{}, false_type{});
  mfma_drain(acc);
  wait_vm_and_barrier<0>();
}

// One tile of kW weight rows by kX rows, of which it.rows are valid.
template <bool gated, int kW, int kX>
__device__ __forceinline__ void small_item(const Q8Args& a, const Item& it, uint8_t* lds) {
  using S = Shape<gated, kW, kX>;
  constexpr int kNI = kW / 32, kNJ = kX / 32;      // fragments per wave of the weights and of the rows
  constexpr int kDmaW = kW / 32, kDmaX = kX / 32;  // DMA instructions per wave and K step
  const int tid = item_thread(), lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lr = lane & 15, lk = lane >> 4;
  const int K = a.K, N = a.N;
  auto quad_n = [&](int i) { return (wave & 1) * (kW / 2) + i * 16 + 4 * lk; };
  auto quad_m = [&](int j) { return (wave >> 1) * (kX / 2) + j * 16 + lr; };
  const int first = it.col * S::kCols;
  auto feature = [&](int n) { return min(first + S::feature(n), N - 1); };
  const uint32_t r8 = (uint32_t)lane >> 3;
  const int cmax = min(K / 16, 8) - 1;
  DmaRows<kDmaW> w;
  DmaRows<kDmaX> x;
  w.step = x.step = kRowBytes;
  const int64_t wofs = (int64_t)it.expert * N;
  {
    const int f0 = feature(wave * (kW / 4));
    w.base = (const uint8_t*)(S::up(wave * (kW / 4)) ? a.w3 : a.w) + (wofs + f0) * K;
#pragma unroll
    for (int i = 0; i < kDmaW; ++i) {
      const uint32_t n = (uint32_t)(wave * (kW / 4) + 8 * i) + r8;
      const uint32_t c = min(((uint32_t)lane & 7) ^ swz(n), (uint32_t)cmax);
      w.off[i] = (uint32_t)(feature((int)n) - f0) * (uint32_t)K + (c << 4);
    }
  }
  // A row that row_index does not name takes row 0 (any readable one) and a scale of NaN.
  auto source = [&](int m, bool& ok) {
    const int i = it.row0 + min(m, it.rows - 1);
    const int64_t r = a.index ? a.index[i] : i;
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
  float my_xs = 0.0f, my_ws = 0.0f;
  if (tid < kX) {
    bool ok;
    const int64_t r = source(tid, ok);
    my_xs = ok ? a.xs[r] : __uint_as_float(0x7FC00000u);
  }
  if (tid < kW) my_ws = (S::up(tid) ? a.ws3 : a.ws)[wofs + feature(tid)];
  // Offsets and scales are complete before the first operand DMA, which the compiler does not count.
#pragma unroll
  for (int i = 0; i < kDmaX; ++i) asm volatile("" ::"v"(x.off[i]));
  asm volatile("" ::"v"(my_xs), "v"(my_ws));

  i32x4 acc[kNI][kNJ];
  const ChunkTail tail(K);
  small_mma<kW, kX>(lds, w, x, K, tail, acc);

  float* scales = (float*)(lds + S::kScales);
  if (tid < kW) scales[tid] = my_ws;
  if (tid < kX) scales[kW + tid] = my_xs;
  __syncthreads();
  float xs[kNJ];
#pragma unroll
  for (int j = 0; j < kNJ; ++j) xs[j] = scales[kW + quad_m(j)];
#pragma unroll
  for (int i = 0; i < (gated ? kNI / 2 : kNI); ++i) {
    const int n = quad_n(i);
    f32x4 ws = *(const f32x4*)(scales + n), ws3 = {};
    if constexpr (gated) ws *= kGateShare, ws3 = *(const f32x4*)(scales + n + kW / 4);
#pragma unroll
    for (int j = 0; j < kNJ; ++j) {
      float v[4];
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        v[q] = (float)acc[i][j][q] * (xs[j] * ws[q]);
        if constexpr (gated) v[q] = silu_mul(v[q], (float)acc[i + kNI / 2][j][q] * (xs[j] * ws3[q]));
      }
      *(u32x2*)(lds + quad_m(j) * S::kStride + S::feature(n) * 2) = u32x2{bf16x2_of(v[0], v[1]), bf16x2_of(v[2], v[3])};
      __builtin_amdgcn_sched_barrier(0);  // block by block, or the accumulators are all read at once
    }
  }
  __syncthreads();
  constexpr int kLanes = S::kCols / 8;  // threads that store one row
  const int c8 = tid % kLanes;
  const int f = first + c8 * 8;
  if (f < N) {
#pragma unroll 4
    for (int p = 0; p < kX * kLanes / kThreads; ++p) {
      const int m = p * (kThreads / kLanes) + tid / kLanes;
      if (m < it.rows) *(u32x4*)(a.out + (int64_t)(it.row0 + m) * N + f) = *(const u32x4*)(lds + m * S::kStride + c8 * 16);
    }
  }
}

template <bool gated, int kW, int kX>
__global__ __launch_bounds__(kThreads, kW + kX <= 128 ? 2 : 1) void q8_small_kernel(Q8Args a, int cols) {
  constexpr int kRing = 4 * (kW + kX) * kRowBytes, kOut = Shape<gated, kW, kX>::kOutBytes;
  __shared__ __attribute__((aligned(1024))) uint8_t lds[kRing > kOut ? kRing : kOut];
  const Item it = uniform(Items<kX>(a, cols).find(a, blockIdx.x % kXcds, blockIdx.x / kXcds));
  if (it.rows <= 0) return;
  small_item<gated, kW, kX>(a, it, lds);
}

// ------------------------------------------------------------------------------------ whole tiles

// An accumulator's word.  As assembly: left to itself the compiler copies whole accumulators to vector registers
// ahead of their use, and spills.
__device__ __forceinline__ int acc_read(int v) {
  int r;
  asm volatile("v_accvgpr_read_b32 %0, %1" : "=v"(r) : "a"(v));
  return r;
}

typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));

// DMA instructions per wave and K step that a tile's rows take: it computes 32, 64, 128, 192 or 256 of them.
__device__ __forceinline__ int row_dmas(int rows) { return rows <= 32 ? 1 : rows <= 64 ? 2 : rows <= 128 ? 4 : rows <= 192 ? 6 : 8; }

// What a tile's DMAs read.
template <bool gated>
struct TileSource {
  using S = Shape<gated, 256, 256>;
  DmaRows<kDmaPerThread> w;
  DmaRows<8> x;
  // First the rows, which may have to be looked up ...
  __device__ __forceinline__ void rows(const Q8Args& a, const Item& it) {
    const int lane = item_thread() & 63, wave = __builtin_amdgcn_readfirstlane(item_thread() >> 6);
    const int dx = row_dmas(it.rows);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int n = (wave * dx + i) * kRowsPerDma + (lane >> 3), m = it.row0 + min(n, it.rows - 1);
      x.off[i] = (uint32_t)(a.index ? a.index[m] : m);
    }
  }
  // ... then the addresses.  A row that row_index does not name takes row 0 (any readable one).
  __device__ __forceinline__ void addresses(const Q8Args& a, const Item& it) {
    const int lane = item_thread() & 63, wave = __builtin_amdgcn_readfirstlane(item_thread() >> 6);
    const int K = a.K, N = a.N, dx = row_dmas(it.rows), cmax = min(K / 16, 8) - 1;
    const uint32_t r8 = (uint32_t)lane >> 3;
    auto chunk = [&](uint32_t n) { return min(((uint32_t)lane & 7) ^ swz(n), (uint32_t)cmax) << 4; };
    auto feature = [&](int n) { return min(it.col * S::kCols + S::feature(n), N - 1); };
    w.step = x.step = kRowBytes;
    const int f0 = feature(wave * 64);
    w.base = (const uint8_t*)(S::up(wave * 64) ? a.w3 : a.w) + ((int64_t)it.expert * N + f0) * K;
#pragma unroll
    for (int i = 0; i < kDmaPerThread; ++i) {
      const uint32_t n = (uint32_t)(wave * 64 + 8 * i) + r8;
      w.off[i] = (uint32_t)(feature((int)n) - f0) * (uint32_t)K + chunk(n);
    }
    const int row0 = a.index ? 0 : it.row0;
    x.base = a.x_rows > 0 ? (const uint8_t*)a.x + (int64_t)row0 * K : (const uint8_t*)a.w;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t r = x.off[i];
      x.off[i] = ((int64_t)r < a.x_rows ? (r - (uint32_t)row0) * (uint32_t)K : 0u) + chunk((uint32_t)(wave * dx + i) * kRowsPerDma + r8);
      asm volatile("" ::"v"(x.off[i]));  // complete before the first DMA, which the compiler does not count
    }
  }
  template <int kDma>
  __device__ __forceinline__ DmaRows<kDma> first_rows() const {
    DmaRows<kDma> r{x.base, x.step, {}};
#pragma unroll
    for (int i = 0; i < kDma; ++i) r.off[i] = x.off[i];
    return r;
  }
  // The first K steps on their way, the bases at the step after them.
  __device__ __forceinline__ void start(const Q8Args& a, const Item& it, uint8_t* lds) {
    const ChunkTail tail(a.K);
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

// The K loop and the epilogue of a tile of 32 kDma rows by 256 weight rows, whose first K steps `src` has started.
// Between the two the next item's are started, so that they arrive under the epilogue: it keeps to registers,
// where a staged tile would take the ring's LDS.
template <bool gated, int kDma>
__device__ __forceinline__ void tile_item(const Q8Args& a, const Item& it, const Item& next, TileSource<gated>& src, uint8_t* lds) {
  using S = Shape<gated, 256, 256>;
  constexpr bool kNarrow = kDma <= 2;              // four waves by the weight rows alone
  constexpr int kNI = kNarrow ? 4 : 8;             // weight fragments per wave
  constexpr int kNJ = kNarrow ? 2 * kDma : kDma;   // row fragments per wave
  constexpr int kQuads = gated ? kNI / 2 : kNI;    // of them outputs
  const int wave = __builtin_amdgcn_readfirstlane(item_thread() >> 6);
  const int N = a.N;
  // The lane is asked for anew in each part (item_thread), or what follows from it would stay in registers
  // through the K loop.
  auto quad_n = [&](int i) {
    return kNarrow ? (wave >> 1) * 128 + (i >> 1) * 64 + (wave & 1) * 32 + (i & 1) * 16 : (wave & 1) * 128 + i * 16;
  };
  auto quad_m = [&](int j, int lane) { return (kNarrow ? 0 : (wave >> 1) * (16 * kNJ)) + j * 16 + (lane & 15); };
  const int first = it.col * S::kCols;
  DmaRows<kDma> x = src.template first_rows<kDma>();
  i32x4 acc[kNI][kNJ];
  const ChunkTail tail(a.K);
  // The scales and the next item's rows are asked for near the loop's end, the row scales (a load that may hang on
  // another) in its last step: all are there when the loop ends, and no wait for them meets a DMA.
  f32x4_any ws[kQuads], ws3[kQuads];
  int r[kNJ];
  float xs[kNJ];
  auto late = [&] {
    const int lane = item_thread() & 63;
#pragma unroll
    for (int i = 0; i < kQuads; ++i) {
      const int64_t f = (int64_t)it.expert * N + min(first + S::feature(quad_n(i)) + 4 * (lane >> 4), N - 4);
      ws[i] = *(const f32x4_any*)(a.ws + f);
      if constexpr (gated) ws3[i] = *(const f32x4_any*)(a.ws3 + f);
    }
#pragma unroll
    for (int j = 0; j < kNJ; ++j) {
      const int m = it.row0 + min(quad_m(j, lane), it.rows - 1);
      r[j] = a.index ? a.index[m] : m;
    }
    if (next.rows > 0) src.rows(a, next);
  };
  auto last = [&] {
#pragma unroll
    for (int j = 0; j < kNJ; ++j) {
      xs[j] = __uint_as_float(0x7FC00000u);
      if (r[j] >= 0 && r[j] < a.x_rows) xs[j] = a.xs[r[j]];
    }
  };
  if constexpr (kNarrow)
    narrow_run<I8Mma>(lds, src.w, x, a.K, tail, acc, late, last);
  else
    tile_run<I8Mma>(lds, src.w, x, a.K, tail, acc, late, last);
#pragma unroll
  for (int j = 0; j < kNJ; ++j) asm volatile("" ::"v"(xs[j]));
#pragma unroll
  for (int i = 0; i < kQuads; ++i) {
    asm volatile("" ::"v"(ws[i]));
    if constexpr (gated) {
      asm volatile("" ::"v"(ws3[i]));
      ws[i] *= kGateShare;
    }
  }
  if (next.rows > 0) {
    src.addresses(a, next);
    src.start(a, next, lds);
  }
  const int lane = item_thread() & 63, lk = lane >> 4;
  // A lane has 4 consecutive features of a row in each of two fragments; the lanes 16 apart exchange quads, so that
  // each stores 8 consecutive features of one.
#pragma unroll
  for (int i = 0; i < kQuads; i += 2) {
    const int f = first + S::feature(quad_n(i)) + (lk & 1) * 16 + (lk >> 1) * 8;
#pragma unroll
    for (int j = 0; j < kNJ; ++j) {
      uint32_t h[2][2];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        float v[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          v[q] = (float)acc_read(acc[i + u][j][q]) * (xs[j] * ws[i + u][q]);
          if constexpr (gated) v[q] = silu_mul(v[q], (float)acc_read(acc[i + u + kNI / 2][j][q]) * (xs[j] * ws3[i + u][q]));
        }
        h[u][0] = bf16x2_of(v[0], v[1]);
        h[u][1] = bf16x2_of(v[2], v[3]);
      }
      const auto lo = __builtin_amdgcn_permlane16_swap(h[0][0], h[1][0], false, false);
      const auto hi = __builtin_amdgcn_permlane16_swap(h[0][1], h[1][1], false, false);
      const int m = quad_m(j, lane);
      if (m < it.rows && f < N) *(u32x4*)(a.out + (int64_t)(it.row0 + m) * N + f) = u32x4{lo[0], hi[0], lo[1], hi[1]};
      __builtin_amdgcn_sched_barrier(0);  // block by block, or the accumulators are all read at once
    }
  }
}

// Workgroups that stay: b takes item (b / 8 + 7 n) mod (workgroups of its XCD) of the n-th set that its XCD's
// workgroups take together.  (Rotating keeps a workgroup from meeting the short last tile of one expert after
// another.)
template <bool gated>
__global__ __launch_bounds__(kThreads, 1) void q8_tile_kernel(Q8Args a, int cols) {
  __shared__ __attribute__((aligned(1024))) uint8_t lds[kLdsBytes];
  const Items<256> items(a, cols);
  const uint32_t xcd = blockIdx.x % kXcds, mine = blockIdx.x / kXcds, set = gridDim.x / kXcds;
  uint32_t n = 0;
  Item it = uniform(items.find(a, xcd, mine));
  if (it.rows <= 0) return;
  TileSource<gated> src;
  src.rows(a, it);
  src.addresses(a, it);
  src.start(a, it, lds);
  while (it.rows > 0) {
    ++n;
    const Item next = uniform(items.find(a, xcd, n * set + (mine + 7 * n) % set));
    switch (row_dmas(it.rows)) {
      case 1: tile_item<gated, 1>(a, it, next, src, lds); break;
      case 2: tile_item<gated, 2>(a, it, next, src, lds); break;
      case 4: tile_item<gated, 4>(a, it, next, src, lds); break;
      case 6: tile_item<gated, 6>(a, it, next, src, lds); break;
      default: tile_item<gated, 8>(a, it, next, src, lds); break;
    }
    it = next;
  }
}

// ------------------------------------------------------------------------------------ few rows

// Row tile t of the experts' rows cut into runs of kTile.
template <int kTile>
__device__ __forceinline__ Item find_rows(const Q8Args& a, uint32_t t) {
  if (!a.offsets) return Item{0, 0, min(kTile, (int)a.rows - (int)t * kTile), (int)t * kTile};
  Before b;
  for (int e0 = 0; e0 < a.experts; e0 += 64) {
    const Experts<kTile> x(a, e0, b);
    const uint64_t past = __ballot(t < x.end);
    if (past != 0) {
      const int l = __builtin_ctzll(past);
      const uint32_t first = l == 0 ? b.tiles : (uint32_t)__builtin_amdgcn_readlane((int)x.end, l - 1);
      const int row0 = __builtin_amdgcn_readlane(x.lo, l) + (int)(t - first) * kTile;
      return Item{e0 + l, 0, min(kTile, __builtin_amdgcn_readlane(x.hi, l) - row0), row0};
    }
    b = x.after(a, e0);
  }
  return Item{0, 0, 0, 0};
}

// A tile of 16 kR rows by 16 kN features (gated: kN of each matrix): the four waves take every fourth 128 bytes
// of K each, straight from memory into registers, so nothing in the loop waits for another wave, and add their
// sums up in LDS at the end.
template <bool gated, int kN, int kR>
__global__ __launch_bounds__(kThreads) void q8_slim_kernel(Q8Args a) {
  constexpr int kM = gated ? 2 : 1;
  constexpr int kFrags = kM * kN * kR;
  constexpr int kWaves = kThreads / 64;
  __shared__ i32x4 sums[kWaves][kFrags][64];
  const Item it = uniform(find_rows<16 * kR>(a, blockIdx.y));
  if (it.rows <= 0) return;
  const int lane = threadIdx.x & 63, lr = lane & 15, lk = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int K = a.K, N = a.N, n0 = blockIdx.x * 16 * kN;
  const int64_t wofs = (int64_t)it.expert * N;
  const int8_t* wp[kM][kN];
  const int8_t* xp[kR];
#pragma unroll
  for (int m = 0; m < kM; ++m)
#pragma unroll
    for (int i = 0; i < kN; ++i) wp[m][i] = (m ? a.w3 : a.w) + (wofs + min(n0 + i * 16 + lr, N - 1)) * K + lk * 16;
#pragma unroll
  for (int j = 0; j < kR; ++j) {
    const int i = it.row0 + min(j * 16 + lr, it.rows - 1);
    const int64_t r = a.index ? a.index[i] : i;
    const bool ok = r >= 0 && r < a.x_rows;
    xp[j] = (ok ? a.x + r * K : a.w) + lk * 16;
  }
  i32x4 acc[kM][kN][kR];
#pragma unroll
  for (int m = 0; m < kM; ++m)
#pragma unroll
    for (int i = 0; i < kN; ++i)
#pragma unroll
      for (int j = 0; j < kR; ++j) acc[m][i][j] = i32x4{};
  struct Chunk {
    i32x4 w[2][kM][kN], x[2][kR];
  };
  auto load = [&](Chunk& c, int k) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
#pragma unroll
      for (int m = 0; m < kM; ++m)
#pragma unroll
        for (int i = 0; i < kN; ++i) c.w[h][m][i] = *(const i32x4*)(wp[m][i] + k + h * 64);
#pragma unroll
      for (int j = 0; j < kR; ++j) c.x[h][j] = *(const i32x4*)(xp[j] + k + h * 64);
    }
  };
  auto multiply = [&](const Chunk& c) {
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int m = 0; m < kM; ++m)
#pragma unroll
        for (int i = 0; i < kN; ++i)
#pragma unroll
          for (int j = 0; j < kR; ++j)
            acc[m][i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(c.w[h][m][i], c.x[h][j], acc[m][i][j], 0, 0, 0);
  };
  const int nfull = K / 128;
  Chunk c0, c1;
  int c = wave;
  if (c < nfull) load(c0, c * 128);
  while (c < nfull) {
    if (c + kWaves < nfull) load(c1, (c + kWaves) * 128);
    multiply(c0);
    c += kWaves;
    if (c >= nfull) break;
    if (c + kWaves < nfull) load(c0, (c + kWaves) * 128);
    multiply(c1);
    c += kWaves;
  }
  if (K % 128 && wave == nfull % kWaves) {  // the last chunks of 16 bytes
    const int k = nfull * 128;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const bool in = k + h * 64 + lk * 16 < K;
#pragma unroll
      for (int m = 0; m < kM; ++m)
#pragma unroll
        for (int i = 0; i < kN; ++i) {
          c0.w[h][m][i] = i32x4{};
          if (in) c0.w[h][m][i] = *(const i32x4*)(wp[m][i] + k + h * 64);
        }
#pragma unroll
      for (int j = 0; j < kR; ++j) {
        c0.x[h][j] = i32x4{};
        if (in) c0.x[h][j] = *(const i32x4*)(xp[j] + k + h * 64);
      }
    }
    multiply(c0);
  }
#pragma unroll
  for (int m = 0; m < kM; ++m)
#pragma unroll
    for (int i = 0; i < kN; ++i)
#pragma unroll
      for (int j = 0; j < kR; ++j) sums[wave][(i * kR + j) * kM + m][lane] = acc[m][i][j];
  __syncthreads();
#pragma unroll
  for (int f = 0; f < kN * kR; ++f) {
    if (f % kWaves != wave) continue;
    const int i = f / kR, j = f % kR;
    const int n = n0 + i * 16 + 4 * lk, m = j * 16 + lr;
    if (n >= N || m >= it.rows) continue;
    const int64_t row = it.row0 + m;
    const int64_t r = a.index ? (int64_t)a.index[row] : row;
    const float xs = r >= 0 && r < a.x_rows ? a.xs[r] : __uint_as_float(0x7FC00000u);
    float v[4];
#pragma unroll
    for (int q = 0; q < kM; ++q) {
      i32x4 s = sums[0][f * kM + q][lane];
#pragma unroll
      for (int w = 1; w < kWaves; ++w) s += sums[w][f * kM + q][lane];
      const float* ws = (q ? a.ws3 : a.ws) + wofs + n;
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const float p = (float)s[t] * (xs * (gated && !q ? ws[t] * kGateShare : ws[t]));
        v[t] = q ? silu_mul(v[t], p) : p;
      }
    }
    *(u32x2*)(a.out + row * N + n) = u32x2{bf16x2_of(v[0], v[1]), bf16x2_of(v[2], v[3])};
  }
}

// Tiles of `height` rows there can be: every expert may end in a partly filled one.
int64_t most_tiles(int64_t rows, bool grouped, int32_t experts, int height) {
  return (rows + height - 1) / height + (grouped ? std::min<int64_t>(experts, rows) : 0);
}

constexpr int64_t kSlimTiles = 65535;  // they are the grid's second axis

// Workgroups along the features of a slim kernel of 16 `n` features (gated: of each matrix).
int64_t slim_cols(int32_t N, int n) { return ((int64_t)N + 16 * n - 1) / (16 * n); }

int64_t dealt(int64_t tiles, int cols) {
  return (tiles * cols + kXcds * kDeal - 1) / (kXcds * kDeal) * (kXcds * kDeal);
}

template <bool gated, int kN>
hipError_t launch_slim(const Q8Args& a, hipStream_t s) {
  const int64_t tiles = most_tiles(a.rows, a.offsets != nullptr, a.experts, 16);
  const int64_t cols = slim_cols(a.N, kN);
  if (tiles > kSlimTiles || !launch_fits(cols, kThreads)) return hipErrorInvalidConfiguration;
  return launch(q8_slim_kernel<gated, kN, 1>, dim3((uint32_t)cols, (uint32_t)tiles), dim3(kThreads), 0, s, a);
}

template <bool gated, int kW, int kX>
hipError_t launch_tiles(const Q8Args& a, hipStream_t s) {
  const int64_t tiles = most_tiles(a.rows, a.offsets != nullptr, a.experts, kX);
  const int cols = (a.N + Shape<gated, kW, kX>::kCols - 1) / Shape<gated, kW, kX>::kCols;
  const int64_t grid = dealt(tiles, cols);
  if (kW == 256 ? grid > INT32_MAX : !launch_fits(grid, kThreads)) return hipErrorInvalidConfiguration;
  if constexpr (kW == 256)
    return launch(q8_tile_kernel<gated>, dim3((uint32_t)std::min<int64_t>(grid, kStaying)), dim3(kThreads), 0, s, a, cols);
  else
    return launch(q8_small_kernel<gated, kW, kX>, dim3((uint32_t)grid), dim3(kThreads), 0, s, a, cols);
}

Q8Kind q8_kind(int64_t rows, bool grouped, int32_t experts, int32_t K, int32_t N, bool gated) {
  // What each kernel would take, in microseconds, from the rows an expert has on average (the host does not know
  // the offsets): the rounds of tiles over 256 compute units, each so many K steps of 128 bytes and something
  // for its start and end; and the reading of every weight, at the rate in TB/s that the kernel reached where that
  // is all.  The figures are fitted to 628 measured products (1 to 49152 rows, 1 to 128 experts, both operators):
  // the kernel chosen takes 1.4 % longer than the best one, 31 % at most.
  const double nk = (K + kRowBytes - 1) / kRowBytes, features = (double)N * (gated ? 2 : 1);
  const double busy = grouped ? experts * (1.0 - std::pow(1.0 - 1.0 / experts, (double)rows)) : 1.0;
  const double per = rows / busy, megabytes = busy * features * K * 1e-6;
  auto tiles = [&](double x) { return grouped ? busy * (1.0 + std::max(0.0, (per - x / 2) / x)) : std::ceil(rows / x); };
  auto items = [&](double w, double x) { return tiles(x) * std::ceil(features / w) / 256.0; };
  auto cost = [&](double work, double rate) { return std::max(work, megabytes / rate) + 0.35 * work; };
  // A K step of a whole tile by its height: 0.41 us for 32 rows, 0.66 for 64, 0.77 for 128, 1.385 for 256.
  auto step = [](double h) {
    return h < 64 ? 0.41 + 0.25 * (h - 32) / 32 : h < 128 ? 0.66 + 0.11 * (h - 64) / 64 : 0.77 + 0.615 * (h - 128) / 128;
  };
  const double whole = items(256, 256), half = items(128, 128), quarter = items(64, 64);
  const double height = std::min(256.0, std::max(32.0, per)), rest = whole - std::floor(whole);
  double tall = std::floor(whole) * (nk * step(height) + 3.5);
  if (rest > 0) {
    const int parts = parts_of((uint32_t)std::ceil(rest * kStaying / kXcds));
    const double idle = parts == 1 ? std::min(1.0, 0.7 + 0.3 * whole) : 1.0;  // fewer at work, at a higher clock
    tall += nk * step(std::max(32.0, std::min(height, 256.0 / parts))) * idle + 5;
  }
  Q8Kind best = kQ8Tiles256;
  double least = cost(1.2 + tall, gated ? 5.5 : 4.7);
  auto consider = [&](Q8Kind kind, double c) {
    if (c < least) best = kind, least = c;
  };
  // The small tiles and the slim kernels have a workgroup for each item, and can be too many for one launch.
  auto launches = [&](int w, int x) {
    return launch_fits(dealt(most_tiles(rows, grouped, experts, x), (int)std::ceil(features / w)), kThreads);
  };
  if (launches(128, 128)) consider(kQ8Tiles128, cost(1.2 + std::ceil(half) * (nk * 0.48 + 2.8), gated ? 5.2 : 4.9));
  if (launches(64, 64)) consider(kQ8Tiles64, cost(2.4 + std::max(1.0, quarter) * (nk * 0.21 + 0.9), gated ? 6.0 : 5.1));
  if (most_tiles(rows, grouped, experts, 16) <= kSlimTiles) {
    const double slim = items(gated ? 32 : 16, 16), slim2 = items(32, 16);
    if (launch_fits(slim_cols(N, 1), kThreads)) consider(kQ8Slim1, cost(2.4 + nk * std::max(0.12, 0.13 * slim), gated ? 6.1 : 6.9));
    if (!gated && launch_fits(slim_cols(N, 2), kThreads)) consider(kQ8Slim2, cost(2.4 + nk * 0.16 * std::max(1.0, slim2), 6.9));
  }
  return best;
}

hipError_t launch_q8_kind(Q8Kind kind, const Q8Args& a, bool gated, hipStream_t s) {
  switch (kind) {
    case kQ8Slim1:
      return gated ? launch_slim<true, 1>(a, s) : launch_slim<false, 1>(a, s);
    case kQ8Slim2:  // gated products have 16 features of each matrix in the other one
      return gated ? launch_slim<true, 1>(a, s) : launch_slim<false, 2>(a, s);
    case kQ8Tiles64:
      return gated ? launch_tiles<true, 64, 64>(a, s) : launch_tiles<false, 64, 64>(a, s);
    case kQ8Tiles128:
      return gated ? launch_tiles<true, 128, 128>(a, s) : launch_tiles<false, 128, 128>(a, s);
    case kQ8Tiles256:
      return gated ? launch_tiles<true, 256, 256>(a, s) : launch_tiles<false, 256, 256>(a, s);
  }
  return hipErrorInvalidValue;
}

hipError_t launch_q8(const Q8Args& a, bool gated, hipStream_t s) {
  return launch_q8_kind(q8_kind(a.rows, a.offsets != nullptr, a.experts, a.K, a.N, gated), a, gated, s);
}

}  // namespace moe
