// expert_tiles.hpp -- how the products divide the experts' rows into tiles and deal the tiles to workgroups: the
// rows of each expert come from offsets in device memory, which only the kernels see.  `Args` has the members
// offsets [experts + 1] (null: one expert), experts and rows.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "plan_types.hpp"

namespace moe {

constexpr int kThreads = 256;   // of every product kernel
constexpr int kBandRows = 1024;  // rows of the tiles that take turns on one weight tile
constexpr int kStaying = 256;    // workgroups of the whole tiles' kernel: one takes all of a compute unit's LDS
constexpr int kDeal = 32;        // consecutive items that one XCD's compute units run at a time

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
  template <class Args>
  __device__ __forceinline__ Experts(const Args& a, int e0, const Before& b) {
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
    end = b.tiles + scan_add(((uint32_t)(hi - lo) + kTile - 1) / kTile);
  }
  template <class Args>
  __device__ __forceinline__ Before after(const Args& a, int e0) const {
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
  template <class Args>
  __device__ __forceinline__ Items(const Args& a, int cols_) : cols((uint32_t)cols_) {
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
  template <class Args>
  __device__ __forceinline__ Item find(const Args& a, uint32_t xcd, uint32_t j) const {
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
  template <class Args>
  __device__ __forceinline__ Item at(const Args& a, uint32_t it) const {
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

// Row tile t of the experts' rows cut into runs of kTile.
template <int kTile, class Args>
__device__ __forceinline__ Item find_rows(const Args& a, uint32_t t) {
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

// DMA instructions per wave and K step that a tile's rows take: it computes 32, 64, 128, 192 or 256 of them.
__device__ __forceinline__ int row_dmas(int rows) { return rows <= 32 ? 1 : rows <= 64 ? 2 : rows <= 128 ? 4 : rows <= 192 ? 6 : 8; }

// ------------------------------------------------------------------------------------ host side

// Tiles of `height` rows there can be: every expert may end in a partly filled one.
inline int64_t most_tiles(int64_t rows, bool grouped, int32_t experts, int height) {
  return (rows + height - 1) / height + (grouped ? std::min<int64_t>(experts, rows) : 0);
}

constexpr int64_t kSlimTiles = 65535;  // they are the grid's second axis

inline int64_t dealt(int64_t tiles, int cols) {
  return (tiles * cols + kXcds * kDeal - 1) / (kXcds * kDeal) * (kXcds * kDeal);
}

}  // namespace moe
