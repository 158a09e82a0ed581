// mma_tile.hpp -- device code: the K loops of the matrix products, shared by the bf16 producer, the 8-bit
// products and the bf16 products and their gradients.  An operand row gives 128 bytes to each K step, whatever its
// type, so they differ in the matrix instruction alone (Op), in how an operand lies in memory (layouts) and in where
// K may end (Tail).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "plan_types.hpp"
#include "row_parts.hpp"

namespace moe {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef int32_t i32x4 __attribute__((ext_vector_type(4)));

// Operand blocks in LDS: 256 rows x 64 k (bf16; 128 k of int8) = 32 KiB, 128 bytes per row -- one whole
// cache line of the row-major operand, so every line a K step touches is used in full (with
// 64-byte rows each line is fetched twice, and the load path then streams about 0.6x as many
// useful bytes per clock).  A K step needs a weight block and a token block; a ring of five
// blocks (all 160 KiB of LDS) keeps one and a half K steps of loads in flight.  Global
// memory is copied straight into LDS with global_load_lds_dwordx4 (no register staging).
// A DMA instruction writes 64 lanes x 16 bytes contiguously, i.e. 8 rows, so each lane
// fetches the 16-byte chunk that belongs at its slot: chunk c of row r sits at physical
// chunk c ^ swz(r).
constexpr int kRowBytes = kTileK * 2;                  // 128: a K step of 64 bf16 or 128 int8
constexpr int kBlockBytes = kTileM * kRowBytes;        // 32 KiB: one operand of one K step
constexpr int kRingBlocks = 5;
constexpr int kLdsBytes = kRingBlocks * kBlockBytes;   // 160 KiB: the whole LDS of a CU
constexpr int kRowsPerDma = 64 * 16 / kRowBytes;       // 8 rows per DMA instruction
constexpr int kDmaPerThread = kTileM / kRowsPerDma / 4;  // 8 per weight block per thread

// Chunk swizzle of the 128-byte operand rows: chunk c of row r is stored at c ^ ((r / 2) % 8).
// A fragment read (ds_read_b128) is served 16 lanes at a time; those lanes read one chunk
// column of 16 consecutive rows, and with 64 four-byte banks (256 bytes) even and odd rows
// fall in opposite bank halves, so the XOR spreads the 16 reads over all 16 bank groups.
__device__ __forceinline__ uint32_t swz(uint32_t row) { return (row >> 1) & 7u; }

// The thread id behind an empty asm statement: what an item computes from it stays in that item.
// Otherwise the compiler keeps every height's lane offsets in registers across the item loop, past
// the count that leaves the consumer's waves room beside a producer wave.
__device__ __forceinline__ int item_thread() {
  int t = threadIdx.x;
  asm volatile("" : "+v"(t));
  return t;
}

// How an operand lies in its block.  A block row is 128 bytes, a matrix instruction's fragment of a lane 16: eight
// 2-byte k of output row (or column) lane % 16, those from 8 (lane / 16) on of a 32-deep sub-step.
//
// ByRow: block row r holds the K step's k of output row r, so a fragment is one chunk.
struct ByRow {
  static constexpr bool transposed = false;
};
// ByK, of 2-byte elements whose rows in memory are k (a matrix that is multiplied from its other side): panels of
// 64 output rows, in each 64 block rows, one for each k of the step.  ds_read_b64_tr_b16 turns them round as they are
// read: 16 lanes read 4 k by 16 output rows, lane t 8 bytes of k t / 4, and get the 4 k of output row t.  The 32
// lanes of a half wave read 32 bytes of 8 block rows, k0 .. k0 + 3 and k0 + 8 .. k0 + 11; chunks are stored at
// c ^ swz_k(k), which spreads those over all 64 banks (two of the block rows fill them).
struct ByK {
  static constexpr bool transposed = true;
};
__device__ __forceinline__ uint32_t swz_k(uint32_t k) { return (k & 2u) | ((k >> 1) & 4u); }

// An accumulator's word.  As assembly: left to itself the compiler copies whole accumulators to vector registers
// ahead of their use, and spills.
__device__ __forceinline__ int acc_read(int v) {
  int r;
  asm volatile("v_accvgpr_read_b32 %0, %1" : "=v"(r) : "a"(v));
  return r;
}
__device__ __forceinline__ float acc_read(float v) {
  float r;
  asm volatile("v_accvgpr_read_b32 %0, %1" : "=v"(r) : "a"(v));
  return r;
}

// Calls f(integral_constant<int, 0>) .. f(integral_constant<int, n - 1>).
template <int n, int i = 0, class F>
__device__ __forceinline__ void static_for(F&& f) {
  if constexpr (i < n) {
    f(std::integral_constant<int, i>{});
    static_for<n, i + 1>(f);
  }
}

#define LDS_PTR(p) ((__attribute__((address_space(3))) void*)(p))

__device__ __forceinline__ uint32_t lds_addr(const void* p) {
  return (uint32_t)(uintptr_t)LDS_PTR(p);
}

// 16 bytes per lane from global memory (scalar base + 32-bit lane offset) straight into
// LDS at M0 + 16 * lane.  Issued as inline assembly so that the compiler's wait-count
// pass does not serialise LDS reads behind every in-flight DMA: the pipeline waits for
// exactly the stage it needs with an explicit vmcnt.  M0 is written just before the
// load and is not used by any compiler-generated code in the producer.
// One wait state separates the scalar write of M0 from the load that reads it: a matrix
// instruction where there is one (dma_m0 before it, dma16_at_m0 after), else an s_nop.
template <int kLdsOff>
__device__ __forceinline__ void dma_m0(uint32_t lds) {
  asm volatile("s_add_u32 m0, %0, %1" ::"s"(lds), "n"(kLdsOff) : "memory", "scc");
}
__device__ __forceinline__ void dma16_at_m0(const uint8_t* sbase, uint32_t voff) {
  asm volatile("global_load_lds_dwordx4 %0, %1" ::"v"(voff), "s"(sbase) : "memory");
}
template <int kLdsOff>
__device__ __forceinline__ void dma16(const uint8_t* sbase, uint32_t voff, uint32_t lds) {
  asm volatile("s_add_u32 m0, %0, %3\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds), "v"(voff),
               "s"(sbase), "n"(kLdsOff)
               : "memory", "scc");
}

// Waits until at most n of this wave's global loads are outstanding and all LDS reads have
// returned, then joins the workgroup barrier.  The empty asm statements keep the compiler
// from moving memory operations across the barrier; no fence is emitted, so in-flight
// LDS-DMA loads of later stages stay in flight.
template <int n>
__device__ __forceinline__ void wait_vm_and_barrier() {
  static_assert(n >= 0 && n < 64, "vmcnt range");
  // gfx9 s_waitcnt: vmcnt[3:0] in bits 3:0, vmcnt[5:4] in bits 15:14, expcnt 6:4, lgkmcnt 11:8.
  constexpr int imm = (n & 15) | ((n >> 4) << 14) | (7 << 4) | (0 << 8);
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(imm);
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// The same of this wave's loads alone, without the barrier.
template <int n>
__device__ __forceinline__ void wait_vm() {
  static_assert(n >= 0 && n < 64, "vmcnt range");
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt((n & 15) | ((n >> 4) << 14) | (7 << 4) | (0 << 8));
  asm volatile("" ::: "memory");
}

// One operand of an item as a DMA source.  Instruction i of a wave fetches 8 rows: lane l the 16 bytes
// at base + off[i], its row's (l / 8) 16-byte chunk that belongs at its slot in LDS.  The scalar base
// advances by `step` per K step, so a DMA costs two instructions beside the matrix ones: with a
// scalar address per instruction (six more scalar instructions for each) and the ring's slots taken
// as block % 5 where they were used, a K step opened with about 45 scalar instructions and no matrix
// instruction in flight.
template <int kDma>
struct DmaRows {
  const uint8_t* base;
  uint32_t step;
  uint32_t off[kDma];
};

// An operand ByK whose k are rows of a matrix that an index names, the item's from index[0] on.  Block row i of the K
// step is k, and a lane's DMAs take those from `first` on, 8 apart.  The wave holds the rows of up to sixteen K steps, a
// k a lane, and passes a step's around as it comes.  The loads behind them make the compiler wait for every DMA as
// well, which it cannot count, once in so many steps; a tile's first ones may be asked for in the tile before it.
constexpr int kIndexSteps = 16;
struct IndexAhead {
  int32_t row[kIndexSteps];
  // From K step `step` of the n entries of index; the last step starts early, as ElementTail has it, or repeats the
  // last row.
  __device__ __forceinline__ void load(const int32_t* index, int n, int step) {
    const int lane = (int)(threadIdx.x & 63);
#pragma unroll
    for (int u = 0; u < kIndexSteps; ++u) row[u] = index[row_of_step(step + u, lane, n)];
  }
  __device__ __forceinline__ void arrived() {  // waited for here: later waits for one each would wait for the DMAs between them
#pragma unroll
    for (int u = 0; u < kIndexSteps; ++u) asm volatile("" : "+v"(row[u]));
  }
};
template <int kDma>
struct IndexedRows {
  const uint8_t* base;       // at the tile's first output row
  uint32_t off[kDma];
  const int32_t* index;
  int n;                     // entries of index
  uint32_t limit, stride;    // of the matrix: rows, and bytes of one
  uint32_t chunk[2];         // the lane's chunk in even and odd DMAs
  int first;                 // block row of the lane's first DMA
  bool bad;                  // an entry outside the matrix was met (its row 0 is taken instead)
  IndexAhead ahead;
  int asked[kDma];
  // The rows of step 0 (whose entries are in `ahead`) or of the step after the last one asked for ...
  __device__ __forceinline__ void ask(int step) {
    if (step > 0) {
      if (step % kIndexSteps == 0) {
        ahead.load(index, n, step);
        ahead.arrived();
      } else {
#pragma unroll
        for (int u = 0; u + 1 < kIndexSteps; ++u) ahead.row[u] = ahead.row[u + 1];
      }
    }
    bad |= (uint32_t)ahead.row[0] >= limit;
    const int row = (uint32_t)ahead.row[0] < limit ? ahead.row[0] : 0;
#pragma unroll
    for (int q = 0; q < kDma; ++q) asked[q] = __builtin_amdgcn_ds_bpermute((first + 8 * q) * 4, row);
  }
  // ... and their addresses, when they have come.
  __device__ __forceinline__ void take() {
#pragma unroll
    for (int q = 0; q < kDma; ++q) off[q] = (uint32_t)asked[q] * stride + chunk[q & 1];
  }
};

// Byte offset from the operand rows' start of lane l's chunk of tile row n = first + l / 8, for rows
// of `stride` bytes of which row `row` (relative to the base) feeds tile row n: chunk c of a row is
// stored at c ^ swz(n), so the lane at slot l % 8 fetches chunk (l % 8) ^ swz(n).
__device__ __forceinline__ uint32_t dma_off(uint32_t n, uint32_t row, uint32_t stride, int lane) {
  return row * stride + (((uint32_t)(lane & 7) ^ swz(n)) << 4);
}

// A wave's fragments of an operand: those of the 16 output rows from d on of the operand's, of sub-step kk of the
// K step in ring slot `slot`.  `first` is the wave's first output row, a multiple of 32.
template <class Layout, class Frag>
struct Fragments;
template <class Frag>
struct Fragments<ByRow, Frag> {
  uint32_t base;
  explicit __device__ __forceinline__ Fragments(uint32_t first, int lane) {
    // The lane reads logical chunk 4kk + lk of its row, stored at chunk (4kk + lk) ^ swz = (lk ^ swz) ^ 4kk: one base
    // per operand and sub-step, the slot added, and the 16-row block an immediate offset.  (Rows of fragment bases,
    // multiples of 16, + lr share lr's swizzle.)
    const uint32_t lr = lane & 15, lk = lane >> 4;
    base = first * kRowBytes + lr * kRowBytes + ((lk ^ swz(lr)) << 4);
  }
  __device__ __forceinline__ Frag read(const uint8_t* lds, uint32_t slot, int kk, int d) const {
    return *(const Frag*)(lds + ((base ^ ((uint32_t)kk << 6)) + slot + d * kRowBytes));
  }
};
template <class Frag>
struct Fragments<ByK, Frag> {
  uint32_t base;
  explicit __device__ __forceinline__ Fragments(uint32_t first, int lane) {
    // k = 32kk + 8lk + 4h + lr / 4: its bits 1 and 3, all that swz_k takes, are the lane's alone.  The 16-row block
    // within a panel (d / 16 % 4) is two bits of the chunk, and so is that of `first`.
    const uint32_t lr = lane & 15, lk = lane >> 4, k = 8 * lk + (lr >> 2);
    const uint32_t c = swz_k(k) ^ (((first >> 4) & 3u) << 1);
    base = (first >> 6) * (64 * kRowBytes) + k * kRowBytes + ((c | ((lr & 3u) >> 1)) << 4) + ((lr & 1u) << 3);
  }
  __device__ __forceinline__ Frag read(const uint8_t* lds, uint32_t slot, int kk, int d) const {
    typedef short s16x4 __attribute__((ext_vector_type(4)));
    const uint8_t* p = lds + ((base ^ (((uint32_t)d & 48u) << 1)) + slot) + (d >> 6) * (64 * kRowBytes) + kk * (32 * kRowBytes);
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)LDS_PTR(p));
    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)LDS_PTR(p + 4 * kRowBytes));
    return __builtin_bit_cast(Frag, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
  }
};

// ---------------------------------------------------------------------------
// The matrix instruction is v_mfma_f32_16x16x32_bf16.  At these sizes the chip is limited by its
// power, and the 16x16 form (32-deep, a quarter of the accumulator traffic per product of the
// 32x32x16 form) draws less: with random operands held in registers and no memory traffic it
// sustained 2.1 PFLOP/s at 2.05 GHz against 1.85 PFLOP/s at 1.79 GHz.  With the K loop below it took
// the gate/up launch of 18160 rows (H 4096, F 14336) from 3101 to 2825 us (1.38 to 1.51 PFLOP/s).  Written as assembly with
// the accumulator tied to one AGPR quad: from the builtin the register allocator moves
// accumulators between registers inside the loop.  The loop's ends keep the distance that
// reading a result needs (mfma_drain).
// ---------------------------------------------------------------------------
struct Bf16Mma {
  typedef bf16x8 Frag;
  typedef f32x4 Acc;
  static __device__ __forceinline__ void mma(Acc& d, const Frag& a, const Frag& b) {
    asm volatile("v_mfma_f32_16x16x32_bf16 %0, %1, %2, %0" : "+a"(d) : "v"(a), "v"(b));
  }
};

// The same product left to the compiler, for kernels that the weights' reading bounds: it may move accumulators, and keeps
// the distances itself.
struct Bf16MmaBuiltin {
  typedef bf16x8 Frag;
  typedef f32x4 Acc;
  static __device__ __forceinline__ void mma(Acc& d, const Frag& a, const Frag& b) {
    d = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, d, 0, 0, 0);
  }
};

// The same shape in bytes with twice the products: 64 k of int8, summed in 32-bit integers.
struct I8Mma {
  typedef i32x4 Frag;
  typedef i32x4 Acc;
  static __device__ __forceinline__ void mma(Acc& d, const Frag& a, const Frag& b) {
    asm volatile("v_mfma_i32_16x16x64_i8 %0, %1, %2, %0" : "+a"(d) : "v"(a), "v"(b));
  }
};

// Where K ends.  WholeSteps: at a K step's end.  ChunkTail: at any 16-byte chunk.  The last K step is then
// taken from the row's last 128 bytes, `back` bytes before where it would start, and the chunks outside
// [lo, hi), which belong to the step before it (or, in a row of less than 128 bytes, to nobody: the DMA's
// offsets are clamped there), are zeroed in the weight fragments as they are used.
struct WholeSteps {  // bf16
  static constexpr bool partial = false;
  static __device__ __forceinline__ int steps(int K) { return K / kTileK; }
};
struct ChunkTail {  // int8
  static constexpr bool partial = true;
  static __device__ __forceinline__ int steps(int K) { return (K + kRowBytes - 1) / kRowBytes; }
  uint32_t back;
  int lo, hi;
  explicit __device__ __forceinline__ ChunkTail(int K) {
    const int rest = K % kRowBytes;
    back = K >= kRowBytes && rest ? (uint32_t)(kRowBytes - rest) : 0;
    lo = (int)back / 16;
    hi = K >= kRowBytes ? 8 : K / 16;
  }
};
// ElementTail: at any element of 2 bytes.  The last K step starts `back` elements early, where K is a whole number of
// chunks and fills a step, so that no row is read past its end; else the lanes past the end read something else of
// the operand.  Elements outside [lo, hi) are zeroed in both operands, since either may hold infinities there.
struct ElementTail {
  static constexpr bool partial = true;
  static __device__ __forceinline__ int steps(int K) { return steps_of(K); }
  uint32_t bytes_w, bytes_x;
  int lo, hi;
  // step_w, step_x: bytes from one k to the next of each operand.
  __device__ __forceinline__ ElementTail(int K, bool early, uint32_t step_w, uint32_t step_x) {
    const int rest = K % kTileK, back = early && K >= kTileK && rest ? kTileK - rest : 0;
    bytes_w = (uint32_t)back * step_w;
    bytes_x = (uint32_t)back * step_x;
    lo = back;
    hi = back || !rest ? kTileK : rest;
  }
  __device__ __forceinline__ uint32_t back_w() const { return bytes_w; }
  __device__ __forceinline__ uint32_t back_x() const { return bytes_x; }
};

// Sub-step kk of a partial last K step: weight fragments of chunks that it does not hold become zeros.  A
// vector write of an operand needs two wait states before the matrix instruction reads it, which the
// compiler does not see to for assembly.
template <class Tail, class Frag, int kNI>
__device__ __forceinline__ void mask_chunks(const Tail& tail, int kk, int lk, Frag (&fa)[kNI]) {
  if constexpr (std::is_same_v<Tail, ChunkTail>) {
    if (tail.lo > 0 || tail.hi < 8) {
      const int c = 4 * kk + lk;
      const bool keep = c >= tail.lo && c < tail.hi;
#pragma unroll
      for (int i = 0; i < kNI; ++i) {
        if (!keep) fa[i] = Frag{};
        asm volatile("s_nop 1" : "+v"(fa[i]));
      }
    }
  }
}

// Fragments first .. first + n - 1 of either operand in sub-step kk of an ElementTail's last K step; the other tails
// need none of it.
template <class Tail, class Frag, int kN>
__device__ __forceinline__ void mask_elements(const Tail& tail, int kk, int lk, Frag (&f)[kN], int first, int n) {
  if constexpr (std::is_same_v<Tail, ElementTail>) {
    if (tail.lo > 0 || tail.hi < kTileK) {
      typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
      u32x4_t keep;
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int k = 32 * kk + 8 * lk + 2 * q;
        keep[q] = (k >= tail.lo && k < tail.hi ? 0xFFFFu : 0u) | (k + 1 >= tail.lo && k + 1 < tail.hi ? 0xFFFF0000u : 0u);
      }
#pragma unroll
      for (int i = 0; i < kN; ++i) {
        if (i < first || i >= first + n) continue;
        f[i] = __builtin_bit_cast(Frag, __builtin_bit_cast(u32x4_t, f[i]) & keep);
        asm volatile("s_nop 1" : "+v"(f[i]));
      }
    }
  }
}

// An operand's source at K step `next`, one step on from where it was, in two parts: what has to be asked for, and
// the move itself, which starts early at the last of nk steps, where its rows do not say so themselves.
template <int kDma>
__device__ __forceinline__ void ask_step(DmaRows<kDma>&, int) {}
template <int kDma>
__device__ __forceinline__ void ask_step(IndexedRows<kDma>& r, int next) {
  r.ask(next);
}
template <int kDma>
__device__ __forceinline__ void take_step(DmaRows<kDma>& r, int next, int nk, uint32_t back) {
  if (next > 0) r.base += r.step;
  if (next == nk - 1) r.base -= back;
}
template <int kDma>
__device__ __forceinline__ void take_step(IndexedRows<kDma>& r, int, int, uint32_t) {
  r.take();
}

// Moves both operands to K step `next` of nk, one step on (none before the first).
template <class W, class X, class Tail>
__device__ __forceinline__ void advance_to(W& w, X& x, int next, int nk, const Tail& tail) {
  if constexpr (std::is_same_v<Tail, ElementTail>) {
    ask_step(w, next);
    take_step(w, next, nk, tail.back_w());
    take_step(x, next, nk, tail.back_x());
  } else {
    if (next > 0) {
      w.base += w.step;
      x.base += x.step;
    }
    if constexpr (Tail::partial) {
      if (next == nk - 1) {
        w.base -= tail.back;
        x.base -= tail.back;
      }
    }
  }
}

// An 8-pass matrix instruction's result may be read by a vector instruction 11 wait states on.  The
// compiler does not see into the assembly, so the wait is written out, and every accumulator passes
// through a statement after it: a read of one could otherwise be moved up to its last product.
template <class Acc, int kNI, int kNJ>
__device__ __forceinline__ void mfma_drain(Acc (&acc)[kNI][kNJ]) {
  asm volatile("s_nop 15" ::: "memory");
#pragma unroll
  for (int i = 0; i < kNI; ++i)
#pragma unroll
    for (int j = 0; j < kNJ; ++j) asm volatile("" : "+a"(acc[i][j]));
}

// ---------------------------------------------------------------------------
// One output tile of 256 weight rows x 32*kNJ token rows (kNJ 8, 6, 4: 256, 192 or 128 rows) by
// 2x2 waves of 128 weight rows x 16*kNJ token rows: acc[i][j] holds D[n][m] for
// n = wn*128 + i*16 + 4*(lane/16) + r, m = wm*16*kNJ + j*16 + lane%16.
// DMA instruction i of a wave fills operand-tile rows wave*64 + i*8 .. +7 of the weight tile and
// wave*8*kNJ + i*8 .. +7 of the token tile.
//
// Block b of the ring holds the weights (b even) or tokens (b odd) of K step b/2, in slot
// b % 5.  Prologue: blocks 0-3 in flight.  K step ks runs two 32-deep sub-steps, each in two
// halves: the first half multiplies all eight weight fragments by the first kNJ/2 token fragments,
// the second half by the others.  One buffer per fragment suffices: the second half's token
// fragments are read under the first half's MFMAs, and the next sub-step's first token fragments
// and each weight fragment, as its last MFMA has issued, under the second half's (64 vector
// registers of operands where two buffers would take 128).  The DMAs go out where slots are free:
// block 2ks+4 in the step's first sub-step (its slot held K step ks-1's tokens), block 2ks+5
// in its last quarter, after the barrier that ends every wave's reads of step ks.  That barrier also
// waits for step ks+1's blocks, with only block 2ks+4 allowed in flight.  The last two K steps are
// peeled so each wait count is a constant on a straight path.
// ---------------------------------------------------------------------------

// The DMAs of a K step: weights to lds_w, tokens to lds_x (this wave's parts of their blocks).
template <class W, class X>
__device__ __forceinline__ void fetch_step(const W& w, const X& x, uint32_t lds_w, uint32_t lds_x) {
  static_for<sizeof(w.off) / 4>([&](auto q) {
    dma16<decltype(q)::value * 1024>(w.base, w.off[decltype(q)::value], lds_w);
  });
  static_for<sizeof(x.off) / 4>([&](auto q) { dma16<decltype(q)::value * 1024>(x.base, x.off[decltype(q)::value], lds_x); });
}

// Prologue: K steps 0 and 1 in flight.  w.base and x.base then point at the next step to fetch.  The ring has to be
// free; nothing is waited for, so the DMAs may run under what the caller does before tile_run.
template <int kNJ, class W, class Tail>
__device__ __forceinline__ void tile_start(uint8_t* __restrict__ lds, W& w, DmaRows<kNJ>& x, int K, const Tail& tail) {
  const int wave = __builtin_amdgcn_readfirstlane(item_thread() >> 6);
  const int nk = Tail::steps(K);
  const uint32_t lds_w = lds_addr(lds) + (uint32_t)wave * kDmaPerThread * 1024;
  const uint32_t lds_x = lds_addr(lds) + (uint32_t)wave * kNJ * 1024;
  advance_to(w, x, 0, nk, tail);
  fetch_step(w, x, lds_w, lds_x + kBlockBytes);
  advance_to(w, x, 1, nk, tail);
  if (nk > 1) {
    fetch_step(w, x, lds_w + 2 * kBlockBytes, lds_x + 3 * kBlockBytes);
    advance_to(w, x, 2, nk, tail);
  }
}

// The K loop after tile_start: late() two K steps (or one) before the end, last() before the last step, when every
// DMA has arrived.  Operands ByRow, whose K ends with a step or a chunk.
template <class Op, int kNJ, class Tail, class Late, class Last>
__device__ __forceinline__ void tile_run(uint8_t* __restrict__ lds, DmaRows<kDmaPerThread>& w, DmaRows<kNJ>& x, int K,
                                         const Tail& tail, typename Op::Acc (&acc)[8][kNJ], Late&& late, Last&& last) {
  typedef typename Op::Frag Frag;
  static_assert(kNJ == 4 || kNJ == 6 || kNJ == 8, "token fragments per wave");
  static_assert(!std::is_same_v<Tail, ElementTail>, "TileStream's");
  constexpr int kHJ = kNJ / 2;
  const int tid = item_thread(), lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wn = wave & 1, wm = wave >> 1;
  const int lk = lane >> 4;

#pragma unroll
  for (int i = 0; i < 8; ++i)
#pragma unroll
    for (int j = 0; j < kNJ; ++j) acc[i][j] = typename Op::Acc{};

  const int nk = Tail::steps(K);
  const uint32_t lds_w = lds_addr(lds) + (uint32_t)wave * kDmaPerThread * 1024;
  const uint32_t lds_x = lds_addr(lds) + (uint32_t)wave * kNJ * 1024;
  // Ring slots by block: o0, o1 hold K step ks's weights and tokens, o2 and o3 step ks+1's, o4 takes
  // step ks+2's weights and o0, once read, its tokens.  They rotate by two per step.
  uint32_t o0 = 0, o1 = kBlockBytes, o2 = 2 * kBlockBytes, o3 = 3 * kBlockBytes, o4 = 4 * kBlockBytes;
  const Fragments<ByRow, Frag> a_lane((uint32_t)(wn * 128), lane);
  const Fragments<ByRow, Frag> b_lane((uint32_t)(wm * 16 * kNJ), lane);
  Frag fa[8], fb[kNJ];
  auto read_a = [&](uint32_t slot, int kk, int i) { fa[i] = a_lane.read(lds, slot, kk, i * 16); };
  auto read_b = [&](uint32_t slot, int kk, int j) { fb[j] = b_lane.read(lds, slot, kk, j * 16); };

  // Step 0 visible, its first sub-step read.
  if (nk > 1)
    wait_vm_and_barrier<kDmaPerThread + kNJ>();
  else
    wait_vm_and_barrier<0>();
#pragma unroll
  for (int j = 0; j < kHJ; ++j) read_b(o1, 0, j);
#pragma unroll
  for (int i = 0; i < 8; ++i) read_a(o0, 0, i);

  // The weight block's DMAs go out over the step's first two quarters, one per two weight fragments:
  // the address units take 16 cycles for each of the four waves' DMAs, so eight per wave in one
  // quarter (512 cycles) fill them, and any delay holds up the wave's matrix instructions.  Against
  // one quarter: the down launch of 18160 rows 1460 -> 1391 us, the gate/up launch of 48960 rows in 16
  // experts (H 2048, F 1408) 418 -> 403; over three quarters the same (1390, 401), with less lead.
  auto w_dma = [](int quarter, int i) { return quarter < 2 && i % 2 == 0 ? quarter * 4 + i / 2 : -1; };
  // First half of sub-step kk: reads its other token fragments; with kDma, block 2ks+4's DMAs.
  auto half0 = [&](auto kkc, auto dma) {
    constexpr int kk = decltype(kkc)::value;
    static_for<8 * kHJ>([&](auto p) {
      constexpr int i = decltype(p)::value / kHJ, j = decltype(p)::value % kHJ;
      constexpr int js = i & 1 ? kHJ - 1 - j : j;
      constexpr int wq = decltype(dma)::value && j == kHJ / 2 ? w_dma(2 * kk, i) : -1;
      if constexpr (wq >= 0) dma_m0<wq * 1024>(lds_w + o4);
      Op::mma(acc[i][js], fa[i], fb[js]);
      if constexpr (wq >= 0) dma16_at_m0(w.base, w.off[wq]);
      if constexpr (j == 1 && i < kHJ) read_b(o1, kk, kHJ + i);
      __builtin_amdgcn_sched_barrier(0);
    });
  };
  // Second half: with kRead, reads what the next sub-step (kk1, slots sa and sb) starts with; with
  // kDma, in the step's last quarter, block 2ks+5's DMAs.
  auto half1 = [&](uint32_t sa, uint32_t sb, auto kk1c, auto rd, auto dma) {
    constexpr int kk1 = decltype(kk1c)::value;
    static_for<8 * kHJ>([&](auto p) {
      constexpr int i = decltype(p)::value / kHJ, j = decltype(p)::value % kHJ;
      constexpr int js = kHJ + (i & 1 ? kHJ - 1 - j : j);
      constexpr bool fetch_x = decltype(dma)::value && kk1 == 0 && j == kHJ / 2 && i < kNJ;
      constexpr int wq = decltype(dma)::value && kk1 == 1 && j == kHJ / 2 ? w_dma(1, i) : -1;
      if constexpr (fetch_x) dma_m0<i * 1024>(lds_x + o0);
      if constexpr (wq >= 0) dma_m0<wq * 1024>(lds_w + o4);
      Op::mma(acc[i][js], fa[i], fb[js]);
      if constexpr (fetch_x) dma16_at_m0(x.base, x.off[i]);
      if constexpr (wq >= 0) dma16_at_m0(w.base, w.off[wq]);
      if constexpr (decltype(rd)::value) {
        if constexpr (j == 0 && i < kHJ) read_b(sb, kk1, i);
        if constexpr (j == kHJ - 1) read_a(sa, kk1, i);
      }
      __builtin_amdgcn_sched_barrier(0);
    });
  };
  // kind 0: steady step (DMAs, then wait with one block in flight); 1: next to last (no
  // DMAs, wait for everything); 2: last step (no wait, nothing to read ahead).
  int ks = 0;
  auto step = [&](auto kind) {
    constexpr int kd = decltype(kind)::value;
    using steady = std::integral_constant<bool, kd == 0>;
    using first = std::integral_constant<int, 0>;
    using second = std::integral_constant<int, 1>;
    if constexpr (kd == 2) mask_chunks(tail, 0, lk, fa);
    half0(first{}, steady{});
    half1(o0, o1, second{}, std::true_type{}, steady{});
    if constexpr (kd == 2) mask_chunks(tail, 1, lk, fa);
    half0(second{}, std::false_type{});
    if constexpr (kd < 2) wait_vm_and_barrier<kd == 0 ? kDmaPerThread : 0>();  // step ks+1 visible, step ks's slots free
    half1(o2, o3, first{}, std::integral_constant<bool, (kd < 2)>{}, steady{});
    if constexpr (kd == 0) advance_to(w, x, ks + 3, nk, tail);
    const uint32_t t0 = o0, t1 = o1;
    o0 = o2, o1 = o3, o2 = o4, o3 = t0, o4 = t1;
  };
  for (; ks + 2 < nk; ++ks) step(std::integral_constant<int, 0>{});
  late();  // two K steps (or one) before the end
  if (ks + 1 < nk) step(std::integral_constant<int, 1>{});
  last();
  step(std::integral_constant<int, 2>{});
  mfma_drain(acc);
  // All waves are done reading LDS before the epilogue or the next tile reuses it.
  wait_vm_and_barrier<0>();
}

// ---------------------------------------------------------------------------
// The same K step for tiles that follow one another without a pause: the last two steps of a tile fetch the first two of
// the next, so that the ring never runs dry and the next tile's products start right after the epilogue.  (With tile_start
// under the epilogue the ring is filled anew for each tile, by all compute units at once.)
//   begin   after tile_start: a ring of its own
//   resume  the ring as the tile before left it, which has fetched the first two steps of this one
//   run     the K loop.  early(): before the first step.  late(): two K steps before the end (or one); it gives the tile
//           that follows, whose first step w and x then are at.
//   end     where none follows
// K has two steps or more where a tile follows, and so has that one.
// ---------------------------------------------------------------------------
struct Ring {
  uint32_t o0, o1, o2, o3, o4;  // slots: this step's weights and tokens, the next one's, the free one
};

template <class Tail>
struct Following {
  uint32_t dma;  // its token DMAs, 4, 6 or 8; 0: there is none
  int nk;        // its K steps
  Tail tail;
};

// The DMA at M0, if n > kAbove.  A branch that the compiler does not see: between its own it would move accumulators.
template <int kAbove>
__device__ __forceinline__ void dma16_at_m0_if(uint32_t n, const uint8_t* sbase, uint32_t voff) {
  asm volatile("s_cmp_gt_u32 %2, %3\n\ts_cbranch_scc0 .Lno_dma%=\n\tglobal_load_lds_dwordx4 %0, %1\n.Lno_dma%=:" ::"v"(voff), "s"(sbase),
               "s"(n), "n"(kAbove)
               : "memory", "scc");
}
// Waits for every load, if n is 0.
__device__ __forceinline__ void wait_all_unless(uint32_t n) {
  asm volatile("s_cmp_lg_u32 %0, 0\n\ts_cbranch_scc1 .Lno_wait%=\n\ts_waitcnt vmcnt(0)\n.Lno_wait%=:" ::"s"(n) : "memory", "scc");
}

template <class Op, class LayoutW, class LayoutX, int kNJ>
struct TileStream {
  typedef typename Op::Frag Frag;
  static_assert(kNJ == 4 || kNJ == 6 || kNJ == 8, "token fragments per wave");
  static_assert(!LayoutX::transposed || kNJ != 6, "a wave's tokens start on half a panel or on a panel");
  static constexpr int kHJ = kNJ / 2;
  uint8_t* lds;
  Ring o;
  Frag fa[8], fb[kNJ];

  __device__ __forceinline__ void begin(uint8_t* lds_, int nk) {
    if (nk > 1)
      wait_vm_and_barrier<kDmaPerThread + kNJ>();
    else
      wait_vm_and_barrier<0>();
    resume(lds_, Ring{0, kBlockBytes, 2 * kBlockBytes, 3 * kBlockBytes, 4 * kBlockBytes});
  }
  __device__ __forceinline__ void resume(uint8_t* lds_, const Ring& ring) {
    lds = lds_;
    o = ring;
    const int lane = item_thread() & 63, wave = __builtin_amdgcn_readfirstlane(item_thread() >> 6);
    const Fragments<LayoutW, Frag> a_lane((uint32_t)((wave & 1) * 128), lane);
    const Fragments<LayoutX, Frag> b_lane((uint32_t)((wave >> 1) * 16 * kNJ), lane);
#pragma unroll
    for (int j = 0; j < kHJ; ++j) fb[j] = b_lane.read(lds, o.o1, 0, j * 16);
#pragma unroll
    for (int i = 0; i < 8; ++i) fa[i] = a_lane.read(lds, o.o0, 0, i * 16);
  }

  template <class W, class X, class Tail, class Early, class Late>
  __device__ __forceinline__ uint32_t run(W& w, X& x, int nk, const Tail& tail, typename Op::Acc (&acc)[8][kNJ], Early&& early, Late&& late) {
    const int tid = item_thread(), lane = tid & 63, lk = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const Fragments<LayoutW, Frag> a_lane((uint32_t)((wave & 1) * 128), lane);
    const Fragments<LayoutX, Frag> b_lane((uint32_t)((wave >> 1) * 16 * kNJ), lane);
    const uint32_t lds_w = lds_addr(lds) + (uint32_t)wave * kDmaPerThread * 1024;
    uint32_t lds_x = lds_addr(lds) + (uint32_t)wave * kNJ * 1024;
    uint32_t follows = kNJ;  // token DMAs of the step that is fetched
    auto read_a = [&](uint32_t slot, int kk, int i) { fa[i] = a_lane.read(lds, slot, kk, i * 16); };
    auto read_b = [&](uint32_t slot, int kk, int j) { fb[j] = b_lane.read(lds, slot, kk, j * 16); };
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int j = 0; j < kNJ; ++j) acc[i][j] = typename Op::Acc{};
    // Halves and DMAs as in tile_run.  other: the step that is fetched is the next tile's, if there is one.
    auto w_dma = [](int quarter, int i) { return quarter < 2 && i % 2 == 0 ? quarter * 4 + i / 2 : -1; };
    auto fetch_w = [&](auto q, auto other) {
      constexpr int wq = decltype(q)::value;
      if constexpr (wq >= 0) {
        if constexpr (decltype(other)::value)
          dma16_at_m0_if<0>(follows, w.base, w.off[wq]);
        else
          dma16_at_m0(w.base, w.off[wq]);
      }
    };
    auto half0 = [&](auto kkc, auto dma, auto other) {
      constexpr int kk = decltype(kkc)::value;
      static_for<8 * kHJ>([&](auto p) {
        constexpr int i = decltype(p)::value / kHJ, j = decltype(p)::value % kHJ;
        constexpr int js = i & 1 ? kHJ - 1 - j : j;
        constexpr int wq = decltype(dma)::value && j == kHJ / 2 ? w_dma(2 * kk, i) : -1;
        if constexpr (wq >= 0) dma_m0<wq * 1024>(lds_w + o.o4);
        Op::mma(acc[i][js], fa[i], fb[js]);
        fetch_w(std::integral_constant<int, wq>{}, other);
        if constexpr (j == 1 && i < kHJ) read_b(o.o1, kk, kHJ + i);
        __builtin_amdgcn_sched_barrier(0);
      });
    };
    auto half1 = [&](uint32_t sa, uint32_t sb, auto kk1c, auto other) {
      constexpr int kk1 = decltype(kk1c)::value;
      static_for<8 * kHJ>([&](auto p) {
        constexpr int i = decltype(p)::value / kHJ, j = decltype(p)::value % kHJ;
        constexpr int js = kHJ + (i & 1 ? kHJ - 1 - j : j);
        constexpr bool kOther = decltype(other)::value;
        constexpr bool fetch_x = kk1 == 0 && j == kHJ / 2 && i < (kOther ? 8 : kNJ);
        constexpr int wq = kk1 == 1 && j == kHJ / 2 ? w_dma(1, i) : -1;
        if constexpr (fetch_x) dma_m0<i * 1024>(lds_x + o.o0);
        if constexpr (wq >= 0) dma_m0<wq * 1024>(lds_w + o.o4);
        Op::mma(acc[i][js], fa[i], fb[js]);
        if constexpr (fetch_x && kOther)
          dma16_at_m0_if<i>(follows, x.base, x.off[i]);
        else if constexpr (fetch_x)
          dma16_at_m0(x.base, x.off[i]);
        fetch_w(std::integral_constant<int, wq>{}, other);
        if constexpr (j == 0 && i < kHJ) read_b(sb, kk1, i);
        if constexpr (j == kHJ - 1) read_a(sa, kk1, i);
        __builtin_amdgcn_sched_barrier(0);
      });
    };
    // last: elements past K's end are zeroed.  The operands go to step `to` of a tile of nk_to steps, where there is one:
    // the weights when their DMAs are out, in two parts under the third quarter, the tokens at the end.
    auto step = [&](auto other, auto last, int to, int nk_to, const Tail& tail_to) {
      constexpr bool kLast = decltype(last)::value;
      using first = std::integral_constant<int, 0>;
      using second = std::integral_constant<int, 1>;
      auto mask0 = [&](int kk) {
        if constexpr (kLast) {
          mask_elements(tail, kk, lk, fa, 0, 8);
          mask_elements(tail, kk, lk, fb, 0, kHJ);
        }
      };
      auto mask1 = [&](int kk) {
        if constexpr (kLast) mask_elements(tail, kk, lk, fb, kHJ, kHJ);
      };
      mask0(0);
      half0(first{}, std::true_type{}, other);
      mask1(0);
      half1(o.o0, o.o1, second{}, other);
      mask0(1);
      if (follows > 0) ask_step(w, to);
      half0(second{}, std::false_type{}, other);
      if (follows > 0) take_step(w, to, nk_to, tail_to.back_w());
      mask1(1);
      if constexpr (decltype(other)::value) wait_all_unless(follows);
      wait_vm_and_barrier<kDmaPerThread>();  // the next step visible, this one's slots free
      half1(o.o2, o.o3, first{}, other);
      if (follows > 0) take_step(x, to, nk_to, tail_to.back_x());
      o = Ring{o.o2, o.o3, o.o4, o.o0, o.o1};
    };
    early();
    for (int ks = 0; ks + 2 < nk; ++ks) step(std::false_type{}, std::false_type{}, ks + 3, nk, tail);
    const Following<Tail> f = late();
    follows = (uint32_t)__builtin_amdgcn_readfirstlane((int)f.dma);
    lds_x = lds_addr(lds) + (uint32_t)wave * follows * 1024;
    if (nk > 1) step(std::true_type{}, std::false_type{}, 1, f.nk, f.tail);
    step(std::true_type{}, std::true_type{}, 2, f.nk, f.tail);
    mfma_drain(acc);
    return follows;
  }
  // All waves are done reading LDS before what comes next writes it.
  __device__ __forceinline__ void end() const { wait_vm_and_barrier<0>(); }
};

template <class Op, int kNJ, class Tail, class Late>
__device__ __forceinline__ void tile_mma(uint8_t* __restrict__ lds, DmaRows<kDmaPerThread>& w, DmaRows<kNJ>& x, int K,
                                         const Tail& tail, typename Op::Acc (&acc)[8][kNJ], Late&& late) {
  tile_start(lds, w, x, K, tail);
  tile_run<Op>(lds, w, x, K, tail, acc, late, [] {});
}

// ---------------------------------------------------------------------------
// One output tile of 256 weight rows x 16*kNB token rows (kNB 4 or 2: at most 64 or 32 routed rows).
// Such a tile reads far more weights than it multiplies: its time is the weight stream, from HBM
// where each expert has few rows.  So the ring is four whole K steps of 32 KiB of weights and the
// few tokens beside them (three in flight, about 100 KiB per compute unit, where 8 TB/s over 256
// compute units at a loaded latency of 2-3 us asks for 60-90 KiB), one barrier per K step.  Each wave
// takes 64 weight rows and every token row, so no weight fragment is read from LDS twice:
// acc[i][j] holds n = (wave/2)*128 + (i/2)*64 + (wave%2)*32 + (i%2)*16 + 4*(lane/16) + r (a gate
// row block and its up rows in the same wave), m = j*16 + lane%16.
// ---------------------------------------------------------------------------
constexpr int kNarrowStages = 4;
template <int kNB>
constexpr uint32_t kNarrowStageBytes = kBlockBytes + 16 * kNB * kRowBytes;

// Prologue: up to three K steps in flight, nothing waited for.
template <int kNB, class Tail>
__device__ __forceinline__ void narrow_start(uint8_t* __restrict__ lds, DmaRows<kDmaPerThread>& w, DmaRows<kNB / 2>& x, int K,
                                             const Tail& tail) {
  const int wave = __builtin_amdgcn_readfirstlane(item_thread() >> 6);
  const int nk = Tail::steps(K);
  const uint32_t lds_w = lds_addr(lds) + (uint32_t)wave * kDmaPerThread * 1024;
  const uint32_t lds_x = lds_addr(lds) + kBlockBytes + (uint32_t)wave * (kNB / 2) * 1024;
  advance_to(w, x, 0, nk, tail);
  for (int ks = 0; ks < min(nk, kNarrowStages - 1); ++ks) {
    fetch_step(w, x, lds_w + ks * kNarrowStageBytes<kNB>, lds_x + ks * kNarrowStageBytes<kNB>);
    advance_to(w, x, ks + 1, nk, tail);
  }
}

// The K loop after narrow_start: late() three K steps (or fewer) before the end, last() before the last one's.
template <class Op, class LayoutW = ByRow, int kNB, class Tail, class Late, class Last>
__device__ __forceinline__ void narrow_run(uint8_t* __restrict__ lds, DmaRows<kDmaPerThread>& w, DmaRows<kNB / 2>& x, int K,
                                           const Tail& tail, typename Op::Acc (&acc)[4][kNB], Late&& late, Last&& last) {
  typedef typename Op::Frag Frag;
  static_assert(kNB == 2 || kNB == 4, "token fragments per wave");
  constexpr int kStages = kNarrowStages;
  constexpr uint32_t kStageBytes = kNarrowStageBytes<kNB>;
  static_assert(kStages * kStageBytes <= (uint32_t)kLdsBytes, "ring of K steps");
  constexpr int kDmaX = kNB / 2;
  constexpr int kDmaStage = kDmaPerThread + kDmaX;
  const int tid = item_thread(), lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lk = lane >> 4;
  const Fragments<LayoutW, Frag> a_lane((uint32_t)((wave >> 1) * 128 + (wave & 1) * 32), lane);
  const Fragments<ByRow, Frag> b_lane(0u, lane);

#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < kNB; ++j) acc[i][j] = typename Op::Acc{};

  const int nk = Tail::steps(K);
  const uint32_t lds_w = lds_addr(lds) + (uint32_t)wave * kDmaPerThread * 1024;
  const uint32_t lds_x = lds_addr(lds) + kBlockBytes + (uint32_t)wave * kDmaX * 1024;
  int loaded = min(nk, kStages - 1);                              // K steps fetched
  uint32_t st_load = (uint32_t)loaded * kStageBytes, st_use = 0;  // ring offsets of the next step to fetch and to multiply
  auto next = [](uint32_t st) { return st == (kStages - 1) * kStageBytes ? 0u : st + kStageBytes; };
  auto load = [&]() {
    fetch_step(w, x, lds_w + st_load, lds_x + st_load);
    advance_to(w, x, ++loaded, nk, tail);
    st_load = next(st_load);
  };
  auto multiply = [&](auto last) {
    const uint32_t st = st_use;
    st_use = next(st_use);
    Frag fa[2][4], fb[2][kNB];
#pragma unroll
    for (int kk = 0; kk < 2; ++kk) {
#pragma unroll
      for (int j = 0; j < kNB; ++j)
        fb[kk][j] = b_lane.read(lds, (uint32_t)kBlockBytes + st, kk, j * 16);
#pragma unroll
      for (int i = 0; i < 4; ++i) fa[kk][i] = a_lane.read(lds, st, kk, (i >> 1) * 64 + (i & 1) * 16);
    }
    if constexpr (decltype(last)::value) {
#pragma unroll
      for (int kk = 0; kk < 2; ++kk) {
        mask_chunks(tail, kk, lk, fa[kk]);
        mask_elements(tail, kk, lk, fa[kk], 0, 4);
        mask_elements(tail, kk, lk, fb[kk], 0, kNB);
      }
    }
#pragma unroll
    for (int kk = 0; kk < 2; ++kk)
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < kNB; ++j) Op::mma(acc[i][j], fa[kk][i], fb[kk][j]);
  };
  int ks = 0;
  for (; ks + kStages - 1 < nk; ++ks) {
    wait_vm_and_barrier<2 * kDmaStage>();  // step ks visible; every wave has read step ks-1
    load();
    multiply(std::false_type{});
  }
  late();  // three K steps (or fewer) before the end
  if (ks + 2 < nk) {
    wait_vm_and_barrier<2 * kDmaStage>();
    multiply(std::false_type{});
    ++ks;
  }
  if (ks + 1 < nk) {
    wait_vm_and_barrier<kDmaStage>();
    multiply(std::false_type{});
  }
  wait_vm_and_barrier<0>();
  last();
  multiply(std::true_type{});
  mfma_drain(acc);
  // All waves are done reading LDS before the epilogue or the next tile reuses it.
  wait_vm_and_barrier<0>();
}

template <class Op, int kNB, class Tail, class Late>
__device__ __forceinline__ void narrow_mma(uint8_t* __restrict__ lds, DmaRows<kDmaPerThread>& w, DmaRows<kNB / 2>& x,
                                           int K, const Tail& tail, typename Op::Acc (&acc)[4][kNB], Late&& late) {
  narrow_start<kNB>(lds, w, x, K, tail);
  narrow_run<Op>(lds, w, x, K, tail, acc, late, [] {});
}

// ---------------------------------------------------------------------------
// kW weight rows by kX rows in two by two waves, for products too small for whole tiles: a ring of kStages K steps.
// A step's second half of fragments is read under the products of the first; the barrier between the two ends
// every wave's reads of the step, whose slot is filled again at once, and the next step's first half is read under
// the products of the second.
template <class Op, int kW, int kX, int kStages = 4, class LayoutW = ByRow, class LayoutX = ByRow, class W, class Tail>
__device__ __forceinline__ void small_mma(uint8_t* __restrict__ lds, W& w, DmaRows<kX / 32>& x, int K, const Tail& tail,
                                          typename Op::Acc (&acc)[kW / 32][kX / 32]) {
  typedef typename Op::Frag Frag;
  constexpr int kNI = kW / 32, kNJ = kX / 32;
  constexpr uint32_t kStageBytes = (kW + kX) * kRowBytes;
  constexpr int kDmaStage = kNI + kNJ;
  const int tid = item_thread(), lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lk = lane >> 4;
  const Fragments<LayoutW, Frag> a_lane((uint32_t)((wave & 1) * (kW / 2)), lane);
  const Fragments<LayoutX, Frag> b_lane((uint32_t)((wave >> 1) * (kX / 2)), lane);
#pragma unroll
  for (int i = 0; i < kNI; ++i)
#pragma unroll
    for (int j = 0; j < kNJ; ++j) acc[i][j] = typename Op::Acc{};
  const int nk = Tail::steps(K);
  const uint32_t lds_w = lds_addr(lds) + (uint32_t)wave * kNI * 1024;
  const uint32_t lds_x = lds_addr(lds) + kW * kRowBytes + (uint32_t)wave * kNJ * 1024;
  int loaded = 0;
  uint32_t st_load = 0, st_use = 0;
  auto next = [](uint32_t st) { return st == (kStages - 1) * kStageBytes ? 0u : st + kStageBytes; };
  auto load = [&]() {
    fetch_step(w, x, lds_w + st_load, lds_x + st_load);
    advance_to(w, x, ++loaded, nk, tail);
    st_load = next(st_load);
  };
  Frag fa[2][kNI], fb[2][kNJ];
  auto read = [&](int kk) {
#pragma unroll
    for (int j = 0; j < kNJ; ++j) fb[kk][j] = b_lane.read(lds, kW * kRowBytes + st_use, kk, j * 16);
#pragma unroll
    for (int i = 0; i < kNI; ++i) fa[kk][i] = a_lane.read(lds, st_use, kk, i * 16);
  };
  auto multiply = [&](int kk) {
#pragma unroll
    for (int i = 0; i < kNI; ++i)
#pragma unroll
      for (int j = 0; j < kNJ; ++j) Op::mma(acc[i][j], fa[kk][i], fb[kk][j]);
  };
  // ahead: K steps behind the next one that may still be in flight; -1: there is no next step.
  auto step = [&](auto ahead, auto fetch) {
    constexpr int n = decltype(ahead)::value;
    read(1);
    if constexpr (n < 0) {
#pragma unroll
      for (int kk = 0; kk < 2; ++kk) {
        mask_chunks(tail, kk, lk, fa[kk]);
        mask_elements(tail, kk, lk, fa[kk], 0, kNI);
        mask_elements(tail, kk, lk, fb[kk], 0, kNJ);
      }
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
  // Step 0 visible, the steps after it in flight.
  static_for<kStages>([&](auto r) {
    constexpr int n = kStages - decltype(r)::value;  // steps that are on their way
    if (n == kStages ? nk >= n : nk == n) wait_vm_and_barrier<(n - 1) * kDmaStage>();
  });
  read(0);
  for (int ks = 0; ks + kStages < nk; ++ks) step(std::integral_constant<int, kStages - 2>{}, std::true_type{});
  static_for<kStages - 1>([&](auto r) {
    constexpr int n = kStages - decltype(r)::value;  // steps that are left
    if (nk >= n) step(std::integral_constant<int, n - 2>{}, false_type{});
  });
  step(std::integral_constant<int, -1>{}, false_type{});
  mfma_drain(acc);
  wait_vm_and_barrier<0>();
}

}  // namespace moe
