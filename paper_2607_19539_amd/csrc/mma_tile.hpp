// mma_tile.hpp -- device code: the K loops of the matrix products, shared by the bf16 producer and the
// 8-bit products.  An operand row gives 128 bytes to each K step, whatever its type, so the two differ in
// the matrix instruction alone (Op), and in where K may end (Tail).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "plan_types.hpp"

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

// Byte offset from the operand rows' start of lane l's chunk of tile row n = first + l / 8, for rows
// of `stride` bytes of which row `row` (relative to the base) feeds tile row n: chunk c of a row is
// stored at c ^ swz(n), so the lane at slot l % 8 fetches chunk (l % 8) ^ swz(n).
__device__ __forceinline__ uint32_t dma_off(uint32_t n, uint32_t row, uint32_t stride, int lane) {
  return row * stride + (((uint32_t)(lane & 7) ^ swz(n)) << 4);
}

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

// Sub-step kk of a partial last K step: weight fragments of chunks that it does not hold become zeros.  A
// vector write of an operand needs two wait states before the matrix instruction reads it, which the
// compiler does not see to for assembly.
template <class Tail, class Frag, int kNI>
__device__ __forceinline__ void mask_chunks(const Tail& tail, int kk, int lk, Frag (&fa)[kNI]) {
  if constexpr (Tail::partial) {
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

// Moves both operands' bases to K step `next` of nk, one step on (none before the first).
template <int kDmaW, int kDmaX, class Tail>
__device__ __forceinline__ void advance_to(DmaRows<kDmaW>& w, DmaRows<kDmaX>& x, int next, int nk, const Tail& tail) {
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
template <int kDmaW, int kDmaX>
__device__ __forceinline__ void fetch_step(const DmaRows<kDmaW>& w, const DmaRows<kDmaX>& x, uint32_t lds_w, uint32_t lds_x) {
  static_for<kDmaW>([&](auto q) {
    dma16<decltype(q)::value * 1024>(w.base, w.off[decltype(q)::value], lds_w);
  });
  static_for<kDmaX>([&](auto q) { dma16<decltype(q)::value * 1024>(x.base, x.off[decltype(q)::value], lds_x); });
}

// Prologue: K steps 0 and 1 in flight.  w.base and x.base then point at the next step to fetch.  The ring has to be
// free; nothing is waited for, so the DMAs may run under what the caller does before tile_run.
template <int kNJ, class Tail>
__device__ __forceinline__ void tile_start(uint8_t* __restrict__ lds, DmaRows<kDmaPerThread>& w, DmaRows<kNJ>& x, int K,
                                           const Tail& tail) {
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
// DMA has arrived.
template <class Op, int kNJ, class Tail, class Late, class Last>
__device__ __forceinline__ void tile_run(uint8_t* __restrict__ lds, DmaRows<kDmaPerThread>& w, DmaRows<kNJ>& x, int K,
                                         const Tail& tail, typename Op::Acc (&acc)[8][kNJ], Late&& late, Last&& last) {
  typedef typename Op::Frag Frag;
  static_assert(kNJ == 4 || kNJ == 6 || kNJ == 8, "token fragments per wave");
  constexpr int kHJ = kNJ / 2;
  const int tid = item_thread(), lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wn = wave & 1, wm = wave >> 1;
  const int lr = lane & 15, lk = lane >> 4;
  const uint32_t lsw = swz(lr);  // rows of fragment bases (multiples of 16) + lr share lr's swizzle

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
  // Fragments of sub-step kk: the lane reads logical chunk 4kk + lk of its row, stored at chunk
  // (4kk + lk) ^ lsw = (lk ^ lsw) ^ 4kk: one base per operand and sub-step, the slot added, and the
  // 16-row block an immediate offset.
  const uint32_t lane_chunk = (uint32_t)lr * kRowBytes + (((uint32_t)lk ^ lsw) << 4);
  const uint32_t a_lane = (uint32_t)(wn * 128) * kRowBytes + lane_chunk;
  const uint32_t b_lane = (uint32_t)(wm * 16 * kNJ) * kRowBytes + lane_chunk;
  Frag fa[8], fb[kNJ];
  auto read_a = [&](uint32_t slot, int kk, int i) {
    fa[i] = *(const Frag*)(lds + ((a_lane ^ ((uint32_t)kk << 6)) + slot + i * 16 * kRowBytes));
  };
  auto read_b = [&](uint32_t slot, int kk, int j) {
    fb[j] = *(const Frag*)(lds + ((b_lane ^ ((uint32_t)kk << 6)) + slot + j * 16 * kRowBytes));
  };

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
template <class Op, int kNB, class Tail, class Late, class Last>
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
  const int lr = lane & 15, lk = lane >> 4;
  const uint32_t lsw = swz(lr);
  const uint32_t lane_chunk = (uint32_t)lr * kRowBytes + (((uint32_t)lk ^ lsw) << 4);
  const uint32_t a_lane = (uint32_t)((wave >> 1) * 128 + (wave & 1) * 32) * kRowBytes + lane_chunk;
  const uint32_t b_lane = (uint32_t)kBlockBytes + lane_chunk;

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
        fb[kk][j] = *(const Frag*)(lds + ((b_lane ^ ((uint32_t)kk << 6)) + st + j * 16 * kRowBytes));
#pragma unroll
      for (int i = 0; i < 4; ++i)
        fa[kk][i] = *(const Frag*)(lds + ((a_lane ^ ((uint32_t)kk << 6)) + st + ((i >> 1) * 64 + (i & 1) * 16) * kRowBytes));
    }
    if constexpr (decltype(last)::value) {
      mask_chunks(tail, 0, lk, fa[0]);
      mask_chunks(tail, 1, lk, fa[1]);
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

}  // namespace moe
