// ops.hpp -- launch interface of the operators around the stage (host side).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace moe {

struct NormArgs {
  const uint16_t* x;         // [rows, H]
  const uint16_t* residual;  // [rows, H] or null
  const uint16_t* weight;    // [H]; null: rows are quantised as they are (no norm)
  uint16_t* sum_out;         // [rows, H] or null
  uint16_t* out;             // [rows, H] or null
  int8_t* out_q;             // [rows, H] or null
  float* scale;              // [rows], with out_q
  float* rstd;               // [rows] or null
  int64_t rows;
  int32_t H;
  float eps;
};

struct NormBackwardArgs {
  const uint16_t* dy;      // [rows, H]
  const uint16_t* h;       // [rows, H]
  const uint16_t* weight;  // [H]
  const float* rstd;       // [rows]
  const uint16_t* dsum;    // [rows, H] or null
  uint16_t* dx;            // [rows, H]
  float* dweight;          // [H]
  float* parts;            // [norm_backward_parts(rows, H), H]
  int64_t rows;
  int32_t H;
};

struct RestoreArgs {
  const int8_t* q;
  const float* scale;
  uint16_t* out;
  int64_t rows;
  int32_t H;
};

struct RouteArgs {
  const void* logits;      // [tokens, experts] fp32 or bf16
  const float* bias;       // [experts] or null
  int32_t* ids;            // [tokens, k] (the backward pass reads it)
  float* weights;          // [tokens, k]
  float* scores;           // [tokens, experts] or null
  const float* dweights;   // [tokens, k]
  const float* dscores;    // [tokens, experts] or null
  void* dlogits;           // [tokens, experts]
  int64_t tokens;
  int32_t experts, k, groups, top_groups, group_best;
  int32_t sigmoid, renormalise, bf16;
  float scale;
};

struct GroupArgs {
  const int32_t* ids;  // [n]
  int32_t* offsets;    // [experts + 1]
  int32_t* row_token;  // [n]
  int32_t* slot;       // [n]
  uint32_t* counts;    // [group_blocks(n, experts), experts]; not used by one workgroup
  int32_t n, k, experts;
};

struct Q8Args {
  const int8_t* x;         // [x_rows, K]
  const float* xs;         // [x_rows]
  const int32_t* index;    // [rows] or null
  const int32_t* offsets;  // [experts + 1] or null (one expert)
  const int8_t* w;         // [experts, N, K]: the product's weights, or the gate's
  const int8_t* w3;        // the up weights (gated products)
  const float* ws;         // [experts, N]
  const float* ws3;
  uint16_t* out;           // [rows, N]
  int64_t x_rows, rows;
  int32_t experts, K, N;
};

struct ProductArgs {       // out[i, n] = sum_k x[index[i], k] W[n, k]
  const uint16_t* x;       // [x_rows, K]
  const int32_t* index;    // [rows] or null
  const int32_t* offsets;  // [experts + 1] or null (one expert)
  const uint16_t* w;       // [experts, N, K]; by_k: [experts, K, N]
  uint16_t* out;           // [rows, N]
  int64_t x_rows, rows;
  int32_t experts, K, N;
};

struct ProductDwArgs {     // dw[e, n, k] = sum over rows i of e: dy[i, n] x[index[i], k]
  const uint16_t* dy;      // [rows, N]
  const uint16_t* x;       // [x_rows, K]
  const int32_t* index;    // [rows] or null
  const int32_t* offsets;  // [experts + 1] or null (one expert)
  void* dw;                // [experts, N, K]
  float* parts;            // [split, experts, N, K] where the rows are split
  int64_t x_rows, rows;
  int32_t experts, K, N;
  int32_t bf16, accumulate;
};

struct GateArgs {
  const uint16_t* gu;      // [rows, 2 F]
  const uint16_t* dact;    // [rows, F]
  uint16_t* act;           // [rows, F]
  uint16_t* dgu;           // [rows, 2 F]
  const int32_t* end;      // rows at or past *end are left alone; null: none are
  int64_t rows;
  int32_t F;
};

struct CombineBackwardArgs {
  const uint16_t* dout;  // [tokens, H]
  const uint16_t* recv;  // [recv_rows, H]
  const int32_t* slot;   // [tokens, k]
  const float* gate;     // [tokens, k]
  uint16_t* drecv;       // [recv_rows, H]
  float* dgate;          // [tokens, k] or null
  int64_t tokens, recv_rows;
  int32_t k, H;
};

// Up to kMost tensors as a kernel's argument.  Their elements are taken in chunks, numbered through.  A short list has
// a table of its own: the runtime copies a kernel's arguments at each launch.
constexpr int kTableTensors = 128, kShortTable = 32;
template <int kMost>
struct TensorTable {
  uint64_t in[kMost];     // address; the top bit marks bf16 (fp32 otherwise)
  uint64_t out[kMost];
  int64_t count[kMost];   // elements, none of them 0
  uint32_t first[kMost];  // the tensor's first chunk
  uint32_t chunk, chunks;  // elements of a chunk, a multiple of 8; chunks there are
  int32_t n;
};
static_assert(sizeof(TensorTable<kTableTensors>) <= 3840, "a kernel's arguments have 4 KiB");

// A launch has fewer than 2^32 threads; one that would need more is refused with hipErrorInvalidConfiguration.
constexpr bool launch_fits(int64_t blocks, int threads) { return blocks <= (int64_t)UINT32_MAX / threads; }

hipError_t launch_norm(const NormArgs& a, hipStream_t s);
// Partial sums of the weight's gradient: rows of [H] floats in the workspace.
int64_t norm_backward_parts(int64_t rows, int32_t H);
hipError_t launch_norm_backward(const NormBackwardArgs& a, hipStream_t s);
hipError_t launch_restore(const RestoreArgs& a, hipStream_t s);
hipError_t launch_route(const RouteArgs& a, hipStream_t s);
hipError_t launch_route_backward(const RouteArgs& a, hipStream_t s);
// Workgroups that count entries apart from each other; 0: one workgroup does the whole call.
int64_t group_blocks(int64_t n, int32_t experts);
hipError_t launch_group(const GroupArgs& a, hipStream_t s);
// Which kernel takes a product: 16 or 32 features and 16 rows at a time straight from memory (gated: 16 of each
// matrix), or tiles of 64, 128 or 256 weight rows and as many rows through LDS.
enum Q8Kind { kQ8Slim1, kQ8Slim2, kQ8Tiles64, kQ8Tiles128, kQ8Tiles256 };
Q8Kind q8_kind(int64_t rows, bool grouped, int32_t experts, int32_t K, int32_t N, bool gated);
hipError_t launch_q8_kind(Q8Kind kind, const Q8Args& a, bool gated, hipStream_t s);
hipError_t launch_q8(const Q8Args& a, bool gated, hipStream_t s);

// Which kernel takes a 16-bit product: 16 rows by 16 or 32 features straight from memory, or tiles of 64, 128 or 256
// features by as many rows through LDS, of 128 features by 64 rows, or (by_k) of 128 with a deeper ring.  by_k: W's
// columns lie in memory, not its rows.
enum ProductKind {
  kProductSlim1, kProductSlim2, kProductTiles64, kProductTiles128, kProductTiles256, kProductTiles128x64, kProductDeep128
};
ProductKind product_kind(int64_t rows, bool grouped, int32_t experts, int32_t K, int32_t N, bool by_k);
hipError_t launch_product_kind(ProductKind kind, const ProductArgs& a, bool by_k, hipStream_t s);
hipError_t launch_product(const ProductArgs& a, bool by_k, hipStream_t s);
// How the weights' gradient is computed: tiles of 64, 128 or 256 each way, an expert's rows in so many parts.
struct DwPlan {
  int tile, split;
};
DwPlan product_dw_plan(int64_t rows, int32_t experts, int32_t K, int32_t N);
hipError_t launch_product_dw_plan(const DwPlan& plan, const ProductDwArgs& a, hipStream_t s);
hipError_t launch_gate(const GateArgs& a, hipStream_t s);
hipError_t launch_gate_backward(const GateArgs& a, hipStream_t s);
// parts: a sum of each of the `blocks` workgroups.
template <int kMost>
hipError_t launch_squares(const TensorTable<kMost>& t, double* parts, int blocks, hipStream_t s);
hipError_t launch_squares_sum(const double* parts, int n, double* total, hipStream_t s);
template <int kMost>
hipError_t launch_clip(const TensorTable<kMost>& t, const double* total, float max_norm, float* norm, int blocks, hipStream_t s);
// Waves that share a choice: 1 or 4.
int combine_backward_parts(int64_t choices, int32_t H);
hipError_t launch_combine_backward_parts(int parts, const CombineBackwardArgs& a, hipStream_t s);
hipError_t launch_combine_backward(const CombineBackwardArgs& a, hipStream_t s);

}  // namespace moe
