// ops_api.cpp -- the C ABI of the operators around the stage: argument checks and launches.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <exception>
#include <vector>

#include "../../include/moe_stage.h"
#include "errors.hpp"
#include "ops.hpp"

using namespace moe;

namespace {

constexpr int32_t kMaxHidden = 65536;
constexpr int32_t kMaxExperts = 1024;
constexpr int32_t kMaxChoices = 64;
constexpr int32_t kMaxGroups = 64;
constexpr int32_t kMaxInFeatures = 131056;  // 2^17 - 16: |sum| of products of up to 128 * 127 stays below 2^31

constexpr int32_t kMaxOutFeatures = INT32_MAX - 511;  // kernels number the features of a last tile that is not full, too

constexpr int32_t kMaxFeatures = 1 << 20;  // of the 16-bit products: 64 rows of them stay within 32 bits

bool misaligned(const void* p, uintptr_t n) { return ((uintptr_t)p & (n - 1)) != 0; }

int launched(hipError_t e, const char* who) {
  if (e == hipErrorInvalidConfiguration) return record_error(MOE_EUNSUPPORTED, who, "more rows or features than one launch takes");
  return e == hipSuccess ? MOE_OK : record_error(MOE_EHIP, who, hipGetErrorString(e));
}

// rows and hidden of the row operators; 1: nothing to do.
int check_rows(const char* who, int64_t rows, int32_t hidden) {
  if (hidden <= 0 || rows < 0) return record_error(MOE_EINVAL, who, "hidden must be positive, rows >= 0");
  if (hidden % 8 || hidden > kMaxHidden)
    return record_error(MOE_EUNSUPPORTED, who, "hidden must be a multiple of 8, <= 65536");
  if (rows > INT32_MAX) return record_error(MOE_EUNSUPPORTED, who, "rows must be below 2^31");
  return MOE_OK;
}

int check_route(const char* who, const moe_route_config_t* c, int32_t type, int64_t tokens) {
  if (!c) return record_error(MOE_EINVAL, who, "null configuration");
  if (c->experts <= 0 || c->k <= 0 || c->k > c->experts || tokens < 0)
    return record_error(MOE_EINVAL, who, "experts must be positive, 1 <= k <= experts, tokens >= 0");
  if (c->groups <= 0 || c->experts % c->groups || c->top_groups <= 0 || c->top_groups > c->groups)
    return record_error(MOE_EINVAL, who, "groups must divide experts, 1 <= top_groups <= groups");
  if (c->group_best < 1 || c->group_best > 2 || c->group_best > c->experts / c->groups)
    return record_error(MOE_EINVAL, who, "group_best must be 1 or 2 and at most a group's experts");
  if (c->score != MOE_SCORE_SOFTMAX && c->score != MOE_SCORE_SIGMOID)
    return record_error(MOE_EINVAL, who, "unknown score");
  if (c->renormalise != 0 && c->renormalise != 1) return record_error(MOE_EINVAL, who, "renormalise must be 0 or 1");
  if (type != MOE_TYPE_F32 && type != MOE_TYPE_BF16) return record_error(MOE_EINVAL, who, "unknown type of logits");
  if (c->experts > kMaxExperts || c->k > kMaxChoices || c->groups > kMaxGroups)
    return record_error(MOE_EUNSUPPORTED, who, "at most 1024 experts, 64 choices and 64 groups");
  if (tokens > INT32_MAX) return record_error(MOE_EUNSUPPORTED, who, "tokens must be below 2^31");
  return MOE_OK;
}

RouteArgs route_args(const moe_route_config_t* c, const void* logits, int32_t type, int64_t tokens) {
  RouteArgs a{};
  a.logits = logits;
  a.bf16 = type == MOE_TYPE_BF16;
  a.tokens = tokens;
  a.experts = c->experts;
  a.k = c->k;
  a.groups = c->groups;
  a.top_groups = c->top_groups;
  a.group_best = c->group_best;
  a.sigmoid = c->score == MOE_SCORE_SIGMOID;
  a.renormalise = c->renormalise;
  a.scale = c->scale;
  return a;
}

int q8(const char* who, bool gated, const Q8Args& a, void* stream) {
  if (a.experts <= 0 || a.K <= 0 || a.N <= 0 || a.rows < 0 || a.x_rows < 0)
    return record_error(MOE_EINVAL, who, "experts and features must be positive, rows >= 0");
  if (!a.offsets && a.experts != 1)
    return record_error(MOE_EINVAL, who, "more than one expert needs expert_offsets");
  if (!a.index && a.x_rows < a.rows) return record_error(MOE_EINVAL, who, "fewer rows of xq than of out");
  if (a.K % 16 || a.K > kMaxInFeatures)
    return record_error(MOE_EUNSUPPORTED, who, "in_features must be a multiple of 16, <= 131056");
  if (a.N % 8 || a.N > kMaxOutFeatures)
    return record_error(MOE_EUNSUPPORTED, who, "out_features must be a multiple of 8, <= 2^31 - 512");
  if (a.experts > kMaxExperts) return record_error(MOE_EUNSUPPORTED, who, "at most 1024 experts");
  if (a.rows > INT32_MAX || a.x_rows > INT32_MAX) return record_error(MOE_EUNSUPPORTED, who, "rows must be below 2^31");
  if (a.index && (uint64_t)a.x_rows * (uint64_t)a.K > UINT32_MAX)
    return record_error(MOE_EUNSUPPORTED, who, "rows taken through row_index must lie within 4 GiB");
  if (a.rows == 0) return MOE_OK;
  if (!a.w || !a.ws || !a.out || (gated && (!a.w3 || !a.ws3)) || (a.x_rows > 0 && (!a.x || !a.xs)))
    return record_error(MOE_EINVAL, who, "null pointer");
  if (misaligned(a.x, 16) || misaligned(a.w, 16) || misaligned(a.w3, 16) || misaligned(a.out, 16))
    return record_error(MOE_EUNSUPPORTED, who, "xq, the weights and out must be 16-byte aligned");
  if (misaligned(a.xs, 4) || misaligned(a.ws, 4) || misaligned(a.ws3, 4) || misaligned(a.index, 4) || misaligned(a.offsets, 4))
    return record_error(MOE_EUNSUPPORTED, who, "scales and indices must be 4-byte aligned");
  return launched(launch_q8(a, gated, (hipStream_t)stream), who);
}

// What the 16-bit products share; 0: the call is to go on.
int check_product(const char* who, const int32_t* offsets, int32_t experts, int64_t rows, int32_t in, int32_t out) {
  if (experts <= 0 || in <= 0 || out <= 0 || rows < 0)
    return record_error(MOE_EINVAL, who, "experts and features must be positive, rows >= 0");
  if (!offsets && experts != 1) return record_error(MOE_EINVAL, who, "more than one expert needs expert_offsets");
  if (in % 8 || in > kMaxFeatures || out % 8 || out > kMaxFeatures)
    return record_error(MOE_EUNSUPPORTED, who, "in_features and out_features must be multiples of 8, <= 2^20");
  if (experts > kMaxExperts) return record_error(MOE_EUNSUPPORTED, who, "at most 1024 experts");
  if (rows > INT32_MAX) return record_error(MOE_EUNSUPPORTED, who, "rows must be below 2^31");
  return MOE_OK;
}

int check_x(const char* who, const int32_t* index, int64_t x_rows, int64_t rows, int32_t in) {
  if (x_rows < 0) return record_error(MOE_EINVAL, who, "x_rows must not be negative");
  if (!index && x_rows < rows) return record_error(MOE_EINVAL, who, "fewer rows of x than there are rows");
  if (x_rows > INT32_MAX) return record_error(MOE_EUNSUPPORTED, who, "rows must be below 2^31");
  if (index && (uint64_t)x_rows * (uint64_t)in * 2 > UINT32_MAX)
    return record_error(MOE_EUNSUPPORTED, who, "rows taken through row_index must lie within 4 GiB");
  return MOE_OK;
}

int check_gate(const char* who, const int32_t* offsets, int32_t experts, int64_t rows, int32_t ffn) {
  if (ffn <= 0 || rows < 0 || (offsets && experts <= 0))
    return record_error(MOE_EINVAL, who, "ffn must be positive, rows >= 0, experts positive with expert_offsets");
  if (ffn % 8 || ffn > kMaxFeatures / 2) return record_error(MOE_EUNSUPPORTED, who, "ffn must be a multiple of 8, <= 2^19");
  if (rows > INT32_MAX) return record_error(MOE_EUNSUPPORTED, who, "rows must be below 2^31");
  return MOE_OK;
}

int check_tensors(const char* who, const moe_tensor_t* t, int32_t n, bool out) {
  if (n < 0 || (n > 0 && !t)) return record_error(MOE_EINVAL, who, "n must not be negative, the list not null");
  int64_t all = 0;
  for (int32_t i = 0; i < n; ++i) {
    if (t[i].count < 0) return record_error(MOE_EINVAL, who, "a tensor's count must not be negative");
    if (t[i].type != MOE_TYPE_F32 && t[i].type != MOE_TYPE_BF16) return record_error(MOE_EINVAL, who, "unknown type of tensor");
    if (t[i].reserved) return record_error(MOE_EINVAL, who, "reserved must be 0");
    if (t[i].count == 0) continue;
    if (!t[i].data || (out && !t[i].out)) return record_error(MOE_EINVAL, who, "null pointer");
    const uintptr_t size = t[i].type == MOE_TYPE_BF16 ? 2 : 4;
    if (misaligned(t[i].data, size) || (out && misaligned(t[i].out, size)))
      return record_error(MOE_EUNSUPPORTED, who, "tensors must be aligned to their elements");
    if (t[i].count > (INT64_MAX >> 4) - all) return record_error(MOE_EUNSUPPORTED, who, "too many elements");
    all += t[i].count;
  }
  return MOE_OK;
}

// Whether an out overlaps another tensor's data or out.
bool overlapping(const moe_tensor_t* t, int32_t n) {
  struct Span {
    uintptr_t from, to;
    bool out;
  };
  std::vector<Span> spans;
  spans.reserve(2 * (size_t)n);
  for (int32_t i = 0; i < n; ++i) {
    const uintptr_t bytes = (uintptr_t)t[i].count * (t[i].type == MOE_TYPE_BF16 ? 2 : 4), in = (uintptr_t)t[i].data, out = (uintptr_t)t[i].out;
    if (bytes == 0) continue;
    spans.push_back({out, out + bytes, true});
    if (in != out) spans.push_back({in, in + bytes, false});
  }
  std::sort(spans.begin(), spans.end(), [](const Span& a, const Span& b) { return a.from < b.from; });
  uintptr_t any = 0, outs = 0;  // where those so far end
  for (const Span& s : spans) {
    if (s.from < (s.out ? any : outs)) return true;
    any = std::max(any, s.to);
    if (s.out) outs = std::max(outs, s.to);
  }
  return false;
}

// The tables of a list, one after another, to f(table, workgroups).  Workgroups take a chunk at a time; a long list has
// some 32 chunks for each.
constexpr int kListBlocks = 2048;  // eight to a compute unit
template <int kMost, class F>
hipError_t for_tables(const moe_tensor_t* t, int32_t n, F&& f) {
  int64_t all = 0;
  for (int32_t i = 0; i < n; ++i) all += t[i].count;
  // At least 4096 elements, and few enough chunks for their number.
  const int64_t chunk = std::min<int64_t>((all / (32 * kListBlocks) / 4096 + 1) * 4096, 1 << 30);
  TensorTable<kMost> table;
  table.n = 0;
  table.chunks = 0;
  table.chunk = (uint32_t)chunk;
  auto flush = [&] {
    const hipError_t e = f(table, (int)std::min<uint32_t>(table.chunks, kListBlocks));
    table.n = 0;
    table.chunks = 0;
    return e;
  };
  for (int32_t i = 0; i < n; ++i) {
    if (t[i].count == 0) continue;
    if (table.n == kMost)
      if (hipError_t e = flush()) return e;
    table.in[table.n] = (uint64_t)t[i].data | (t[i].type == MOE_TYPE_BF16 ? 1ull << 63 : 0);
    table.out[table.n] = (uint64_t)t[i].out;
    table.count[table.n] = t[i].count;
    table.first[table.n++] = table.chunks;
    table.chunks += (uint32_t)((t[i].count + chunk - 1) / chunk);
  }
  return table.n ? flush() : hipSuccess;
}
template <class F>
hipError_t for_each_table(const moe_tensor_t* t, int32_t n, F&& f) {
  return n <= kShortTable ? for_tables<kShortTable>(t, n, f) : for_tables<kTableTensors>(t, n, f);
}

}  // namespace

int moe_norm(const void* x, const void* residual, const void* weight, int64_t rows, int32_t hidden, float eps,
             void* sum_out, void* out, void* out_q, float* scale, float* rstd, void* stream) {
  constexpr const char* who = "moe_norm";
  if (int rc = check_rows(who, rows, hidden)) return rc;
  if (!(eps >= 0.0f)) return record_error(MOE_EINVAL, who, "eps must not be negative");
  if (rows == 0) return MOE_OK;
  if (!sum_out && !out && !out_q && !rstd) return record_error(MOE_EINVAL, who, "no output asked for");
  if (!out_q != !scale) return record_error(MOE_EINVAL, who, "out_q and scale go together");
  if (!x || !weight) return record_error(MOE_EINVAL, who, "null pointer");
  if (misaligned(x, 16) || misaligned(residual, 16) || misaligned(weight, 16) || misaligned(sum_out, 16) ||
      misaligned(out, 16) || misaligned(out_q, 16) || misaligned(scale, 4) || misaligned(rstd, 4))
    return record_error(MOE_EUNSUPPORTED, who, "16-bit and 8-bit tensors must be 16-byte aligned");
  NormArgs a{};
  a.x = (const uint16_t*)x;
  a.residual = (const uint16_t*)residual;
  a.weight = (const uint16_t*)weight;
  a.sum_out = (uint16_t*)sum_out;
  a.out = (uint16_t*)out;
  a.out_q = (int8_t*)out_q;
  a.scale = scale;
  a.rstd = rstd;
  a.rows = rows;
  a.H = hidden;
  a.eps = eps;
  return launched(launch_norm(a, (hipStream_t)stream), who);
}

int64_t moe_norm_backward_workspace(int64_t rows, int32_t hidden) {
  if (rows <= 0 || hidden <= 0 || hidden > kMaxHidden) return 0;
  const int64_t parts = norm_backward_parts(rows, hidden);
  return parts > 1 ? parts * hidden * (int64_t)sizeof(float) : 0;
}

int moe_norm_backward(const void* dy, const void* h, const void* weight, const float* rstd, const void* dsum,
                      int64_t rows, int32_t hidden, void* dx, float* dweight, void* workspace,
                      int64_t workspace_bytes, void* stream) {
  constexpr const char* who = "moe_norm_backward";
  if (int rc = check_rows(who, rows, hidden)) return rc;
  if (!dweight || (rows > 0 && (!dy || !h || !weight || !rstd || !dx)))
    return record_error(MOE_EINVAL, who, "null pointer");
  if (misaligned(dy, 16) || misaligned(h, 16) || misaligned(weight, 16) || misaligned(dsum, 16) || misaligned(dx, 16) ||
      misaligned(workspace, 16) || misaligned(rstd, 4) || misaligned(dweight, 4))
    return record_error(MOE_EUNSUPPORTED, who, "16-bit tensors and the workspace must be 16-byte aligned");
  const int64_t need = moe_norm_backward_workspace(rows, hidden);
  if (need > 0 && (!workspace || workspace_bytes < need))
    return record_error(MOE_ECAPACITY, who, "the workspace is smaller than moe_norm_backward_workspace says");
  NormBackwardArgs a{};
  a.dy = (const uint16_t*)dy;
  a.h = (const uint16_t*)h;
  a.weight = (const uint16_t*)weight;
  a.rstd = rstd;
  a.dsum = (const uint16_t*)dsum;
  a.dx = (uint16_t*)dx;
  a.dweight = dweight;
  a.parts = (float*)workspace;
  a.rows = rows;
  a.H = hidden;
  return launched(launch_norm_backward(a, (hipStream_t)stream), who);
}

int moe_q8_rows(const void* x, int64_t rows, int32_t hidden, void* q, float* scale, void* stream) {
  constexpr const char* who = "moe_q8_rows";
  if (int rc = check_rows(who, rows, hidden)) return rc;
  if (rows == 0) return MOE_OK;
  if (!x || !q || !scale) return record_error(MOE_EINVAL, who, "null pointer");
  if (misaligned(x, 16) || misaligned(q, 16) || misaligned(scale, 4))
    return record_error(MOE_EUNSUPPORTED, who, "x and q must be 16-byte aligned");
  NormArgs a{};
  a.x = (const uint16_t*)x;
  a.out_q = (int8_t*)q;
  a.scale = scale;
  a.rows = rows;
  a.H = hidden;
  return launched(launch_norm(a, (hipStream_t)stream), who);
}

int moe_q8_restore(const void* q, const float* scale, int64_t rows, int32_t hidden, void* out, void* stream) {
  constexpr const char* who = "moe_q8_restore";
  if (int rc = check_rows(who, rows, hidden)) return rc;
  if (rows == 0) return MOE_OK;
  if (!q || !scale || !out) return record_error(MOE_EINVAL, who, "null pointer");
  if (misaligned(q, 16) || misaligned(out, 16) || misaligned(scale, 4))
    return record_error(MOE_EUNSUPPORTED, who, "q and out must be 16-byte aligned");
  const RestoreArgs a{(const int8_t*)q, scale, (uint16_t*)out, rows, hidden};
  return launched(launch_restore(a, (hipStream_t)stream), who);
}

int moe_route(const moe_route_config_t* cfg, const void* logits, int32_t logits_type, const float* bias, int64_t tokens,
              int32_t* ids, float* weights, float* scores, void* stream) {
  constexpr const char* who = "moe_route";
  if (int rc = check_route(who, cfg, logits_type, tokens)) return rc;
  if (tokens == 0) return MOE_OK;
  if (!logits || !ids || !weights) return record_error(MOE_EINVAL, who, "null pointer");
  if (misaligned(logits, logits_type == MOE_TYPE_BF16 ? 2 : 4) || misaligned(bias, 4) || misaligned(ids, 4) ||
      misaligned(weights, 4) || misaligned(scores, 4))
    return record_error(MOE_EUNSUPPORTED, who, "tensors must be aligned to their elements");
  RouteArgs a = route_args(cfg, logits, logits_type, tokens);
  a.bias = bias;
  a.ids = ids;
  a.weights = weights;
  a.scores = scores;
  return launched(launch_route(a, (hipStream_t)stream), who);
}

int moe_route_backward(const moe_route_config_t* cfg, const void* logits, int32_t logits_type, const int32_t* ids,
                       const float* dweights, const float* dscores, int64_t tokens, void* dlogits, void* stream) {
  constexpr const char* who = "moe_route_backward";
  if (int rc = check_route(who, cfg, logits_type, tokens)) return rc;
  if (tokens == 0) return MOE_OK;
  if (!logits || !ids || !dweights || !dlogits) return record_error(MOE_EINVAL, who, "null pointer");
  const uintptr_t align = logits_type == MOE_TYPE_BF16 ? 2 : 4;
  if (misaligned(logits, align) || misaligned(dlogits, align) || misaligned(ids, 4) || misaligned(dweights, 4) ||
      misaligned(dscores, 4))
    return record_error(MOE_EUNSUPPORTED, who, "tensors must be aligned to their elements");
  RouteArgs a = route_args(cfg, logits, logits_type, tokens);
  a.ids = const_cast<int32_t*>(ids);
  a.dweights = dweights;
  a.dscores = dscores;
  a.dlogits = dlogits;
  return launched(launch_route_backward(a, (hipStream_t)stream), who);
}

int64_t moe_group_workspace(int64_t entries, int32_t experts) {
  if (entries <= 0 || entries > INT32_MAX || experts <= 0) return 0;
  return group_blocks(entries, experts) * experts * (int64_t)sizeof(uint32_t);
}

int moe_group(const int32_t* ids, int64_t tokens, int32_t k, int32_t experts, int32_t* expert_offsets,
              int32_t* row_token, int32_t* slot, void* workspace, int64_t workspace_bytes, void* stream) {
  constexpr const char* who = "moe_group";
  if (tokens < 0 || k <= 0 || experts <= 0)
    return record_error(MOE_EINVAL, who, "k and experts must be positive, tokens >= 0");
  if (experts > kMaxExperts) return record_error(MOE_EUNSUPPORTED, who, "at most 1024 experts");
  if (tokens > INT32_MAX / k) return record_error(MOE_EUNSUPPORTED, who, "tokens * k must be below 2^31");
  if (!expert_offsets || (tokens > 0 && (!ids || !row_token || !slot)))
    return record_error(MOE_EINVAL, who, "null pointer");
  if (misaligned(ids, 4) || misaligned(expert_offsets, 4) || misaligned(row_token, 4) || misaligned(slot, 4) ||
      misaligned(workspace, 4))
    return record_error(MOE_EUNSUPPORTED, who, "arrays must be 4-byte aligned");
  const int64_t need = moe_group_workspace(tokens * k, experts);
  if (need > 0 && (!workspace || workspace_bytes < need))
    return record_error(MOE_ECAPACITY, who, "the workspace is smaller than moe_group_workspace says");
  const GroupArgs a{ids, expert_offsets, row_token, slot, need > 0 ? (uint32_t*)workspace : nullptr, (int32_t)(tokens * k),
                    k, experts};
  return launched(launch_group(a, (hipStream_t)stream), who);
}

int moe_q8_product(const void* xq, const float* x_scale, int64_t x_rows, const int32_t* row_index,
                   const int32_t* expert_offsets, int32_t experts, const void* w, const float* w_scale, int64_t rows,
                   int32_t in_features, int32_t out_features, void* out, void* stream) {
  const Q8Args a{(const int8_t*)xq, x_scale, row_index, expert_offsets, (const int8_t*)w, nullptr, w_scale, nullptr,
                 (uint16_t*)out, x_rows, rows, experts, in_features, out_features};
  return q8("moe_q8_product", false, a, stream);
}

int moe_q8_gated(const void* xq, const float* x_scale, int64_t x_rows, const int32_t* row_index,
                 const int32_t* expert_offsets, int32_t experts, const void* w1, const float* w1_scale, const void* w3,
                 const float* w3_scale, int64_t rows, int32_t in_features, int32_t out_features, void* out,
                 void* stream) {
  const Q8Args a{(const int8_t*)xq, x_scale, row_index, expert_offsets, (const int8_t*)w1, (const int8_t*)w3, w1_scale,
                 w3_scale, (uint16_t*)out, x_rows, rows, experts, in_features, out_features};
  return q8("moe_q8_gated", true, a, stream);
}

int moe_product(const void* x, int64_t x_rows, const int32_t* row_index, const int32_t* expert_offsets, int32_t experts,
                const void* w, int64_t rows, int32_t in_features, int32_t out_features, void* out, void* stream) {
  constexpr const char* who = "moe_product";
  if (int rc = check_product(who, expert_offsets, experts, rows, in_features, out_features)) return rc;
  if (int rc = check_x(who, row_index, x_rows, rows, in_features)) return rc;
  if (rows == 0) return MOE_OK;
  if (!w || !out || (x_rows > 0 && !x)) return record_error(MOE_EINVAL, who, "null pointer");
  if (misaligned(x, 16) || misaligned(w, 16) || misaligned(out, 16) || misaligned(row_index, 4) || misaligned(expert_offsets, 4))
    return record_error(MOE_EUNSUPPORTED, who, "x, w and out must be 16-byte aligned, indices 4-byte");
  const ProductArgs a{(const uint16_t*)x, row_index, expert_offsets, (const uint16_t*)w, (uint16_t*)out, x_rows, rows,
                      experts, in_features, out_features};
  return launched(launch_product(a, false, (hipStream_t)stream), who);
}

int moe_product_dx(const void* dy, const int32_t* expert_offsets, int32_t experts, const void* w, int64_t rows,
                   int32_t in_features, int32_t out_features, void* dx, void* stream) {
  constexpr const char* who = "moe_product_dx";
  if (int rc = check_product(who, expert_offsets, experts, rows, in_features, out_features)) return rc;
  if (rows == 0) return MOE_OK;
  if (!dy || !w || !dx) return record_error(MOE_EINVAL, who, "null pointer");
  if (misaligned(dy, 16) || misaligned(w, 16) || misaligned(dx, 16) || misaligned(expert_offsets, 4))
    return record_error(MOE_EUNSUPPORTED, who, "dy, w and dx must be 16-byte aligned, offsets 4-byte");
  const ProductArgs a{(const uint16_t*)dy, nullptr, expert_offsets, (const uint16_t*)w, (uint16_t*)dx, rows, rows,
                      experts, out_features, in_features};
  return launched(launch_product(a, true, (hipStream_t)stream), who);
}

int64_t moe_product_dw_workspace(int64_t rows, int32_t experts, int32_t in_features, int32_t out_features) {
  if (rows <= 0 || experts <= 0 || experts > kMaxExperts || in_features <= 0 || in_features > kMaxFeatures || out_features <= 0 ||
      out_features > kMaxFeatures)
    return 0;
  const DwPlan plan = product_dw_plan(rows, experts, in_features, out_features);
  return plan.split > 1 ? (int64_t)plan.split * experts * in_features * out_features * (int64_t)sizeof(float) : 0;
}

int moe_product_dw(const void* dy, const void* x, int64_t x_rows, const int32_t* row_index, const int32_t* expert_offsets,
                   int32_t experts, int64_t rows, int32_t in_features, int32_t out_features, void* dw, int32_t dw_type,
                   int32_t accumulate, void* workspace, int64_t workspace_bytes, void* stream) {
  constexpr const char* who = "moe_product_dw";
  if (int rc = check_product(who, expert_offsets, experts, rows, in_features, out_features)) return rc;
  if (int rc = check_x(who, row_index, x_rows, rows, in_features)) return rc;
  if (dw_type != MOE_TYPE_F32 && dw_type != MOE_TYPE_BF16) return record_error(MOE_EINVAL, who, "unknown type of dw");
  if (accumulate != 0 && accumulate != 1) return record_error(MOE_EINVAL, who, "accumulate must be 0 or 1");
  if (accumulate && dw_type != MOE_TYPE_F32) return record_error(MOE_EUNSUPPORTED, who, "sums are added to an fp32 dw only");
  if (!dw || (rows > 0 && (!dy || (x_rows > 0 && !x)))) return record_error(MOE_EINVAL, who, "null pointer");
  if (misaligned(dy, 16) || misaligned(x, 16) || misaligned(dw, 16) || misaligned(workspace, 16) || misaligned(row_index, 4) ||
      misaligned(expert_offsets, 4))
    return record_error(MOE_EUNSUPPORTED, who, "dy, x, dw and the workspace must be 16-byte aligned, indices 4-byte");
  const int64_t need = moe_product_dw_workspace(rows, experts, in_features, out_features);
  if (need > 0 && (!workspace || workspace_bytes < need))
    return record_error(MOE_ECAPACITY, who, "the workspace is smaller than moe_product_dw_workspace says");
  if (rows == 0 && accumulate) return MOE_OK;
  const ProductDwArgs a{(const uint16_t*)dy, (const uint16_t*)x, row_index, expert_offsets, dw, (float*)workspace, x_rows, rows,
                        experts, in_features, out_features, dw_type == MOE_TYPE_BF16, accumulate};
  const DwPlan plan = rows > 0 ? product_dw_plan(rows, experts, in_features, out_features) : DwPlan{256, 1};
  return launched(launch_product_dw_plan(plan, a, (hipStream_t)stream), who);
}

int moe_gate(const void* gu, const int32_t* expert_offsets, int32_t experts, int64_t rows, int32_t ffn, void* act,
             void* stream) {
  constexpr const char* who = "moe_gate";
  if (int rc = check_gate(who, expert_offsets, experts, rows, ffn)) return rc;
  if (rows == 0) return MOE_OK;
  if (!gu || !act) return record_error(MOE_EINVAL, who, "null pointer");
  if (misaligned(gu, 16) || misaligned(act, 16) || misaligned(expert_offsets, 4))
    return record_error(MOE_EUNSUPPORTED, who, "16-bit tensors must be 16-byte aligned, offsets 4-byte");
  GateArgs a{};
  a.gu = (const uint16_t*)gu;
  a.act = (uint16_t*)act;
  a.end = expert_offsets ? expert_offsets + experts : nullptr;
  a.rows = rows;
  a.F = ffn;
  return launched(launch_gate(a, (hipStream_t)stream), who);
}

int moe_gate_backward(const void* gu, const void* dact, const int32_t* expert_offsets, int32_t experts, int64_t rows,
                      int32_t ffn, void* dgu, void* act, void* stream) {
  constexpr const char* who = "moe_gate_backward";
  if (int rc = check_gate(who, expert_offsets, experts, rows, ffn)) return rc;
  if (rows == 0) return MOE_OK;
  if (!gu || !dact || !dgu) return record_error(MOE_EINVAL, who, "null pointer");
  if (misaligned(gu, 16) || misaligned(dact, 16) || misaligned(dgu, 16) || misaligned(act, 16) || misaligned(expert_offsets, 4))
    return record_error(MOE_EUNSUPPORTED, who, "16-bit tensors must be 16-byte aligned, offsets 4-byte");
  GateArgs a{};
  a.gu = (const uint16_t*)gu;
  a.dact = (const uint16_t*)dact;
  a.act = (uint16_t*)act;
  a.dgu = (uint16_t*)dgu;
  a.end = expert_offsets ? expert_offsets + experts : nullptr;
  a.rows = rows;
  a.F = ffn;
  return launched(launch_gate_backward(a, (hipStream_t)stream), who);
}

int moe_combine_backward(const void* dout, const void* recv, int64_t recv_rows, int32_t hidden, const int32_t* slot,
                         const float* gate, int64_t tokens, int32_t k, void* drecv, float* dgate, void* stream) {
  constexpr const char* who = "moe_combine_backward";
  if (int rc = check_rows(who, tokens, hidden)) return rc;
  if (k <= 0 || recv_rows < 0) return record_error(MOE_EINVAL, who, "k must be positive, recv_rows >= 0");
  if (k > kMaxChoices) return record_error(MOE_EUNSUPPORTED, who, "at most 64 choices");
  if (recv_rows > INT32_MAX) return record_error(MOE_EUNSUPPORTED, who, "rows must be below 2^31");
  if (!drecv && !dgate) return record_error(MOE_EINVAL, who, "no output asked for");
  if (tokens == 0) return MOE_OK;
  if (!dout || !slot || !gate || (recv_rows > 0 && !recv)) return record_error(MOE_EINVAL, who, "null pointer");
  if (misaligned(dout, 16) || misaligned(recv, 16) || misaligned(drecv, 16) || misaligned(slot, 4) || misaligned(gate, 4) ||
      misaligned(dgate, 4))
    return record_error(MOE_EUNSUPPORTED, who, "16-bit tensors must be 16-byte aligned, the others 4-byte");
  const CombineBackwardArgs a{(const uint16_t*)dout, (const uint16_t*)recv, slot, gate, (uint16_t*)drecv, dgate, tokens, recv_rows,
                              k, hidden};
  return launched(launch_combine_backward(a, (hipStream_t)stream), who);
}

int64_t moe_squares_workspace(const moe_tensor_t* tensors, int32_t n) {
  if (n <= 0 || !tensors) return 0;
  int64_t held = 0;
  for (int32_t i = 0; i < n; ++i) held += tensors[i].count > 0;
  // A sum of every workgroup of every table.
  return (held + kTableTensors - 1) / kTableTensors * kListBlocks * (int64_t)sizeof(double);
}

int moe_squares(const moe_tensor_t* tensors, int32_t n, double* total, void* workspace, int64_t workspace_bytes,
                void* stream) {
  constexpr const char* who = "moe_squares";
  if (int rc = check_tensors(who, tensors, n, false)) return rc;
  if (!total) return record_error(MOE_EINVAL, who, "null pointer");
  if (misaligned(total, 8) || misaligned(workspace, 8)) return record_error(MOE_EUNSUPPORTED, who, "total and the workspace must be 8-byte aligned");
  const int64_t need = moe_squares_workspace(tensors, n);
  if (need > 0 && (!workspace || workspace_bytes < need))
    return record_error(MOE_ECAPACITY, who, "the workspace is smaller than moe_squares_workspace says");
  const hipStream_t s = (hipStream_t)stream;
  int parts = 0;
  hipError_t e = for_each_table(tensors, n, [&](const auto& t, int blocks) {
    const hipError_t one = launch_squares(t, (double*)workspace + parts, blocks, s);
    parts += blocks;
    return one;
  });
  if (e == hipSuccess) e = launch_squares_sum((const double*)workspace, parts, total, s);
  return launched(e, who);
}

int moe_clip(const moe_tensor_t* tensors, int32_t n, const double* total, float max_norm, float* norm, void* stream) {
  constexpr const char* who = "moe_clip";
  if (int rc = check_tensors(who, tensors, n, true)) return rc;
  if (!(max_norm >= 0.0f)) return record_error(MOE_EINVAL, who, "max_norm must not be negative");
  if (!total) return record_error(MOE_EINVAL, who, "null pointer");
  if (misaligned(total, 8) || misaligned(norm, 4)) return record_error(MOE_EUNSUPPORTED, who, "total must be 8-byte aligned, norm 4-byte");
  try {
    if (overlapping(tensors, n)) return record_error(MOE_EINVAL, who, "an out overlaps another tensor");
  } catch (const std::exception&) {
    return record_error(MOE_ECAPACITY, who, "no memory for the list");
  }
  const hipStream_t s = (hipStream_t)stream;
  bool told = false;
  hipError_t e = for_each_table(tensors, n, [&](const auto& t, int blocks) {
    const hipError_t one = launch_clip(t, total, max_norm, told ? nullptr : norm, blocks, s);
    told = true;
    return one;
  });
  if (e == hipSuccess && !told && norm) {  // no tensors: the norm alone
    TensorTable<kShortTable> none;
    none.n = 0;
    none.chunks = 0;
    none.chunk = 4096;
    e = launch_clip(none, total, max_norm, norm, 1, s);
  }
  return launched(e, who);
}
