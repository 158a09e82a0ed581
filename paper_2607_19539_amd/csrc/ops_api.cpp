// ops_api.cpp -- the C ABI of the operators around the stage: argument checks and launches.
#include <hip/hip_runtime.h>
#include <stdint.h>

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
