// route.hip -- gfx950 kernels of the router: each token's scores, the choice of its experts, their weights,
// and the gradient by the logits.
//
//   p = softmax(l) or sigmoid(l);  pick = p + bias;  ids = top k of pick within the best groups
//   w_j = scale p_j / P,  P = sum of the chosen p (or 1)
//   gradient: dp_j = scale / P (dw_j - sum_i dw_i p_i / P) (+ dscores),
//             softmax dl_e = p_e (dp_e - sum dp p),  sigmoid dl_e = dp_e p_e (1 - p_e)
//
// One wave takes a token; lane i holds experts i, i + 64, ...  A score has to come out the same however it
// is computed, or near ties fall differently from one pass (or one launch shape) to the next: expf and the
// division are the correctly specified ones, and the softmax's sum is taken in 64 bits, whose rounding to 32
// does not depend on the order of the terms.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <type_traits>

#include "ops.hpp"
#include "vec_device.hpp"

namespace moe {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr float kInf = __builtin_inff();

__device__ __forceinline__ float load_logit(const RouteArgs& a, int64_t i) {
  return a.bf16 ? __uint_as_float((uint32_t)((const uint16_t*)a.logits)[i] << 16) : ((const float*)a.logits)[i];
}

// Scores of the token's experts lane, lane + 64, ... into p; returns with l still the logits.
template <int kPer>
__device__ __forceinline__ void scores(const RouteArgs& a, int64_t t, int lane, float (&l)[kPer], float (&p)[kPer]) {
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int e = lane + 64 * i;
    l[i] = e < a.experts ? load_logit(a, t * a.experts + e) : -kInf;
  }
  if (a.sigmoid) {
#pragma unroll
    for (int i = 0; i < kPer; ++i) p[i] = 1.0f / (1.0f + expf(-l[i]));
    return;
  }
  float m = -kInf;
  bool nan = false;
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    m = fmaxf(m, l[i]);
    nan |= l[i] != l[i];
  }
  m = wave_reduce(m, [](float x, float y) { return fmaxf(x, y); });
  if (__any(nan)) m = __uint_as_float(0x7FC00000u);
  if (m == -kInf) m = 0.0f;  // no expert left: every score is 0
  double s = 0.0;
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    p[i] = expf(l[i] - m);
    s += (double)p[i];
  }
  s = wave_reduce(s, [](double x, double y) { return x + y; });
  const float sum = (float)s;
#pragma unroll
  for (int i = 0; i < kPer; ++i) p[i] = sum > 0.0f || sum != sum ? p[i] / sum : 0.0f;
}

// A float as an unsigned integer of the same order (-0 counts as 0).
__device__ __forceinline__ uint32_t ordered(float f) {
  const uint32_t u = __float_as_uint(f + 0.0f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

template <int kPer>
__global__ __launch_bounds__(kThreads) void route_kernel(RouteArgs a) {
  __shared__ float picks[kWaves][1024];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  for (int64_t t = (int64_t)blockIdx.x * kWaves + wave; t < a.tokens; t += (int64_t)gridDim.x * kWaves) {
    float l[kPer], p[kPer], pick[kPer];
    scores<kPer>(a, t, lane, l, p);
    bool nan = false;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int e = lane + 64 * i;
      pick[i] = -kInf;
      if (e >= a.experts) continue;
      if (a.scores) a.scores[t * a.experts + e] = p[i];
      pick[i] = a.bias ? p[i] + a.bias[e] : p[i];
      nan |= pick[i] != pick[i];
      if (l[i] == -kInf) pick[i] = -kInf;
    }
    if (__any(nan)) {
      if (lane < a.k) {
        a.ids[t * a.k + lane] = lane;
        a.weights[t * a.k + lane] = __uint_as_float(0x7FC00000u);
      }
      continue;
    }
    if (a.groups > 1) {
      const int size = a.experts / a.groups;
#pragma unroll
      for (int i = 0; i < kPer; ++i)
        if (lane + 64 * i < a.experts) picks[wave][lane + 64 * i] = pick[i];
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
      __builtin_amdgcn_wave_barrier();
      float value = -kInf;
      if (lane < a.groups) {
        float b0 = -kInf, b1 = -kInf;
        for (int i = 0; i < size; ++i) {
          const float v = picks[wave][lane * size + i];
          b1 = fmaxf(b1, fminf(b0, v));
          b0 = fmaxf(b0, v);
        }
        value = a.group_best == 2 ? b0 + b1 : b0;
      }
      __builtin_amdgcn_wave_barrier();
      int better = 0;
      for (int g = 0; g < a.groups; ++g) {
        const float v = __shfl(value, g);
        better += v > value || (v == value && g < lane);
      }
      const uint64_t keep = __ballot(lane < a.groups && better < a.top_groups);
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        const int e = lane + 64 * i;
        if (e < a.experts && !((keep >> (e / size)) & 1)) pick[i] = -kInf;
      }
    }
    // One choice after another: the largest pick, the lowest index among equals.
    int id = -1;
    float chosen = 0.0f;
    for (int j = 0; j < a.k; ++j) {
      uint64_t best = 0;
#pragma unroll
      for (int i = 0; i < kPer; ++i)
        if (pick[i] > -kInf) best = max(best, (uint64_t)ordered(pick[i]) << 32 | (uint32_t)(1023 - (lane + 64 * i)));
      best = wave_reduce(best, [](uint64_t x, uint64_t y) { return max(x, y); });
      if (best == 0) break;
      const int e = 1023 - (int)(uint32_t)best;
      float v = 0.0f;
#pragma unroll
      for (int i = 0; i < kPer; ++i)
        if (e == lane + 64 * i) {
          v = p[i];
          pick[i] = -kInf;
        }
      v = __shfl(v, e & 63);
      if (lane == j) {
        id = e;
        chosen = v;
      }
    }
    float w = chosen;
    if (a.renormalise) {
      const float total = wave_reduce(chosen, [](float x, float y) { return x + y; });
      w = total > 0.0f ? chosen / total : 0.0f;
    }
    if (lane < a.k) {
      a.ids[t * a.k + lane] = id;
      a.weights[t * a.k + lane] = w * a.scale;
    }
  }
}

template <int kPer>
__global__ __launch_bounds__(kThreads) void route_backward_kernel(RouteArgs a) {
  __shared__ float probs[kWaves][1024], grads[kWaves][1024];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  for (int64_t t = (int64_t)blockIdx.x * kWaves + wave; t < a.tokens; t += (int64_t)gridDim.x * kWaves) {
    float l[kPer], p[kPer];
    scores<kPer>(a, t, lane, l, p);
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int e = lane + 64 * i;
      if (e >= a.experts) continue;
      probs[wave][e] = p[i];
      grads[wave][e] = a.dscores ? a.dscores[t * a.experts + e] : 0.0f;
    }
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    const int id = lane < a.k ? a.ids[t * a.k + lane] : -1;
    const bool have = id >= 0 && id < a.experts;
    const float dw = have ? a.dweights[t * a.k + lane] : 0.0f;
    const float v = have ? probs[wave][id] : 0.0f;
    float dp = dw * a.scale;
    if (a.renormalise) {
      const float total = wave_reduce(v, [](float x, float y) { return x + y; });
      const float mean = wave_reduce(dw * v, [](float x, float y) { return x + y; }) / total;
      dp = total > 0.0f || total != total ? a.scale / total * (dw - mean) : 0.0f;
    }
    for (int j = 0; j < a.k; ++j)
      if (lane == j && have) grads[wave][id] += dp;  // one choice at a time: ids may repeat
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    float g[kPer], dot = 0.0f;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int e = lane + 64 * i;
      g[i] = e < a.experts ? grads[wave][e] : 0.0f;
      dot += e < a.experts ? g[i] * p[i] : 0.0f;
    }
    dot = wave_reduce(dot, [](float x, float y) { return x + y; });
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int e = lane + 64 * i;
      if (e >= a.experts) continue;
      const float d = a.sigmoid ? g[i] * p[i] * (1.0f - p[i]) : p[i] * (g[i] - dot);
      if (a.bf16)
        ((uint16_t*)a.dlogits)[t * a.experts + e] = (uint16_t)bf16x2_of(d, 0.0f);
      else
        ((float*)a.dlogits)[t * a.experts + e] = d;
    }
    __builtin_amdgcn_wave_barrier();
  }
}

template <class F>
hipError_t by_experts(const RouteArgs& a, F&& f) {
  const int per = (a.experts + 63) / 64;
  const dim3 grid((uint32_t)std::min<int64_t>((a.tokens + kWaves - 1) / kWaves, 1 << 20));
  if (per <= 1)
    f(std::integral_constant<int, 1>{}, grid);
  else if (per <= 2)
    f(std::integral_constant<int, 2>{}, grid);
  else if (per <= 4)
    f(std::integral_constant<int, 4>{}, grid);
  else if (per <= 8)
    f(std::integral_constant<int, 8>{}, grid);
  else
    f(std::integral_constant<int, 16>{}, grid);
  return hipGetLastError();
}

hipError_t launch_route(const RouteArgs& a, hipStream_t s) {
  return by_experts(a, [&](auto per, dim3 grid) {
    hipLaunchKernelGGL((route_kernel<decltype(per)::value>), grid, dim3(kThreads), 0, s, a);
  });
}

hipError_t launch_route_backward(const RouteArgs& a, hipStream_t s) {
  return by_experts(a, [&](auto per, dim3 grid) {
    hipLaunchKernelGGL((route_backward_kernel<decltype(per)::value>), grid, dim3(kThreads), 0, s, a);
  });
}

}  // namespace moe
