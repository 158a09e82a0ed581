// route.hip -- gfx950 kernels of the router: each token's scores, the choice of its experts, their weights,
// and the gradient by the logits.
//
//   p = softmax(l) or sigmoid(l);  pick = p + bias;  ids = top k of pick within the best groups
//   w_j = scale p_j / P,  P = sum of the chosen p (or 1)
//   gradient: u_j = scale p_j / P (dw_j - sum_i dw_i p_i / P),  u_e += p_e dscores_e,
//             softmax dl_e = u_e - p_e sum u,  sigmoid dl_e = u_e (1 - p_e)
// u is the scores' gradient times the scores.  The gradient itself would overflow where the chosen scores sum to less
// than scale / 2^128, as a bias can make them; p_j / P is at most 1.
// 1 - p is taken as e^-l p: a difference from a p near 1 would keep few of its bits (at l = 16 it is 6 % off).
//
// Many tokens are bound by vector instructions, not by memory: 32768 tokens of 256 experts take 25 us forward (1600
// instructions for four tokens, half of them in the choice of 8; reading the logits alone would take 7) and 18 to 19
// back (71 MB, 3.8 TB/s).  A few are bound by the chain of the choices: 32 of 256 take 5 us.
//
// kLanes lanes take a token; lane i holds the experts i * run .. i * run + run - 1 (run <= kPer) in registers.
// A score has to come out the same however it is computed, or near ties fall differently from one pass (or one
// launch shape) to the next: expf and the division are the correctly specified ones, and the softmax's sum is
// taken in 64 bits, whose rounding to 32 does not depend on the order of the terms.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <type_traits>

#include "launch.hpp"
#include "ops.hpp"
#include "vec_device.hpp"

namespace moe {

constexpr int kThreads = 256;
constexpr float kInf = __builtin_inff();
constexpr uint32_t kNan = 0x7FC00000u;

typedef float f32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ float fmax2(float a, float b) { return fmaxf(a, b); }
__device__ __forceinline__ float add(float a, float b) { return a + b; }

// How a token's experts lie in its lanes.
template <int kLanes>
struct Place {
  int64_t t;      // token
  bool have;      // t is one of the call's tokens
  int lane;       // within the token's lanes
  int run, e0;    // experts per lane, this lane's first
  int n;          // this lane's experts
  __device__ __forceinline__ explicit Place(const RouteArgs& a) {
    constexpr int kTokens = kThreads / kLanes;
    t = (int64_t)blockIdx.x * kTokens + (int)threadIdx.x / kLanes;
    have = t < a.tokens;
    lane = threadIdx.x % kLanes;
    run = (a.experts + kLanes - 1) / kLanes;
    e0 = lane * run;
    n = have ? min(max(a.experts - e0, 0), run) : 0;
  }
  // The bits of the token's own lanes in a ballot.
  __device__ __forceinline__ uint64_t mine(uint64_t ballot) const {
    if constexpr (kLanes == 64) return ballot;
    return (ballot >> ((threadIdx.x & 63) / kLanes * kLanes)) & ((1ull << kLanes) - 1);
  }
};

__device__ __forceinline__ float logit(const RouteArgs& a, int64_t i) {
  return a.bf16 ? __uint_as_float((uint32_t)((const uint16_t*)a.logits)[i] << 16) : ((const float*)a.logits)[i];
}

// The lane's floats from p on, `none` past its last.
template <int kLanes, int kPer, bool kVec>
__device__ __forceinline__ void load_floats(const Place<kLanes>& at, const float* p, float none, float (&l)[kPer]) {
  if constexpr (kVec) {
#pragma unroll
    for (int i = 0; i < kPer; i += 4) {
      f32x4 v = {none, none, none, none};
      if (i < at.n) v = *(const f32x4*)(p + i);
#pragma unroll
      for (int q = 0; q < 4; ++q) l[i + q] = v[q];
    }
  } else {
#pragma unroll
    for (int i = 0; i < kPer; ++i) l[i] = i < at.n ? p[i] : none;
  }
}

// The lane's logits; -infinity where it has no expert.  kVec: rows and runs are whole vectors of 16 bytes
// (fp32) or 8 (bf16).
template <int kLanes, int kPer, bool kVec>
__device__ __forceinline__ void load_logits(const RouteArgs& a, const Place<kLanes>& at, float (&l)[kPer]) {
  const int64_t base = at.t * a.experts + at.e0;
  if constexpr (!kVec) {
#pragma unroll
    for (int i = 0; i < kPer; ++i) l[i] = i < at.n ? logit(a, base + i) : -kInf;
  } else if (a.bf16) {
    u32x2 v[kPer / 4];
#pragma unroll
    for (int i = 0; i < kPer / 4; ++i) {
      v[i] = u32x2{0xFF80FF80u, 0xFF80FF80u};
      if (4 * i < at.n) v[i] = *(const u32x2*)((const uint16_t*)a.logits + base + 4 * i);
    }
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const uint32_t u = v[i / 4][i % 4 / 2];
      l[i] = __uint_as_float(i % 2 ? u & 0xFFFF0000u : u << 16);
    }
  } else {
    load_floats<kLanes, kPer, kVec>(at, (const float*)a.logits + base, -kInf, l);
  }
}

// 1 - p of a sigmoid score p, from the exponential that p was made with; where that is infinite, p is 0.
__device__ __forceinline__ float sigmoid_rest(float l, float p) { return fminf(expf(-l), 0x1.fffffep127f) * p; }

// The token's maximum and sum, all that a softmax score needs beside its logit.
struct Softmax {
  float m, sum;
};

template <bool kSig>
__device__ __forceinline__ float score(float l, const Softmax& s) {
  if constexpr (kSig) return 1.0f / (1.0f + expf(-l));
  return s.sum > 0.0f || s.sum != s.sum ? expf(l - s.m) / s.sum : 0.0f;
}

template <bool kSig, int kLanes, int kPer>
__device__ __forceinline__ Softmax softmax_of(const Place<kLanes>& at, const float (&l)[kPer]) {
  Softmax s{0.0f, 1.0f};
  if constexpr (kSig) return s;
  float m = -kInf;
  bool nan = false;
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    m = fmaxf(m, l[i]);
    nan |= l[i] != l[i];
  }
  m = wave_reduce<kLanes>(m, fmax2);
  s.m = at.mine(__ballot(nan)) ? __uint_as_float(kNan) : m == -kInf ? 0.0f : m;  // no expert left: every score is 0
  double sum = 0.0;
#pragma unroll
  for (int i = 0; i < kPer; ++i) sum += (double)expf(l[i] - s.m);
  s.sum = (float)wave_reduce<kLanes>(sum, [](double x, double y) { return x + y; });
  return s;
}

// Leaves the picks of the token's best groups and makes the others -infinity.  A group of a whole power of
// two of lanes is reduced in registers, another through the wave's LDS.
template <int kLanes, int kPer>
__device__ __forceinline__ void keep_groups(const RouteArgs& a, const Place<kLanes>& at, float (&pick)[kPer], float* picks) {
  const int size = a.experts / a.groups;
  const int span = size / at.run;  // lanes of a group
  auto two = [&](float& b0, float& b1, float v) {
    b1 = fmaxf(b1, fminf(b0, v));
    b0 = fmaxf(b0, v);
  };
  // A group with fewer experts left than count for it is worth nothing (and infinity less infinity is no NaN).
  auto worth = [&](float b0, float b1) { return a.group_best == 2 ? (b1 == -kInf ? -kInf : b0 + b1) : b0; };
  if (size % at.run == 0 && (span & (span - 1)) == 0 && span <= 16) {
    float b0 = -kInf, b1 = -kInf;
#pragma unroll
    for (int i = 0; i < kPer; ++i) two(b0, b1, pick[i]);
    auto merge = [&](float o0, float o1) {
      b1 = fmaxf(fminf(b0, o0), fmaxf(b1, o1));
      b0 = fmaxf(b0, o0);
    };
    if (span >= 2) merge(dpp_of<0xB1>(b0), dpp_of<0xB1>(b1));
    if (span >= 4) merge(dpp_of<0x4E>(b0), dpp_of<0x4E>(b1));
    if (span >= 8) merge(dpp_of<0x141>(b0), dpp_of<0x141>(b1));
    if (span >= 16) merge(dpp_of<0x140>(b0), dpp_of<0x140>(b1));
    const float value = worth(b0, b1);
    const int group = at.lane / span;
    int better = 0;
    for (int g = 0; g < a.groups; ++g) {
      const float v = __shfl(value, g * span, kLanes);
      better += v > value || (v == value && g < group);
    }
    if (better >= a.top_groups) {
#pragma unroll
      for (int i = 0; i < kPer; ++i) pick[i] = -kInf;
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < kPer; ++i)
    if (i < at.n) picks[at.e0 + i] = pick[i];
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  // Lane g has group g; 16 lanes have up to four each.
  constexpr int kMost = 64 / kLanes;
  uint64_t keep = 0;
  float value[kMost];
#pragma unroll
  for (int u = 0; u < kMost; ++u) {
    const int g = u * kLanes + at.lane;
    float b0 = -kInf, b1 = -kInf;
    if (g < a.groups && at.have)
      for (int i = 0; i < size; ++i) two(b0, b1, picks[g * size + i]);
    value[u] = worth(b0, b1);
  }
  __builtin_amdgcn_wave_barrier();
#pragma unroll
  for (int u = 0; u < kMost; ++u) {
    const int mine = u * kLanes + at.lane;
    int better = 0;
    for (int g = 0; g < a.groups; ++g) {
      float v = __shfl(value[0], g, kLanes);
#pragma unroll
      for (int o = 1; o < kMost; ++o) {
        const float w = __shfl(value[o], g, kLanes);
        if (g / kLanes == o) v = w;
      }
      better += v > value[u] || (v == value[u] && g < mine);
    }
    keep |= at.mine(__ballot(mine < a.groups && better < a.top_groups)) << (u * kLanes % 64);
  }
#pragma unroll
  for (int i = 0; i < kPer; ++i)
    if (!((keep >> ((at.e0 + i) / size & 63)) & 1)) pick[i] = -kInf;
}

// v of the token's lane `lane`; a whole wave's is the same in all of its lanes, and a scalar read.
template <int kLanes>
__device__ __forceinline__ int from_lane(int v, int lane) {
  if constexpr (kLanes == 64) return __builtin_amdgcn_readlane(v, __builtin_amdgcn_readfirstlane(lane));
  return __shfl(v, lane, kLanes);
}

template <int kLanes, int kPer, bool kVec, bool kSig>
__global__ __launch_bounds__(kThreads) void route_kernel(RouteArgs a) {
  __shared__ float picks[kThreads / kLanes][kLanes * kPer];
  const Place<kLanes> at(a);
  float l[kPer], pick[kPer];
  load_logits<kLanes, kPer, kVec>(a, at, l);
  if (a.bias) {
    load_floats<kLanes, kPer, kVec>(at, a.bias + at.e0, 0.0f, pick);
  } else {
#pragma unroll
    for (int i = 0; i < kPer; ++i) pick[i] = 0.0f;
  }
  const Softmax sm = softmax_of<kSig, kLanes, kPer>(at, l);
  if (a.scores) {
#pragma unroll
    for (int i = 0; i < kPer; ++i)
      if (i < at.n) a.scores[at.t * a.experts + at.e0 + i] = score<kSig>(l[i], sm);
  }
  bool nan = false;
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    pick[i] += score<kSig>(l[i], sm);
    nan |= pick[i] != pick[i];
    if (l[i] == -kInf) pick[i] = -kInf;
  }
  const bool poisoned = at.mine(__ballot(nan)) != 0;
  if (a.groups > 1) keep_groups<kLanes, kPer>(a, at, pick, picks[threadIdx.x / kLanes]);
  // One choice after another: the largest pick, the lowest expert among equals; -infinity is none.
  int id = -1;
  for (int j = 0; j < a.k; ++j) {
    float best = pick[0];
#pragma unroll
    for (int i = 1; i < kPer; ++i) best = fmaxf(best, pick[i]);
    best = wave_reduce<kLanes>(best, fmax2);
    // The first of the lane's experts with it; of several lanes' the first lane's, whose experts come first.
    int found = kPer;
#pragma unroll
    for (int i = kPer - 1; i >= 0; --i) found = pick[i] == best ? i : found;
    const uint64_t who = at.mine(__ballot(found < kPer && best > -kInf));
    const int first = __builtin_ctzll(who | 1ull << 63);
    const int e = from_lane<kLanes>(at.e0 + found, first);
    if (at.lane == j && who != 0) id = e;
    if (at.lane != first) found = kPer;
#pragma unroll
    for (int i = 0; i < kPer; ++i) pick[i] = found == i ? -kInf : pick[i];
  }
  const bool mine = at.have && at.lane < a.k;
  if (poisoned) id = at.lane;
  float chosen = 0.0f;
  if (mine && id >= 0) chosen = score<kSig>(logit(a, at.t * a.experts + id), sm);
  float w = chosen;
  if (a.renormalise) {
    const float total = wave_reduce<kLanes>(chosen, add);
    w = total > 0.0f ? chosen / total : 0.0f;
  }
  if (mine) {
    a.ids[at.t * a.k + at.lane] = id;
    a.weights[at.t * a.k + at.lane] = poisoned ? __uint_as_float(kNan) : w * a.scale;
  }
}

template <int kLanes, int kPer, bool kVec, bool kSig>
__global__ __launch_bounds__(kThreads) void route_backward_kernel(RouteArgs a) {
  __shared__ __attribute__((aligned(16))) float table[kThreads / kLanes][kLanes * kPer];
  const Place<kLanes> at(a);
  float* grads = table[threadIdx.x / kLanes];
  float l[kPer], p[kPer], g[kPer];
  load_logits<kLanes, kPer, kVec>(a, at, l);
  const int id = at.have && at.lane < a.k ? a.ids[at.t * a.k + at.lane] : -1;
  const bool have = id >= 0 && id < a.experts;
  const float dw = have ? a.dweights[at.t * a.k + at.lane] : 0.0f;
  const float own = have ? logit(a, at.t * a.experts + id) : -kInf;
  if (a.dscores) {
    load_floats<kLanes, kPer, kVec>(at, a.dscores + at.t * a.experts + at.e0, 0.0f, g);
  } else {
#pragma unroll
    for (int i = 0; i < kPer; ++i) g[i] = 0.0f;
  }
  const Softmax sm = softmax_of<kSig, kLanes, kPer>(at, l);
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    p[i] = score<kSig>(l[i], sm);
    grads[at.lane * kPer + i] = p[i] * g[i];
    if constexpr (kSig) p[i] = sigmoid_rest(l[i], p[i]);  // all that is asked of it from here on
  }
  const float v = have ? score<kSig>(own, sm) : 0.0f;
  float u = a.scale * v * dw;
  if (a.renormalise) {
    const float total = wave_reduce<kLanes>(v, add), share = v / total;
    const float mean = wave_reduce<kLanes>(dw * share, add);
    u = total > 0.0f || total != total ? a.scale * share * (dw - mean) : 0.0f;
  }
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  // One choice at a time, as ids may repeat: a wave's LDS operations happen in their order.
  const int slot = have ? id / at.run * kPer + id % at.run : 0;
  for (int j = 0; j < a.k; ++j)
    if (at.lane == j && have) atomicAdd(&grads[slot], u);
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
  float dot = 0.0f;
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    g[i] = grads[at.lane * kPer + i];
    dot += g[i];
  }
  if constexpr (!kSig) dot = wave_reduce<kLanes>(dot, add);
#pragma unroll
  for (int i = 0; i < kPer; ++i) g[i] = kSig ? g[i] * p[i] : g[i] - p[i] * dot;
  const int64_t base = at.t * a.experts + at.e0;
#pragma unroll
  for (int i = 0; i < kPer; i += kVec ? 4 : 1) {
    if (i >= at.n) continue;
    if constexpr (kVec) {
      if (a.bf16)
        *(u32x2*)((uint16_t*)a.dlogits + base + i) = u32x2{bf16x2_of(g[i], g[i + 1]), bf16x2_of(g[i + 2], g[i + 3])};
      else
        *(f32x4*)((float*)a.dlogits + base + i) = f32x4{g[i], g[i + 1], g[i + 2], g[i + 3]};
    } else if (a.bf16) {
      ((uint16_t*)a.dlogits)[base + i] = (uint16_t)bf16x2_of(g[i], 0.0f);
    } else {
      ((float*)a.dlogits)[base + i] = g[i];
    }
  }
}

// Calls f(lanes per token, experts per lane at most, whole vectors, sigmoid) as compile-time values; `f32`:
// fp32 arrays read or written in vectors beside the logits, `also` one of the logits' type.
template <class F>
void by_shape(const RouteArgs& a, const void* also, const void* f32, F&& f) {
  // Few lanes to a token cost the least work in all (a reduction over 16 is four steps, and four tokens share
  // each): 32768 tokens of 256 experts 25 us with 16 lanes, 69 with 64; 21082 of 384 and back 34 with 32 lanes, 43
  // with 64.  64 lanes have the shorter chain, for few tokens.  A choice has a lane, so more of them ask for more lanes.
  const bool many = a.tokens > 2048;
  const int lanes = many && a.experts <= 256 && a.k <= 16 ? 16 : many && a.experts <= 512 && a.k <= 32 ? 32 : 64;
  const int run = (a.experts + lanes - 1) / lanes;
  const uintptr_t align = a.bf16 ? 8 : 16;
  const bool vec = run % 4 == 0 && a.experts % 4 == 0 && (((uintptr_t)a.logits | (uintptr_t)also) & (align - 1)) == 0 &&
                   ((uintptr_t)f32 & 15) == 0;
  auto kind = [&](auto lanes, auto per, auto v) {
    if (a.sigmoid)
      f(lanes, per, v, std::true_type{});
    else
      f(lanes, per, v, std::false_type{});
  };
  auto with = [&](auto lanes, auto per) {
    if constexpr (decltype(per)::value >= 4) {
      if (vec) return kind(lanes, per, std::true_type{});
    }
    kind(lanes, per, std::false_type{});
  };
  auto pick = [&](auto lanes) {
    if constexpr (decltype(lanes)::value == 32)
      return with(lanes, std::integral_constant<int, 16>{});  // more than 256 experts, or 16 choices
    else if (run <= 1)
      with(lanes, std::integral_constant<int, 1>{});
    else if (run <= 2)
      with(lanes, std::integral_constant<int, 2>{});
    else if (run <= 4)
      with(lanes, std::integral_constant<int, 4>{});
    else if (run <= 8)
      with(lanes, std::integral_constant<int, 8>{});
    else
      with(lanes, std::integral_constant<int, 16>{});
  };
  if (lanes == 16)
    pick(std::integral_constant<int, 16>{});
  else if (lanes == 32)
    pick(std::integral_constant<int, 32>{});
  else
    pick(std::integral_constant<int, 64>{});
}

int64_t token_blocks(const RouteArgs& a, int lanes) {
  const int64_t per = kThreads / lanes;
  return (a.tokens + per - 1) / per;
}

hipError_t launch_route(const RouteArgs& a, hipStream_t s) {
  hipError_t e = hipErrorInvalidConfiguration;
  by_shape(a, nullptr, a.bias, [&](auto lanes, auto per, auto vec, auto sig) {
    constexpr int L = decltype(lanes)::value, P = decltype(per)::value;
    const int64_t blocks = token_blocks(a, L);
    if (!launch_fits(blocks, kThreads)) return;
    e = launch(route_kernel<L, P, decltype(vec)::value, decltype(sig)::value>, dim3((uint32_t)blocks), dim3(kThreads), 0, s, a);
  });
  return e;
}

hipError_t launch_route_backward(const RouteArgs& a, hipStream_t s) {
  hipError_t e = hipErrorInvalidConfiguration;
  by_shape(a, a.dlogits, a.dscores, [&](auto lanes, auto per, auto vec, auto sig) {
    constexpr int L = decltype(lanes)::value, P = decltype(per)::value;
    const int64_t blocks = token_blocks(a, L);
    if (!launch_fits(blocks, kThreads)) return;
    e = launch(route_backward_kernel<L, P, decltype(vec)::value, decltype(sig)::value>, dim3((uint32_t)blocks), dim3(kThreads), 0, s, a);
  });
  return e;
}

}  // namespace moe
