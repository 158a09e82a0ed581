// gate.hip -- gfx950 kernels of the gated activation and its gradient, of rows that hold g and u side by side.
//
//   act = silu(g) u,   du = dact silu(g),   dg = dact u s (1 + g (1 - s)),   s = 1 / (1 + e^-g)
//
// Eight features a thread, each tensor read or written once in 16-byte pieces: memory bounds both (49152 rows of 1408:
// 415 MB in 75 us, 692 MB in 116, 5.6 and 6.0 TB/s).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "launch.hpp"
#include "ops.hpp"
#include "vec_device.hpp"

namespace moe {

namespace {

constexpr int kThreads = 256;

// The thread's row and first feature, if it has any.
struct Place {
  int64_t row;
  int f;
  bool have;
  __device__ __forceinline__ explicit Place(const GateArgs& a) {
    const uint32_t per = (uint32_t)a.F / 8, q = blockIdx.x * (uint32_t)kThreads + threadIdx.x;
    row = q / per;
    f = (int)(q % per) * 8;
    have = row < (a.end ? min((int64_t)*a.end, a.rows) : a.rows);
  }
};

__global__ __launch_bounds__(kThreads) void gate_kernel(GateArgs a) {
  const Place p(a);
  if (!p.have) return;
  const uint16_t* gu = a.gu + p.row * 2 * a.F + p.f;
  float g[8], u[8];
  unpack8(*(const u32x4*)gu, g);
  unpack8(*(const u32x4*)(gu + a.F), u);
#pragma unroll
  for (int i = 0; i < 8; ++i) g[i] = silu_mul(g[i] * kGateShare, u[i]);
  *(u32x4*)(a.act + p.row * a.F + p.f) = pack8(g);
}

// With e^-g infinite (g below -88.7) s is 0 here and 1 - s is 1.  1 - s is within some 2^-24, so 1 + g (1 - s) is off by a
// few |g| 2^-24 beside terms of 1 and |g|.  Relative to the sum itself that is most next to its zero: -0.0028 at g = -1.28125,
// the nearest value of bf16, is still within 2^-14 of itself, far inside of bf16's half step.
template <bool with_act>
__global__ __launch_bounds__(kThreads) void gate_backward_kernel(GateArgs a) {
  const Place p(a);
  if (!p.have) return;
  const uint16_t* gu = a.gu + p.row * 2 * a.F + p.f;
  float g[8], u[8], d[8], dg[8], act[8];
  unpack8(*(const u32x4*)gu, g);
  unpack8(*(const u32x4*)(gu + a.F), u);
  unpack8(*(const u32x4*)(a.dact + p.row * a.F + p.f), d);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float q = g[i] * kGateShare, s4 = sigmoid4(q);
    // The larger of the two factors first, a quarter of it: s (1 + g (1 - s)) reaches 1.1, so neither a small nor a large
    // one is lost on the way to a middling product.
    const bool swap = fabsf(d[i]) < fabsf(u[i]);
    dg[i] = fmaf(q, 1.0f - kGateShare * s4, kGateShare) * s4 * ((swap ? u[i] : d[i]) * 0.25f) * (swap ? d[i] : u[i]) * 4.0f;
    if constexpr (with_act) act[i] = q * s4 * u[i];
    d[i] *= q * s4;
  }
  uint16_t* out = a.dgu + p.row * 2 * a.F + p.f;
  *(u32x4*)out = pack8(dg);
  *(u32x4*)(out + a.F) = pack8(d);
  if constexpr (with_act) *(u32x4*)(a.act + p.row * a.F + p.f) = pack8(act);
}

hipError_t launch_rows(void (*kernel)(GateArgs), const GateArgs& a, hipStream_t s) {
  const int64_t blocks = (a.rows * (a.F / 8) + kThreads - 1) / kThreads;
  if (!launch_fits(blocks, kThreads)) return hipErrorInvalidConfiguration;
  return launch(kernel, dim3((uint32_t)blocks), dim3(kThreads), 0, s, a);
}

}  // namespace

hipError_t launch_gate(const GateArgs& a, hipStream_t s) { return launch_rows(gate_kernel, a, s); }
hipError_t launch_gate_backward(const GateArgs& a, hipStream_t s) {
  return launch_rows(a.act ? gate_backward_kernel<true> : gate_backward_kernel<false>, a, s);
}

}  // namespace moe
