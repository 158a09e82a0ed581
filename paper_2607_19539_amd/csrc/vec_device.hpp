// vec_device.hpp -- small device helpers shared by the operators around the stage.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace moe {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// The 8 floats of 8 packed bf16.
__device__ __forceinline__ void unpack8(const u32x4& v, float (&f)[8]) {
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    f[2 * q] = __uint_as_float(v[q] << 16);
    f[2 * q + 1] = __uint_as_float(v[q] & 0xFFFF0000u);
  }
}

// Two floats -> two bf16, round to nearest even (v_cvt_pk_bf16_f32).
__device__ __forceinline__ uint32_t bf16x2_of(float lo, float hi) {
  typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
  typedef float f32x2_t __attribute__((ext_vector_type(2)));
  const f32x2_t v = {lo, hi};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2_t));
}

__device__ __forceinline__ u32x4 pack8(const float (&f)[8]) {
  u32x4 v;
#pragma unroll
  for (int q = 0; q < 4; ++q) v[q] = bf16x2_of(f[2 * q], f[2 * q + 1]);
  return v;
}

// The magnitude of a float as an integer that orders as it does, infinities and NaN on top: a maximum
// taken of these does not lose a NaN as one of floats would.
__device__ __forceinline__ uint32_t magnitude(float f) { return __float_as_uint(f) & 0x7FFFFFFFu; }

template <class T, class F>
__device__ __forceinline__ T wave_reduce(T v, F&& f) {
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) v = f(v, __shfl_xor(v, d));
  return v;
}

}  // namespace moe
