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

// v as the lanes of one step of wave_reduce hold it.
template <int kDpp>
__device__ __forceinline__ uint32_t dpp(uint32_t v) {
  return (uint32_t)__builtin_amdgcn_mov_dpp((int)v, kDpp, 0xF, 0xF, false);
}
template <int kDpp, class T>
__device__ __forceinline__ T dpp_of(T v) {
  if constexpr (sizeof(T) == 4) {
    return __builtin_bit_cast(T, dpp<kDpp>(__builtin_bit_cast(uint32_t, v)));
  } else {
    const u32x2 u = __builtin_bit_cast(u32x2, v);
    return __builtin_bit_cast(T, u32x2{dpp<kDpp>(u[0]), dpp<kDpp>(u[1])});
  }
}
template <int kRow, class T, class F>  // kRow 16 or 32: f of v and of the other half of each 2 kRow lanes
__device__ __forceinline__ T swapped(T v, F&& f) {
  auto one = [](uint32_t u) {
    if constexpr (kRow == 16)
      return __builtin_amdgcn_permlane16_swap(u, u, false, false);
    else
      return __builtin_amdgcn_permlane32_swap(u, u, false, false);
  };
  if constexpr (sizeof(T) == 4) {
    const auto r = one(__builtin_bit_cast(uint32_t, v));
    return f(__builtin_bit_cast(T, (uint32_t)r[0]), __builtin_bit_cast(T, (uint32_t)r[1]));
  } else {
    const u32x2 u = __builtin_bit_cast(u32x2, v);
    const auto lo = one(u[0]), hi = one(u[1]);
    return f(__builtin_bit_cast(T, u32x2{lo[0], hi[0]}), __builtin_bit_cast(T, u32x2{lo[1], hi[1]}));
  }
}

// f over kLanes consecutive lanes (16, 32 or 64), in every one of them and in the same order for each: all on
// the vector unit, where a shuffle through LDS costs some sixty cycles a step.
template <int kLanes = 64, class T, class F>
__device__ __forceinline__ T wave_reduce(T v, F&& f) {
  v = f(v, dpp_of<0xB1>(v));   // lanes 1 0 3 2
  v = f(v, dpp_of<0x4E>(v));   // lanes 2 3 0 1
  v = f(v, dpp_of<0x141>(v));  // 8 lanes mirrored
  v = f(v, dpp_of<0x140>(v));  // 16 lanes mirrored
  if constexpr (kLanes >= 32) v = swapped<16>(v, f);
  if constexpr (kLanes >= 64) v = swapped<32>(v, f);
  return v;
}

}  // namespace moe
