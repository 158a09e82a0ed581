// launch.hpp -- a kernel launch that reports its own status (host side).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

namespace moe {

// The launch's own result.  hipGetLastError after a launch would also report what some earlier call of the program
// left behind, of which the caller would take a kernel that runs for one that was refused.
template <class... P>
hipError_t launch(void (*kernel)(P...), dim3 grid, dim3 threads, uint32_t lds, hipStream_t s, std::common_type_t<P>... args) {
  void* pointers[] = {(void*)&args...};
  return hipLaunchKernel((const void*)kernel, grid, threads, pointers, lds, s);
}

}  // namespace moe
