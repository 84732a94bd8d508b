// Host side of every entry point: argument checks they share, and the launch of one kernel.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <tuple>

namespace hydra {

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

inline bool head_dim_supported(int d) { return d == 64 || d == 80 || d == 128; }

// Enqueues one kernel and returns the status of THIS launch (the runtime's sticky last-error slot
// is shared by every caller of the process and may hold somebody else's failure).
template <typename... Params, typename... Args>
hipError_t launch_lds(void (*kernel)(Params...), dim3 grid, dim3 block, size_t lds_bytes, hipStream_t stream, const Args&... args) {
  static_assert(sizeof...(Params) == sizeof...(Args), "one argument per kernel parameter");
  std::tuple<Params...> vals(args...);
  return std::apply(
      [&](auto&... v) {
        void* ptrs[] = {static_cast<void*>(&v)...};
        return hipLaunchKernel(reinterpret_cast<const void*>(kernel), grid, block, ptrs, lds_bytes, stream);
      },
      vals);
}
template <typename... Params, typename... Args>
hipError_t launch(void (*kernel)(Params...), dim3 grid, dim3 block, hipStream_t stream, const Args&... args) {
  return launch_lds(kernel, grid, block, 0, stream, args...);
}

}  // namespace hydra
