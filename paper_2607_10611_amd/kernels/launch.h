// Host helpers of the entry points outside madd.hip: kernel launches and
// argument checks.
#pragma once

#include <hip/hip_runtime.h>

#include <stdint.h>

#include <tuple>
#include <utility>

#include "madd.h"

namespace madd_detail {

// Kernel launch that reports the launch's own status (hipLaunchKernel returns
// it directly); the thread's last-error state, which belongs to the caller, is
// neither read nor cleared.
template <typename Tuple, size_t... I>
inline void kernel_args(void** argv, Tuple& t, std::index_sequence<I...>) {
  ((argv[I] = (void*)&std::get<I>(t)), ...);
}

// Workgroups of `threads` threads that a launch holds: fewer than 2^32 threads.
constexpr int64_t most_workgroups(int64_t threads) { return 0xFFFFFFFFll / threads; }

template <typename... P, typename... A>
inline int32_t launch_kernel_lds(void (*k)(P...), dim3 grid, dim3 block, unsigned lds,
                                 hipStream_t stream, A&&... a) {
  if ((int64_t)grid.x > most_workgroups(block.x)) return MADD_EUNSUPPORTED;
  std::tuple<P...> args(std::forward<A>(a)...);
  void* argv[sizeof...(P) > 0 ? sizeof...(P) : 1];
  kernel_args(argv, args, std::index_sequence_for<P...>{});
  return hipLaunchKernel(reinterpret_cast<const void*>(k), grid, block, argv, lds, stream) ==
                 hipSuccess
             ? MADD_OK
             : MADD_EDEVICE;
}

template <typename... P, typename... A>
inline int32_t launch_kernel(void (*k)(P...), dim3 grid, dim3 block, hipStream_t stream, A&&... a) {
  return launch_kernel_lds(k, grid, block, 0u, stream, std::forward<A>(a)...);
}

// Whether a matrix of rows `ld` elements apart ends within 2^57 bytes, the addresses
// that there are (so that its offsets and the ranges below do not wrap round).
inline bool rows_fit(int64_t rows, int64_t ld, int64_t bytes) {
  return rows <= 1 || ld <= 0 || rows - 1 <= ((int64_t)1 << 57) / bytes / ld;
}

// A byte range of device memory that a call reads or writes.
struct Range {
  const void* p;
  uint64_t bytes;
};
inline bool overlap(const Range& a, const Range& b) {
  if (!a.p || !b.p || a.bytes == 0 || b.bytes == 0) return false;
  const uintptr_t a0 = (uintptr_t)a.p, b0 = (uintptr_t)b.p;
  return a0 < b0 + b.bytes && b0 < a0 + a.bytes;
}
// Whether the ranges from `first_written` on share no byte with any other one
// (inputs may overlap each other).
inline bool writes_are_apart(const Range* r, int n, int first_written) {
  for (int i = first_written; i < n; ++i)
    for (int j = 0; j < i; ++j)
      if (overlap(r[i], r[j])) return false;
  return true;
}

}  // namespace madd_detail
