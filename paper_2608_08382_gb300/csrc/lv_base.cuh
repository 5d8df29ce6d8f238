// What all kernels share: the bits of the status word and programmatic dependent
// launch.
#pragma once

#include <cstdint>

namespace lv {

// Bits of the sticky status word (bit 2 is reserved).
constexpr int kStatusData = 1;      // invalid input data
constexpr int kStatusOverflow = 4;  // a fit feature beyond the exact range
constexpr int kStatusTimeout = 8;   // a bounded wait inside a kernel ran out

// Programmatic dependent launch.  A kernel launched so (launch_after in the host
// code) may start while the one before it in the stream still runs: it waits
// here before it reads or writes anything that one does.  The other, early in
// its run, lets it be launched.
__device__ __forceinline__ void wait_previous() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void let_next() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

__device__ __forceinline__ void flag(int *status, int bit) {
  if (status) atomicOr(status, bit);
}

}  // namespace lv
