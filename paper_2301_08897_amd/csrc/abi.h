// abi.h -- what the C entry points of the training operators check their
// arguments with. Host side, internal to libscadles.
#pragma once

#include <hip/hip_runtime.h>
#include <cstddef>
#include <cstdint>

#include "scadles.h"

namespace scadles {

scadles_status fail(scadles_status st, const char* fmt, ...);

inline scadles_status launch_status(hipError_t e, const char* where)
{
  return e == hipSuccess ? SCADLES_OK : fail(SCADLES_EHIP, "%s: %s", where, hipGetErrorString(e));
}

inline bool is_aligned(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }

// Whether [a, a + na) and [b, b + nb) share memory; a NULL or empty range shares none.
inline bool bytes_overlap(const void* a, uint64_t na, const void* b, uint64_t nb)
{
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return a && b && na && nb && x < y + nb && y < x + na;
}

inline uint64_t div_up(uint64_t a, uint64_t b) { return (a + b - 1) / b; }

}  // namespace scadles
