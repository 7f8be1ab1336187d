// What the entry points of the C ABI share: argument checks and the error state around launches. Host code only.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "../../include/slapo.h"

namespace slapo {

inline size_t align256(size_t v) { return (v + 255) & ~(size_t)255; }
inline bool overlap(const void* a, size_t a_bytes, const void* b, size_t b_bytes) {
  const uintptr_t p = reinterpret_cast<uintptr_t>(a), q = reinterpret_cast<uintptr_t>(b);
  return p < q + b_bytes && q < p + a_bytes;
}
inline bool overlap(const void* a, const void* b, size_t bytes) { return overlap(a, bytes, b, bytes); }   // arrays of `bytes` each
inline bool misaligned(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) != 0; }
inline bool known_dtype(int dtype) { return dtype == SLAPO_BF16 || dtype == SLAPO_FP32 || dtype == SLAPO_FP16; }

// A launch that failed leaves its error in the runtime's per-thread "last error". Every entry point samples that
// slot before its first launch (entry_error) and again after its last one (finish): an error that was already
// there belongs to somebody else and is neither reported as ours nor cleared; one that appeared in between is
// ours, is reported as SLAPO_ERR_HIP and cleared.
inline thread_local hipError_t g_error_at_entry = hipSuccess;
inline void entry_error() { g_error_at_entry = hipPeekAtLastError(); }
inline int finish() {
  if (g_error_at_entry != hipSuccess) return SLAPO_OK;   // cannot tell ours from the stale one: leave it to its owner
  return hipGetLastError() == hipSuccess ? SLAPO_OK : SLAPO_ERR_HIP;
}

}  // namespace slapo
