// Host-side checks that the operators on the caller's own tensors share (norm.cu, ffn_sm100.cu).
#pragma once

#include <atomic>

#include "common.h"

namespace moe {

constexpr int kMaxOperatorTokens = 1 << 24;

// Multiprocessors of the current device; 148 where there is none to ask.
inline int sm_count() {
  static std::atomic<int> known[64] = {};
  int dev = 0, v = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0) return 148;
  if (dev < 64 && (v = known[dev].load(std::memory_order_relaxed))) return v;
  if (cudaDeviceGetAttribute(&v, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || v < 1) return 148;
  if (dev < 64) known[dev].store(v, std::memory_order_relaxed);
  return v;
}

inline bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }
inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// [p, p + n) against [q, q + m); a null pointer overlaps nothing
inline bool overlap(const void* p, size_t n, const void* q, size_t m) {
  const uintptr_t a = reinterpret_cast<uintptr_t>(p), b = reinterpret_cast<uintptr_t>(q);
  return p && q && a < b + m && b < a + n;
}

inline int element_size(int dtype) { return dtype == MOE_FP32 ? 4 : dtype == MOE_BF16 || dtype == MOE_FP16 ? 2 : 0; }

}  // namespace moe
