// Host-side checks that the operators on the caller's own tensors share (norm.cu, ffn_sm100.cu).
#pragma once

#include "common.h"

namespace moe {

constexpr int kMaxOperatorTokens = 1 << 24;

// Multiprocessors of the current device.
inline int sm_count() {
  static int n[64] = {};
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return 148;
  if (!n[dev]) {
    int v = 0;
    n[dev] = cudaDeviceGetAttribute(&v, cudaDevAttrMultiProcessorCount, dev) == cudaSuccess && v > 0 ? v : 148;
  }
  return n[dev];
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
