// Checks and limits shared by the host sides of the C ABI (vico_api.hip, cache_api.hip).
#pragma once

#include <stdint.h>

namespace vico {

constexpr int64_t kMaxChunk = int64_t(1) << 20;
constexpr int64_t kMaxKeys = int64_t(1) << 30;
constexpr int kMaxHeads = 1024;
constexpr int64_t kMaxTensorBytes = int64_t(1) << 31;

inline bool aligned_to(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
inline bool aligned16(const void* p) { return aligned_to(p, 16); }

inline bool overlaps(const void* a, int64_t na, const void* b, int64_t nb) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return na > 0 && nb > 0 && x < y + (uintptr_t)nb && y < x + (uintptr_t)na;
}

inline int64_t align256(int64_t x) { return (x + 255) & ~int64_t(255); }

}  // namespace vico
