// What the C entries of the layers share: limits, checks of pointers, status of a launch.
#pragma once

#include <algorithm>
#include <initializer_list>

#include "layers.hpp"

namespace stripe {

constexpr int64_t kMaxFeatures = (int64_t)1 << 24, kMaxStride = (int64_t)1 << 40;
constexpr int kMaxGroups = 4096;

inline int64_t round_up_256(int64_t v) { return (v + 255) / 256 * 256; }
inline int64_t elem_size(int dtype) { return dtype == STRIPE_F32 ? 4 : 2; }

// No exception leaves a C entry: what runs out here is host memory (or a mutex).
template <typename F>
stripe_status_t guarded(F&& body) {
  try {
    return body();
  } catch (...) {
    return STRIPE_ERR_NOMEM;
  }
}

inline stripe_status_t launched(hipError_t e) {
  return e == hipSuccess ? STRIPE_OK : api_fail(STRIPE_ERR_HIP, std::string("kernel launch failed: ") + hipGetErrorString(e));
}

inline bool misaligned(const void* p, int64_t to) { return (uintptr_t)p % (uintptr_t)to != 0; }

// An output that begins where an input or another output does (overlaps with other beginnings are the caller's word).
inline bool shared(std::initializer_list<const void*> outs, std::initializer_list<const void*> ins) {
  for (const void* const* o = outs.begin(); o != outs.end(); ++o)
    if (*o && (std::find(ins.begin(), ins.end(), *o) != ins.end() || std::find(o + 1, outs.end(), *o) != outs.end())) return true;
  return false;
}

// Offsets within a buffer are 64-bit byte counts.
inline bool beyond(int64_t n, int64_t stride) { return (__int128)n * stride > (__int128)1 << 56; }

}  // namespace stripe
