// Argument checks that the entry points share (api.hip, api8.hip).
#pragma once
#include <stddef.h>
#include <stdint.h>

#include <hip/hip_runtime.h>

#include "../../include/rmm.h"

namespace rmm {

namespace {

constexpr int64_t kMaxDim = (int64_t)1 << 31;
constexpr int64_t kMaxElems = (int64_t)1 << 40;

inline bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
inline size_t round_up(size_t x, size_t a) { return (x + a - 1) / a * a; }

inline bool dims_ok(int64_t a, int64_t b) { return a >= 1 && b >= 1 && a < kMaxDim && b < kMaxDim && a * b < kMaxElems; }

inline int from_hip(hipError_t e) { return e == hipSuccess ? RMM_OK : RMM_ERR_LAUNCH; }

}  // namespace

}  // namespace rmm
