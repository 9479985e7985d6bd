// Host helpers of the C ABI's entry points.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "fp8rl.h"

namespace {

constexpr int64_t kMaxDim = int64_t(1) << 31;   // per-dimension limit (32-bit tile indices)
constexpr int64_t kMaxLd = int64_t(1) << 24;     // GEMM operand row pitch limit (32-bit in-tile DMA offsets)

inline bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

inline int hip_status(hipError_t e) { return e == hipSuccess ? FP8RL_OK : FP8RL_ERR_HIP; }

inline hipStream_t as_stream(void* s) { return reinterpret_cast<hipStream_t>(s); }

// What a validation gives for a call that is to be launched; an FP8RL_* error, or FP8RL_OK for a
// valid call with nothing to do, otherwise.
constexpr int kLaunch = -1;

}  // namespace
