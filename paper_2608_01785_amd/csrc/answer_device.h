// Device helpers of the answering kernels: elements of the three row types.
#pragma once

#include "horizon.h"
#include "hs_device.h"

namespace hs {

// Element i of a row of fp32, bf16 (raw bits) or fp16 values.
__device__ __forceinline__ float elem(const float* p, int64_t i) { return p[i]; }
__device__ __forceinline__ float elem(const uint16_t* p, int64_t i) { return bf2f(p[i]); }
__device__ __forceinline__ float elem(const _Float16* p, int64_t i) { return float(p[i]); }

}  // namespace hs
