// Device helpers of the answering kernels: elements of the three row types, lanes.
#pragma once

#include "horizon.h"
#include "hs_device.h"

namespace hs {

// Element i of a row of fp32, bf16 (raw bits) or fp16 values.
__device__ __forceinline__ float elem(const float* p, int64_t i) { return p[i]; }
__device__ __forceinline__ float elem(const uint16_t* p, int64_t i) { return bf2f(p[i]); }
__device__ __forceinline__ float elem(const _Float16* p, int64_t i) { return float(p[i]); }

// Value of lane (lane ^ J).
template <int J>
__device__ __forceinline__ uint32_t xor_lane(uint32_t v) {
  if constexpr (J == 1) {
    return __builtin_amdgcn_mov_dpp(v, 0xB1, 0xf, 0xf, true);  // quad_perm 1 0 3 2
  } else if constexpr (J == 2) {
    return __builtin_amdgcn_mov_dpp(v, 0x4E, 0xf, 0xf, true);  // quad_perm 2 3 0 1
  } else if constexpr (J == 4) {
    const uint32_t u = __builtin_amdgcn_mov_dpp(v, 0x141, 0xf, 0xf, true);  // half row mirrored: ^ 7
    return __builtin_amdgcn_mov_dpp(u, 0x1B, 0xf, 0xf, true);               // quad_perm 3 2 1 0: ^ 3
  } else if constexpr (J == 8) {
    return __builtin_amdgcn_mov_dpp(v, 0x128, 0xf, 0xf, true);  // rotate a row of 16 by 8
  } else if constexpr (J == 16) {
    const auto s = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    return (threadIdx.x & 16) ? s[0] : s[1];
  } else {
    static_assert(J == 32, "lane distance");
    const auto s = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    return (threadIdx.x & 32) ? s[0] : s[1];
  }
}
template <int J>
__device__ __forceinline__ float xor_lane(float v) {
  return __uint_as_float(xor_lane<J>(__float_as_uint(v)));
}
template <int J>
__device__ __forceinline__ uint64_t xor_lane(uint64_t v) {
  return (uint64_t(xor_lane<J>(uint32_t(v >> 32))) << 32) | xor_lane<J>(uint32_t(v));
}
template <int J>
__device__ __forceinline__ double xor_lane(double v) {
  return __builtin_bit_cast(double, xor_lane<J>(__builtin_bit_cast(uint64_t, v)));
}

// f over the 64 lanes, in every lane.
template <typename V, typename F>
__device__ __forceinline__ V reduce_wave(V v, F f) {
  v = f(v, xor_lane<1>(v));
  v = f(v, xor_lane<2>(v));
  v = f(v, xor_lane<4>(v));
  v = f(v, xor_lane<8>(v));
  v = f(v, xor_lane<16>(v));
  return f(v, xor_lane<32>(v));
}
}  // namespace hs
