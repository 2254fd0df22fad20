// 8-bit integer products with one scale per token and per channel:
//   out[m, n] = a_scale[m] * w_scale[n] * sum_k a[m, k] w[n, k] + bias[n]
// The sum is exact (32-bit accumulators, k <= 131071); the conversion of the
// sum, the product of the scales, their product and the bias are one fp32
// rounding each, and the result is rounded once to the output's type.
#include "answer_kernels.h"
#include "horizon.h"
#include "hs_device.h"

namespace hs {
namespace {

typedef int32_t i32x4 __attribute__((ext_vector_type(4)));

constexpr int BT = 64;  // rows and channels per block
constexpr int BK = 64;  // K per stage

__device__ __forceinline__ i32x4 mfma16_i8(const i32x4& a, const i32x4& b, const i32x4& c) {
  return __builtin_amdgcn_mfma_i32_16x16x64_i8(a, b, c, 0, 0, 0);
}

__device__ __forceinline__ void store_out(void* out, int type, int64_t i, float v) {
  if (type == HS_TYPE_F32) {
    static_cast<float*>(out)[i] = v;
  } else if (type == HS_TYPE_F16) {
    static_cast<_Float16*>(out)[i] = _Float16(v);
  } else {
    static_cast<__bf16*>(out)[i] = __bf16(v);
  }
}

// Four waves, each 16 channels x 64 rows; operands byte by byte through LDS.
__global__ __launch_bounds__(256) void linear_kernel(LinearI8Args a) {
  __shared__ __attribute__((aligned(16))) int8_t sa[BT][BK + 16], sw[BT][BK + 16];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int m0 = blockIdx.y * BT, n0 = blockIdx.x * BT;
  i32x4 acc[4] = {};
  for (int k0 = 0; k0 < a.k; k0 += BK) {
    for (int i = tid; i < BT * BK; i += 256) {
      const int r = i / BK, k = k0 + i % BK;
      sa[r][i % BK] = (m0 + r < a.m && k < a.k) ? a.a[int64_t(m0 + r) * a.lda + k] : int8_t(0);
      sw[r][i % BK] = (n0 + r < a.n && k < a.k) ? a.w[int64_t(n0 + r) * a.ldw + k] : int8_t(0);
    }
    __syncthreads();
    const i32x4 w = *reinterpret_cast<const i32x4*>(&sw[wave * 16 + lane % 16][lane / 16 * 16]);
#pragma unroll
    for (int j = 0; j < 4; ++j)
      acc[j] = mfma16_i8(w, *reinterpret_cast<const i32x4*>(&sa[j * 16 + lane % 16][lane / 16 * 16]), acc[j]);
    __syncthreads();
  }
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int m = m0 + j * 16 + lane % 16;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int n = n0 + wave * 16 + 4 * (lane / 16) + r;
      if (m >= a.m || n >= a.n) continue;
      float v = __fmul_rn(float(acc[j][r]), __fmul_rn(a.a_scale[m], a.w_scale[n]));
      if (a.bias) v = __fadd_rn(v, bf2f(a.bias[n]));
      store_out(a.out, a.out_type, int64_t(m) * a.ldo + n, v);
    }
  }
}

}  // namespace

hipError_t launch_linear_i8(const LinearI8Args& a, int cus, hipStream_t s) {
  (void)cus;
  if (a.m < 1 || a.n < 1) return hipSuccess;
  const dim3 grid((a.n + BT - 1) / BT, (a.m + BT - 1) / BT);
  if (grid.y > 65535) return hipErrorInvalidValue;
  hipLaunchKernelGGL(linear_kernel, grid, dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace hs
