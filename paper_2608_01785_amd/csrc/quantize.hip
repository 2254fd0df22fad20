// Rows to 8-bit integers with one scale each, RMS-normalised on the way when a
// gain is given.
//
//   y = x                                   (no gain)
//   y = x / sqrt(mean(x^2) + eps) * gain    (RMSNorm)
//   a = max |y|,  scale = a / 127,  q = rint(127 y / a), ties to even
//
// The row's reciprocal root mean square scales y and a alike, so it cancels in
// q = rint(127 x g / max |x g|): the integers are a function of exact products
// and depend on no rounding.
#include "answer_device.h"
#include "answer_kernels.h"

namespace hs {
namespace {

constexpr int kThreads = 256;

__device__ __forceinline__ double block_max(double v, double* lds) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v = fmax(v, __shfl_xor(v, o, 64));
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
  __syncthreads();
  v = fmax(fmax(lds[0], lds[1]), fmax(lds[2], lds[3]));
  __syncthreads();
  return v;
}

__device__ __forceinline__ double block_sum(double v, double* lds) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
  __syncthreads();
  v = (lds[0] + lds[1]) + (lds[2] + lds[3]);
  __syncthreads();
  return v;
}

// One block per row, the row read twice, everything in 64 bits.
template <typename T>
__global__ __launch_bounds__(kThreads) void quantize_kernel(QuantizeArgs a) {
  __shared__ double lds[4];
  for (int row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const T* x = static_cast<const T*>(a.x) + int64_t(row) * a.ldx;
    int8_t* q = a.q + int64_t(row) * a.ldq;
    double top = 0.0, ss = 0.0, bad = 0.0;
    for (int i = threadIdx.x; i < a.d; i += kThreads) {
      const double v = elem(x, i);
      const double y = a.gain ? v * double(bf2f(a.gain[i])) : v;
      top = fmax(top, fabs(y));
      ss = fma(v, v, ss);
      if (!(fabs(y) < __builtin_inf())) bad = 1.0;
    }
    top = block_max(top, lds);
    ss = block_sum(ss, lds);
    bad = block_max(bad, lds);
    const bool none = bad != 0.0 || top == 0.0;
    if (threadIdx.x == 0) {
      const double r = a.gain ? 1.0 / sqrt(ss / a.d + double(a.eps)) : 1.0;
      a.scale[row] = bad != 0.0 ? __builtin_nanf("") : float(top * r / 127.0);
    }
    for (int i = threadIdx.x; i < a.d; i += kThreads) {
      const double v = elem(x, i);
      const double y = a.gain ? v * double(bf2f(a.gain[i])) : v;
      q[i] = none ? int8_t(0) : int8_t(int(rint(127.0 * y / top)));
    }
  }
}

}  // namespace

hipError_t launch_quantize(const QuantizeArgs& a, int cus, hipStream_t s) {
  if (a.rows < 1) return hipSuccess;
  const int grid = a.rows < 16 * cus ? a.rows : 16 * cus;
  switch (a.type) {
    case HS_TYPE_F32: hipLaunchKernelGGL(quantize_kernel<float>, dim3(grid), dim3(kThreads), 0, s, a); break;
    case HS_TYPE_BF16: hipLaunchKernelGGL(quantize_kernel<uint16_t>, dim3(grid), dim3(kThreads), 0, s, a); break;
    case HS_TYPE_F16: hipLaunchKernelGGL(quantize_kernel<_Float16>, dim3(grid), dim3(kThreads), 0, s, a); break;
    default: return hipErrorInvalidValue;
  }
  return hipGetLastError();
}

}  // namespace hs
