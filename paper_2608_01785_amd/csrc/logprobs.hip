// Log probabilities of given tokens, entropy and top alternatives of rows of
// logits z:
//   m = max z,  S = sum e^(z - m),  log p[t] = z[t] - m - log S,
//   H = log S - sum e^(z - m) (z - m) / S
// Alternatives are ordered by logit, equal ones by the lower token.
#include "answer_device.h"
#include "answer_kernels.h"

namespace hs {
namespace {

constexpr int kThreads = 256;

// Larger for the logit that is listed first: the value's order (-0 as +0),
// then the lower token.  0: no token.
__device__ __forceinline__ uint64_t order_key(float z, uint32_t token) {
  const uint32_t b = __float_as_uint(z + 0.0f);
  const uint32_t o = (b & 0x80000000u) ? ~b : (b | 0x80000000u);
  return (uint64_t(o) << 32) | (0xffffffffu - token);
}

template <typename V, typename F>
__device__ __forceinline__ V block_reduce(V v, V* lds, F f) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v = f(v, V(__shfl_xor(v, o, 64)));
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
  __syncthreads();
  v = f(f(lds[0], lds[1]), f(lds[2], lds[3]));
  __syncthreads();
  return v;
}

// One block per row, the row read again for the sums and for each alternative.
template <typename T>
__global__ __launch_bounds__(kThreads) void logprobs_kernel(LogprobsArgs a) {
  __shared__ double lds[4];
  __shared__ unsigned long long keys[4];
  auto add = [](double x, double y) { return x + y; };
  auto most = [](double x, double y) { return fmax(x, y); };
  auto first = [](unsigned long long x, unsigned long long y) { return x > y ? x : y; };
  for (int row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const T* z = static_cast<const T*>(a.logits) + int64_t(row) * a.ld;
    double m = -__builtin_inf(), bad = 0.0;
    for (int i = threadIdx.x; i < a.vocab; i += kThreads) {
      const float v = elem(z, i);
      m = fmax(m, double(v));
      if (!(v < __builtin_inff())) bad = 1.0;
    }
    m = block_reduce(m, lds, most);
    bad = block_reduce(bad, lds, most);
    const bool none = m == -__builtin_inf();
    double s = 0.0, t = 0.0;
    for (int i = threadIdx.x; i < a.vocab; i += kThreads) {
      const float v = elem(z, i);
      if (v == -__builtin_inff()) continue;
      const double d = double(v) - m, e = exp(d);
      s += e;
      t += e * d;
    }
    s = block_reduce(s, lds, add);
    t = block_reduce(t, lds, add);
    const double log_s = none ? 0.0 : log(s);
    const float nan = __builtin_nanf("");
    auto logp = [&](float v) {
      return bad != 0.0 ? nan : v == -__builtin_inff() ? v : float(double(v) - m - log_s);
    };
    if (threadIdx.x == 0 && a.entropy) a.entropy[row] = bad != 0.0 ? nan : none ? 0.0f : float(log_s - t / s);
    for (int j = threadIdx.x; j < a.n_tokens; j += kThreads) {
      const int64_t o = int64_t(row) * a.n_tokens + j;
      const int tok = a.tokens[o];
      a.token_lp[o] = tok == -1 ? 0.0f : (tok < 0 || tok >= a.vocab) ? nan : logp(elem(z, tok));
    }
    unsigned long long last = ~0ull;
    for (int j = 0; j < a.top_k; ++j) {
      unsigned long long best = 0;
      for (int i = threadIdx.x; i < a.vocab && last; i += kThreads) {
        const float v = elem(z, i);
        if (v == -__builtin_inff()) continue;
        const unsigned long long k = order_key(v, i);
        if (k < last && k > best) best = k;
      }
      last = block_reduce(best, keys, first);
      if (threadIdx.x == 0) {
        const int64_t o = int64_t(row) * a.top_k + j;
        const int tok = int(0xffffffffu - uint32_t(last));
        const bool listed = last != 0 && bad == 0.0;
        a.top_tokens[o] = listed ? tok : -1;
        a.top_lp[o] = bad != 0.0 ? nan : listed ? logp(elem(z, tok)) : -__builtin_inff();
      }
    }
  }
}

}  // namespace

hipError_t launch_logprobs(const LogprobsArgs& a, int cus, hipStream_t s) {
  if (a.rows < 1) return hipSuccess;
  const int grid = a.rows < 8 * cus ? a.rows : 8 * cus;
  switch (a.type) {
    case HS_TYPE_F32: hipLaunchKernelGGL(logprobs_kernel<float>, dim3(grid), dim3(kThreads), 0, s, a); break;
    case HS_TYPE_BF16: hipLaunchKernelGGL(logprobs_kernel<uint16_t>, dim3(grid), dim3(kThreads), 0, s, a); break;
    case HS_TYPE_F16: hipLaunchKernelGGL(logprobs_kernel<_Float16>, dim3(grid), dim3(kThreads), 0, s, a); break;
    default: return hipErrorInvalidValue;
  }
  return hipGetLastError();
}

}  // namespace hs
