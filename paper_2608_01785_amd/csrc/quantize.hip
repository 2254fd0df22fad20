// Rows to 8-bit integers with one scale each, RMS-normalised on the way when a
// gain is given.
//
//   y = x                                   (no gain)
//   y = x / sqrt(mean(x^2) + eps) * gain    (RMSNorm)
//   a = max |y|,  scale = a / 127,  q = rint(127 y / a), ties to even
//
// The row's reciprocal root mean square scales y and a alike, so it cancels in
// q = rint(127 x g / max |x g|): the integers are a function of exact products
// (24 + 8 bits) and depend on no rounding.  They are formed in fp32 first: with
// t = fl(fl(x g) c), c = fl(127 / fl(max |x g|)), four roundings of 2^-24 put t
// within |t| 2^-22 of its exact value, so rint(t) is the answer unless t lies
// that close to a border.  Groups with such an element (one row of 3584 in
// twenty has any, of bf16 rows with a gain one in six, mostly ties) are decided
// in 64 bits afterwards: 127 x g is exact there (39 bits), and so are the borders
// (i + 1/2) a it is compared with.  Products of 16-bit values and rows without a
// gain are exact in fp32 already; fp32 rows with one are read again.
//
// The scale takes the largest product as fp32 and the sum of squares in fp32: at
// most 8 NG + W + 6 roundings on a square's way, halved by the root, and two more,
// 15 half steps for 3584 columns (the tests hold it to that).  64-bit sums would be
// two more instructions an element of a kernel that memory bounds.  Rows beyond a
// block's registers, whose sums are longer, have 64 bits.
//
// A row stays in the registers of W wavefronts from its one read to its
// store.  Rows whose products or squares leave fp32's comfortable range, or
// are not finite, take a second, plain path in 64 bits.
//
// Memory bounds it: 5 bytes an element with fp32 rows against some 15 vector
// operations.
#include "answer_device.h"
#include "answer_kernels.h"

namespace hs {
namespace {

constexpr int kVec = 8;            // elements of a lane's group
constexpr int kGroup = 64 * kVec;  // elements of a wavefront's groups

// The largest |value| as fp32 bits: an integer order that also ranks
// infinities and NaN, on top.
__device__ __forceinline__ uint32_t magnitude(float v) { return __float_as_uint(v) & 0x7fffffffu; }

template <typename T>
__device__ __forceinline__ double product(const T* x, const uint16_t* gain, int i) {
  const double v = elem(x, i);
  return gain ? v * double(bf2f(gain[i])) : v;
}

// rint(127 y / a) of exact products, ties to even.
__device__ __forceinline__ int exact_step(double y, double a) { return int(rint(127.0 * y / a)); }

// 127 v / top rounded to an integer, c = fl(127 / top); `off` reaches 1/2 where it
// needs another look.
//   16-bit values themselves (EXACT): 127 v is exact and one Newton step rounds the
//   quotient correctly.  Its distance from a tie it does not equal is 16
//   times that rounding or more (2^-21 at 1/2), so rint() is right; ties
//   are common (every v = top / 2).
//   Otherwise: |t - rint(t)| and what t may be off by reach 1/2.
template <bool EXACT>
__device__ __forceinline__ int fast_step(float v, float top, float c, float& off) {
  float t = v * c;
  if constexpr (EXACT) t = fmaf(fmaf(-t, top, 127.0f * v), c * (1.0f / 127.0f), t);
  const float i = rintf(t);
  if constexpr (!EXACT) off = fmaxf(off, fmaf(fabsf(t), 0x1.01p-22f, fabsf(t - i)));
  return int(i);
}

// rint(127 y / top) of an exact product y (32 bits or less), ties to even, from
// fast_step's guess: 127 |y| is compared with (i +- 1/2) top, which are exact.
__device__ __forceinline__ int exact_round(double y, double top, float c) {
  const double a = 127.0 * fabs(y);
  double i = rintf(fabsf(float(y)) * c);
  const bool odd = int(i) & 1;
  const double hi = (i + 0.5) * top, lo = (i - 0.5) * top;
  if (a > hi || (a == hi && odd))
    i += 1.0;
  else if (a < lo || (a == lo && odd))
    i -= 1.0;
  return int(y < 0.0 ? -i : i);
}

// Whether fast_step may take a row: false also for what is not a number.
__device__ __forceinline__ bool comfortable(float top, bool with_gain, float ss) {
  return top > 0x1p-100f && top < 0x1p100f && (!with_gain || (ss > 0x1p-80f && ss < 0x1p100f));
}

// f over the row's W wavefronts.
template <int W, typename V, typename F>
__device__ __forceinline__ V reduce_row(V v, V* lds, F f) {
  v = reduce_wave(v, f);
  if constexpr (W > 1) {
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    v = lds[0];
#pragma unroll
    for (int w = 1; w < W; ++w) v = f(v, lds[w]);
    __syncthreads();
  }
  return v;
}

template <int W>
struct RowLds {
  double d[W];
  uint32_t u[W];
  // Of quantize_kernel, rows in turn in one half and the other: a wavefront
  // that writes a half has passed a barrier behind its last reads.
  uint32_t top[2][W], near[2][W];
  float ss[2][W];
};

// The row from memory, twice, in 64 bits.
template <typename T, int W>
__device__ __forceinline__ void plain_row(const QuantizeArgs& a, const T* x, int8_t* q, int row, RowLds<W>& lds) {
  const int t = W > 1 ? int(threadIdx.x) : int(threadIdx.x & 63);
  double top = 0.0, ss = 0.0, bad = 0.0;
#pragma unroll 1
  for (int i = t; i < a.d; i += 64 * W) {
    const double v = elem(x, i), y = product(x, a.gain, i);
    top = fmax(top, fabs(y));
    ss = fma(v, v, ss);
    if (!(fabs(y) < __builtin_inf())) bad = 1.0;
  }
  auto most = [](double p, double r) { return fmax(p, r); };
  top = reduce_row<W>(top, lds.d, most);
  ss = reduce_row<W>(ss, lds.d, [](double p, double r) { return p + r; });
  bad = reduce_row<W>(bad, lds.d, most);
  const bool none = bad != 0.0 || top == 0.0;
  if (t == 0) {
    const double r = a.gain ? 1.0 / sqrt(ss / a.d + double(a.eps)) : 1.0;
    a.scale[row] = bad != 0.0 ? __builtin_nanf("") : float(top * r / 127.0);
  }
#pragma unroll 1
  for (int i = t; i < a.d; i += 64 * W) q[i] = none ? int8_t(0) : int8_t(exact_step(product(x, a.gain, i), top));
}

// Eight elements from p on, aligned as an element is.
template <typename T>
__device__ __forceinline__ void load_group(const T* p, float (&v)[kVec]) {
  u32x4 raw[sizeof(T) * kVec / 16];
  __builtin_memcpy(raw, p, sizeof(raw));
#pragma unroll
  for (int e = 0; e < kVec; ++e) {
    if constexpr (sizeof(T) == 4) {
      v[e] = __uint_as_float(raw[e >> 2][e & 3]);
    } else {
      const uint32_t w = raw[0][e >> 1];
      if constexpr (__is_same(T, uint16_t))
        v[e] = __uint_as_float((e & 1) ? w & 0xffff0000u : w << 16);
      else
        v[e] = h2f(uint16_t((e & 1) ? w >> 16 : w & 0xffffu));
    }
  }
}

__device__ __forceinline__ void store_group(int8_t* p, const int (&r)[kVec]) {
  uint32_t w[2];
#pragma unroll
  for (int h = 0; h < 2; ++h)
    w[h] = (uint32_t(r[4 * h]) & 0xffu) | (uint32_t(r[4 * h + 1]) & 0xffu) << 8 |
           (uint32_t(r[4 * h + 2]) & 0xffu) << 16 | uint32_t(r[4 * h + 3]) << 24;
  __builtin_memcpy(p, w, kVec);
}

// W wavefronts per row, NG groups per lane: d / 8 <= 64 W NG.  Group number n of a
// row is elements 8 n .. 8 n + 7; what is left of d modulo 8 goes one element
// to a lane.
template <typename T, int W, int NG, bool GAIN>
__global__ __launch_bounds__(W > 1 ? 64 * W : 256) void quantize_kernel(QuantizeArgs a) {
  constexpr int kRows = W > 1 ? 1 : 4;  // rows of a block
  constexpr bool kExact = !GAIN && sizeof(T) == 2;
  constexpr bool kLocal = !(GAIN && sizeof(T) == 4);  // products and their maximum are exact in fp32
  __shared__ RowLds<W> lds;
  const int wave = threadIdx.x >> 6;
  const int first = W > 1 ? int(threadIdx.x) : int(threadIdx.x & 63);  // the lane's first group; then 64 W on
  const int n_groups = a.d / kVec, rest = n_groups * kVec + first;
  const bool has_rest = first < a.d % kVec;
  int half = 0;
  for (int row = blockIdx.x * kRows + (W > 1 ? 0 : wave); row < a.rows; row += gridDim.x * kRows, half ^= 1) {
    const T* x = static_cast<const T*>(a.x) + int64_t(row) * a.ldx;
    int8_t* q = a.q + int64_t(row) * a.ldq;
    float y[NG][kVec], y_rest = 0.0f;
#pragma unroll
    for (int g = 0; g < NG; ++g) {
#pragma unroll
      for (int e = 0; e < kVec; ++e) y[g][e] = 0.0f;
      const int n = first + 64 * W * g;
      if (n < n_groups) load_group(x + n * kVec, y[g]);
    }
    if (has_rest) y_rest = elem(x, rest);
    float ss = 0.0f;
    uint32_t top = 0;
    if constexpr (GAIN) {
      ss = y_rest * y_rest;
      if (has_rest) y_rest *= bf2f(a.gain[rest]);
    }
    top = magnitude(y_rest);
#pragma unroll
    for (int g = 0; g < NG; ++g) {
      const int n = first + 64 * W * g;
      if constexpr (GAIN) {
        float gain[kVec] = {};
        if (n < n_groups) load_group(a.gain + n * kVec, gain);
#pragma unroll
        for (int e = 0; e < kVec; ++e) {
          ss = fmaf(y[g][e], y[g][e], ss);
          y[g][e] *= gain[e];
        }
      }
#pragma unroll
      for (int e = 0; e < kVec; ++e) top = max(top, magnitude(y[g][e]));
    }
    top = reduce_wave(top, [](uint32_t p, uint32_t r) { return max(p, r); });
    if constexpr (GAIN) ss = reduce_wave(ss, [](float p, float r) { return p + r; });
    if constexpr (W > 1) {
      if ((threadIdx.x & 63) == 0) {
        lds.top[half][wave] = top;
        lds.ss[half][wave] = ss;
      }
      __syncthreads();
      top = lds.top[half][0];
      ss = lds.ss[half][0];
#pragma unroll
      for (int w = 1; w < W; ++w) {
        top = max(top, lds.top[half][w]);
        ss += lds.ss[half][w];
      }
    }
    const float top32 = __uint_as_float(top);
    if (!comfortable(top32, GAIN, ss)) {
      plain_row<T, W>(a, x, q, row, lds);
      continue;
    }
    if (first == 0) {
      const double r = GAIN ? 1.0 / sqrt(double(ss) / a.d + double(a.eps)) : 1.0;
      a.scale[row] = float(double(top32) * r / 127.0);
    }
    const float c = 127.0f / top32;
    uint32_t near = 0;  // groups to decide again; bit NG: the rest
#pragma unroll
    for (int g = 0; g < NG; ++g) {
      const int n = first + 64 * W * g;
      int r[kVec];
      float off = 0.0f;
#pragma unroll
      for (int e = 0; e < kVec; ++e) r[e] = fast_step<kExact>(y[g][e], top32, c, off);
      near |= uint32_t(off >= 0.5f) << g;
      if (n < n_groups) store_group(q + n * kVec, r);
    }
    if (has_rest) {
      float off = 0.0f;
      q[rest] = int8_t(fast_step<kExact>(y_rest, top32, c, off));
      near |= uint32_t(off >= 0.5f) << NG;
    }
    if constexpr (kExact) continue;
    double exact = top32;
    if constexpr (!kLocal) {
      uint32_t any = __ballot(near != 0) != 0;
      if constexpr (W > 1) {
        if ((threadIdx.x & 63) == 0) lds.near[half][wave] = any;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < W; ++w) any |= lds.near[half][w];
      }
      if (!any) continue;
      // The exact maximum.
      exact = has_rest ? fabs(product(x, a.gain, rest)) : 0.0;
#pragma unroll 1
      for (int n = first; n < n_groups; n += 64 * W) {
        float v[kVec], gain[kVec];
        load_group(x + n * kVec, v);
        load_group(a.gain + n * kVec, gain);
#pragma unroll
        for (int e = 0; e < kVec; ++e) exact = fmax(exact, fabs(double(v[e]) * double(gain[e])));
      }
      exact = reduce_row<W>(exact, lds.d, [](double p, double r) { return fmax(p, r); });
    }
    // The groups in doubt, from memory.
    if (near >> NG) q[rest] = int8_t(exact_round(product(x, a.gain, rest), exact, c));
    near &= (1u << NG) - 1;
#pragma unroll 1
    while (near) {
      const int n = first + 64 * W * __builtin_ctz(near);
      near &= near - 1;
      float v[kVec], gain[kVec];
      int r[kVec];
      load_group(x + n * kVec, v);
      if constexpr (GAIN) load_group(a.gain + n * kVec, gain);
#pragma unroll
      for (int e = 0; e < kVec; ++e)
        r[e] = exact_round(GAIN ? double(v[e]) * double(gain[e]) : double(v[e]), exact, c);
      store_group(q + n * kVec, r);
    }
  }
}

// Rows of at most 8 LR elements, LR lanes each: a wavefront has 64 / LR of them.
// 50000 x 64 fp32 with a gain: 6.8 us, 23 with a wavefront a row; 500000 x 256:
// 132 us (4.9 TB/s), 203.
template <typename T, int LR, bool GAIN>
__global__ __launch_bounds__(256) void quantize_narrow_kernel(QuantizeArgs a) {
  constexpr int kRows = 256 / LR;  // of a block
  constexpr bool kExact = !GAIN && sizeof(T) == 2;
  __shared__ RowLds<1> lds;  // not used by one wavefront
  auto reduce = [](auto v, auto f) {
    v = f(v, xor_lane<1>(v));
    v = f(v, xor_lane<2>(v));
    v = f(v, xor_lane<4>(v));
    if constexpr (LR > 8) v = f(v, xor_lane<8>(v));
    if constexpr (LR > 16) v = f(v, xor_lane<16>(v));
    return v;
  };
  const int first = threadIdx.x % LR, at = first * kVec, rest = a.d / kVec * kVec + first;
  const bool has_group = at + kVec <= a.d, has_rest = first < a.d % kVec;
  float gain[kVec] = {}, gain_rest = 0.0f;  // the same for all its rows
  if constexpr (GAIN) {
    if (has_group) load_group(a.gain + at, gain);
    if (has_rest) gain_rest = bf2f(a.gain[rest]);
  }
  for (int row0 = blockIdx.x * kRows; row0 < a.rows; row0 += gridDim.x * kRows) {
    const int row = row0 + int(threadIdx.x) / LR;
    const bool valid = row < a.rows;
    const T* x = static_cast<const T*>(a.x) + int64_t(row) * a.ldx;
    int8_t* q = a.q + int64_t(row) * a.ldq;
    float v[kVec] = {}, v_rest = 0.0f, ss = 0.0f;
    if (valid && has_group) load_group(x + at, v);
    if (valid && has_rest) v_rest = elem(x, rest);
    auto y = [&](int e) { return GAIN ? v[e] * gain[e] : v[e]; };
    const float y_rest = GAIN ? v_rest * gain_rest : v_rest;
    uint32_t top = magnitude(y_rest);
    if constexpr (GAIN) ss = v_rest * v_rest;
#pragma unroll
    for (int e = 0; e < kVec; ++e) {
      if constexpr (GAIN) ss = fmaf(v[e], v[e], ss);
      top = max(top, magnitude(y(e)));
    }
    top = reduce(top, [](uint32_t p, uint32_t r) { return max(p, r); });
    if constexpr (GAIN) ss = reduce(ss, [](float p, float r) { return p + r; });
    const float top32 = __uint_as_float(top), c = 127.0f / top32;
    const bool fast = valid && comfortable(top32, GAIN, ss);
    float off = 0.0f;
    if (fast) {
      if (first == 0) {
        const double r = GAIN ? 1.0 / sqrt(double(ss) / a.d + double(a.eps)) : 1.0;
        a.scale[row] = float(double(top32) * r / 127.0);
      }
      int r[kVec];
#pragma unroll
      for (int e = 0; e < kVec; ++e) r[e] = fast_step<kExact>(y(e), top32, c, off);
      if (has_group) store_group(q + at, r);
      if (has_rest) q[rest] = int8_t(fast_step<kExact>(y_rest, top32, c, off));
    }
    if constexpr (!kExact) {
      if (__ballot(off >= 0.5f)) {
        // The exact maxima, then the lanes in doubt.
        double exact = fabs(double(v_rest) * (GAIN ? double(gain_rest) : 1.0));
#pragma unroll
        for (int e = 0; e < kVec; ++e) exact = fmax(exact, fabs(double(v[e]) * (GAIN ? double(gain[e]) : 1.0)));
        exact = reduce(exact, [](double p, double r) { return fmax(p, r); });
        if (off >= 0.5f) {
          int r[kVec];
#pragma unroll
          for (int e = 0; e < kVec; ++e) r[e] = exact_step(double(v[e]) * (GAIN ? double(gain[e]) : 1.0), exact);
          if (has_group) store_group(q + at, r);
          if (has_rest) q[rest] = int8_t(exact_step(double(v_rest) * (GAIN ? double(gain_rest) : 1.0), exact));
        }
      }
    }
    // The others one after another, a wavefront for each.
    for (uint64_t slow = __ballot(valid && !fast && first == 0); slow != 0; slow &= slow - 1) {
      const int other = row0 + (int(threadIdx.x) / 64 * 64 + __builtin_ctzll(slow)) / LR;
      plain_row<T, 1>(a, static_cast<const T*>(a.x) + int64_t(other) * a.ldx, a.q + int64_t(other) * a.ldq, other, lds);
    }
  }
}

// Rows longer than a block's registers: read twice, the second time from a cache.
// With the exact maximum at hand a group in doubt is decided at once.  300 x
// 131072 fp32 with a gain: 77 us, 593 on the plain path.
template <typename T, bool GAIN>
__global__ __launch_bounds__(512) void quantize_long_kernel(QuantizeArgs a) {
  constexpr int W = 8;
  constexpr bool kExact = !GAIN && sizeof(T) == 2;
  __shared__ RowLds<W> lds;
  const int first = threadIdx.x, n_groups = a.d / kVec, rest = n_groups * kVec + first;
  const bool has_rest = first < a.d % kVec;
  for (int row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const T* x = static_cast<const T*>(a.x) + int64_t(row) * a.ldx;
    int8_t* q = a.q + int64_t(row) * a.ldq;
    auto load = [&](int n, float (&v)[kVec], float (&gain)[kVec]) {
      load_group(x + n * kVec, v);
      if constexpr (GAIN) load_group(a.gain + n * kVec, gain);
    };
    uint32_t top = 0;
    double ss = 0.0, exact = 0.0;  // sums of more elements than fp32 adds up well
    if (has_rest) {
      const double y = product(x, a.gain, rest), v = elem(x, rest);
      ss = v * v;
      exact = fabs(y);
      top = magnitude(GAIN ? elem(x, rest) * bf2f(a.gain[rest]) : elem(x, rest));
    }
    for (int n = first; n < n_groups; n += 64 * W) {
      float v[kVec], gain[kVec], sum = 0.0f;
      load(n, v, gain);
#pragma unroll
      for (int e = 0; e < kVec; ++e) {
        if constexpr (GAIN) {
          sum = fmaf(v[e], v[e], sum);
          exact = fmax(exact, fabs(double(v[e]) * double(gain[e])));
        }
        top = max(top, magnitude(GAIN ? v[e] * gain[e] : v[e]));
      }
      ss += sum;
    }
    top = reduce_row<W>(top, lds.u, [](uint32_t p, uint32_t r) { return max(p, r); });
    if constexpr (GAIN) {
      ss = reduce_row<W>(ss, lds.d, [](double p, double r) { return p + r; });
      exact = reduce_row<W>(exact, lds.d, [](double p, double r) { return fmax(p, r); });
    }
    const float top32 = __uint_as_float(top);
    if (!comfortable(top32, GAIN, float(ss))) {
      plain_row<T, W>(a, x, q, row, lds);
      continue;
    }
    if constexpr (!GAIN) exact = top32;
    if (first == 0) {
      const double r = GAIN ? 1.0 / sqrt(ss / a.d + double(a.eps)) : 1.0;
      a.scale[row] = float(exact * r / 127.0);
    }
    const float c = 127.0f / top32;
    for (int n = first; n < n_groups; n += 64 * W) {
      float v[kVec], gain[kVec], off = 0.0f;
      int i[kVec];
      load(n, v, gain);
#pragma unroll
      for (int e = 0; e < kVec; ++e) i[e] = fast_step<kExact>(GAIN ? v[e] * gain[e] : v[e], top32, c, off);
      if (off >= 0.5f)
#pragma unroll
        for (int e = 0; e < kVec; ++e)
          i[e] = exact_round(GAIN ? double(v[e]) * double(gain[e]) : double(v[e]), exact, c);
      store_group(q + n * kVec, i);
    }
    if (has_rest) q[rest] = int8_t(exact_step(product(x, a.gain, rest), exact));
  }
}

template <typename T, int W, int NG>
hipError_t launch(const QuantizeArgs& a, int cus, hipStream_t s) {
  constexpr int kRows = W > 1 ? 1 : 4, kThreads = W > 1 ? 64 * W : 256;
  const int64_t blocks = (int64_t(a.rows) + kRows - 1) / kRows;
  const int64_t most = int64_t(cus) * 16;
  const unsigned grid = unsigned(blocks < most ? blocks : most);
  if (a.gain)
    hipLaunchKernelGGL((quantize_kernel<T, W, NG, true>), dim3(grid), dim3(kThreads), 0, s, a);
  else
    hipLaunchKernelGGL((quantize_kernel<T, W, NG, false>), dim3(grid), dim3(kThreads), 0, s, a);
  return hipGetLastError();
}

template <typename T, int LR>
hipError_t launch_narrow(const QuantizeArgs& a, int cus, hipStream_t s) {
  const int64_t blocks = (int64_t(a.rows) * LR + 255) / 256, most = int64_t(cus) * 16;
  const unsigned grid = unsigned(blocks < most ? blocks : most);
  if (a.gain)
    hipLaunchKernelGGL((quantize_narrow_kernel<T, LR, true>), dim3(grid), dim3(256), 0, s, a);
  else
    hipLaunchKernelGGL((quantize_narrow_kernel<T, LR, false>), dim3(grid), dim3(256), 0, s, a);
  return hipGetLastError();
}

template <typename T>
hipError_t launch_type(const QuantizeArgs& a, int cus, hipStream_t s) {
  if (a.d <= 64) return launch_narrow<T, 8>(a, cus, s);
  if (a.d <= 128) return launch_narrow<T, 16>(a, cus, s);
  if (a.d <= 256) return launch_narrow<T, 32>(a, cus, s);
  // Two groups a lane, with wavefronts enough for the row, keep the most loads
  // in flight: 10515 x 3584 fp32 takes 37 us in 4 x 2 (5.1 TB/s), 44 in 2 x 4
  // and 51 in 1 x 8.  Past four wavefronts the joins cost more than more
  // groups do: 9000 x 4096 fp32 36 us in 4 x 2, 55 in 8 x 2; 3000 x 18944
  // fp32 72 us in 8 x 5, 86 in 16 x 3, 92 in 4 x 10 (both with three barriers
  // a row more, which were 8 us in 8 x 5).  Short rows need one (30000 x 1024
  // fp32: 31 us in 1 x 2, 36 in 2 x 1).  Few rows take 6 us in any of them.
  const int groups = (a.d / kVec + 63) / 64;  // per wavefront if it were one; the rest rides along
  if (groups <= 1) return launch<T, 1, 1>(a, cus, s);
  if (groups <= 2) return launch<T, 1, 2>(a, cus, s);
  if (groups <= 4) return launch<T, 2, 2>(a, cus, s);
  if (groups <= 8) return launch<T, 4, 2>(a, cus, s);
  if (groups <= 16) return launch<T, 4, 4>(a, cus, s);
  if (groups <= 32) return launch<T, 8, 4>(a, cus, s);
  if (groups <= 40) return launch<T, 8, 5>(a, cus, s);
  if (groups <= 64) return launch<T, 16, 4>(a, cus, s);
  const int grid = a.rows < 16 * cus ? a.rows : 16 * cus;
  if (a.gain)
    hipLaunchKernelGGL((quantize_long_kernel<T, true>), dim3(grid), dim3(512), 0, s, a);
  else
    hipLaunchKernelGGL((quantize_long_kernel<T, false>), dim3(grid), dim3(512), 0, s, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_quantize(const QuantizeArgs& a, int cus, hipStream_t s) {
  if (a.rows < 1) return hipSuccess;
  switch (a.type) {
    case HS_TYPE_F32: return launch_type<float>(a, cus, s);
    case HS_TYPE_BF16: return launch_type<uint16_t>(a, cus, s);
    case HS_TYPE_F16: return launch_type<_Float16>(a, cus, s);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace hs
