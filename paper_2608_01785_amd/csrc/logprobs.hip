// Log probabilities of given tokens, entropy and top alternatives of rows of
// logits z, in one read of them:
//   m = max z,  S = sum e^(z - m),  log p[t] = z[t] - m - log S,
//   H = log S - T / S,  T = sum e^(z - m) (z - m)
// Alternatives are ordered by logit, equal ones by the lower token.
//
// A wavefront keeps a running m, and each of its lanes the sums of its elements
// against it: S, T, and F, which is S without the elements at m themselves, so
// that log S = log1p(F) keeps its digits where one token has nearly all the
// probability.  A 4 KB chunk of a row sits in the wavefront's registers: its
// maximum first, then e^(z - m) of each element.  Vector instructions bound it
// (the exponential alone takes four issue slots), so the usual chunk, all of
// it below m, takes the shortest form: y = z log2(e) - M in one operation with
// M = m log2(e) rounded, whose rounding error is a factor common to the
// chunk's sums.  Only a chunk that reaches m (one in c of the first c), or comes
// under an m beyond 2^20, keeps F apart and takes exact differences.
//
// Alternatives cost the loop over the chunks next to nothing: every lane leaves
// the maximum of its elements of each chunk in LDS.  At the end 64 or 256
// maxima of disjoint parts of the row give a value that at least top_k of them
// reach (and few elements more: 24 to be expected for 20), the lanes' maxima
// that reach it name the words to read again, and what reaches it there leaves
// a key (order of the value, then the lower token).  The keys are ranked by
// counting the larger ones.  Where too many elements share the last value, as
// in a row of equal logits, the wavefront goes through its chunks once more:
// every 64 keys are sorted over the lanes and merged into a list of the 64
// best, which raises the bound.
#include "answer_device.h"
#include "answer_kernels.h"

namespace hs {
namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kLowest = -3.4028234663852886e38f;  // running maximum before any element
constexpr float kInf = __builtin_inff();
constexpr float kFar = -200.0f;  // e^-200 is 0 in fp32: differences are clamped here where 0 * -inf could arise
// Maxima up to here take the short form of a lower chunk: what rounding m log2(e)
// takes off is then at most 2^-4, and its power of two next to 1.  It grows with
// m, past 2^128 from |m| of some 10^9 on, and such a factor times a sum of 0 is NaN.
constexpr float kFarMaximum = 0x1p20f;

// ---------------------------------------------------------------- running sums

struct Sums {
  float m, s, f, t;  // maximum, S, S without the elements at the maximum, T
};

__device__ __forceinline__ float exp_of(float d) { return exp2_raw(d * kLog2e); }

// The sums against a maximum m >= a.m.
__device__ __forceinline__ void rescale(Sums& a, float m) {
  const float d = fmaxf(a.m - m, kFar), f = exp_of(d), s = a.s * f;
  a.f = a.m < m ? s : a.f;
  a.t = fmaf(s, d, f * a.t);
  a.s = s;
  a.m = m;
}

// ---------------------------------------------------------------- lanes

__device__ __forceinline__ float max_wave(float v) {
  return reduce_wave(v, [](float a, float b) { return fmaxf(a, b); });
}
__device__ __forceinline__ float sum_wave(float v) {
  return reduce_wave(v, [](float a, float b) { return a + b; });
}

// Lanes of the mask below this one.
__device__ __forceinline__ int lanes_before(uint64_t mask) {
  return int(__builtin_amdgcn_mbcnt_hi(uint32_t(mask >> 32), __builtin_amdgcn_mbcnt_lo(uint32_t(mask), 0)));
}

// One stage of a bitonic network over the 64 lanes: lane pairs J apart, the
// larger value to the lower lane where `down`.
template <int J, typename V>
__device__ __forceinline__ V stage(V v, bool down) {
  const V o = xor_lane<J>(v);
  const bool keep_large = ((threadIdx.x & J) == 0) == down;
  if constexpr (sizeof(V) == 4) {
    const V large = max(v, o), small = min(v, o);
    return keep_large ? large : small;
  } else {
    return (v > o) == keep_large ? v : o;
  }
}
template <int J, typename V>
__device__ __forceinline__ V merge_stages(V v, bool down) {
  v = stage<J>(v, down);
  if constexpr (J > 1) v = merge_stages<J / 2>(v, down);
  return v;
}
// Sorted, largest in lane 0.
template <typename V>
__device__ __forceinline__ V sort_wave(V v) {
  const int l = threadIdx.x;
  v = merge_stages<1>(v, (l & 2) == 0);
  v = merge_stages<2>(v, (l & 4) == 0);
  v = merge_stages<4>(v, (l & 8) == 0);
  v = merge_stages<8>(v, (l & 16) == 0);
  v = merge_stages<16>(v, (l & 32) == 0);
  return merge_stages<32>(v, true);
}
// The 64 largest of two sorted lists, sorted.
__device__ __forceinline__ uint64_t merge_lists(uint64_t a, uint64_t b) {
  const uint64_t r = __shfl(b, 63 - int(threadIdx.x & 63), 64);
  return merge_stages<32>(a > r ? a : r, true);
}

// ---------------------------------------------------------------- keys

// Larger for the logit that is listed first: the value's order (-0 as +0),
// then the lower token.  Masked tokens never get a key; 0 is no token.
__device__ __forceinline__ uint32_t order_of(float z) {
  const uint32_t b = __float_as_uint(z + 0.0f);
  return b ^ (uint32_t(int32_t(b) >> 31) | 0x80000000u);
}
__device__ __forceinline__ uint64_t key_of(float z, uint32_t token) {
  return (uint64_t(order_of(z)) << 32) | (0xffffffffu - token);
}
__device__ __forceinline__ float value_of(uint64_t key) {
  const uint32_t o = uint32_t(key >> 32);
  return __uint_as_float((o & 0x80000000u) ? o ^ 0x80000000u : ~o);
}
__device__ __forceinline__ int token_of(uint64_t key) { return int(0xffffffffu - uint32_t(key)); }

constexpr int kBuffer = 128;  // keys of a wavefront in LDS: 63 left over and 64 new

// One wavefront's best keys.
struct Best {
  uint64_t list = 0;   // lane i: the i-th best of those merged so far
  uint64_t kth;        // a candidate's key must exceed this
  float above;         // so its value must be at least this
  int count = 0;       // keys in the buffer
  bool merged = false;
  int k;
  uint64_t* buf;

  __device__ __forceinline__ void init(int top_k, uint64_t* lds) {
    k = top_k;
    buf = lds;
    kth = key_of(-kInf, 0);  // above every masked token
    above = kLowest;
  }
  // At least top_k elements reach v.
  __device__ __forceinline__ void bound(float v) {
    const uint64_t key = (uint64_t(order_of(v)) << 32) - 1;
    if (key > kth) {
      kth = key;
      above = v;
    }
  }
  __device__ __forceinline__ void absorb(uint64_t key) {
    list = merge_lists(list, sort_wave(key));
    merged = true;
    const uint64_t last = (uint64_t(__builtin_amdgcn_readlane(uint32_t(list >> 32), k - 1)) << 32) |
                          uint32_t(__builtin_amdgcn_readlane(uint32_t(list), k - 1));
    if (last > kth) {
      // Elements still to come have higher tokens than those in the list, so
      // one that only equals the k-th value loses: the next value up is the
      // least to look at.
      kth = last;
      above = value_of(last + (uint64_t(1) << 32));
    }
  }
  // Every lane offers a key (0: none).
  __device__ __forceinline__ void offer(uint64_t key) {
    const bool take = key > kth;
    const uint64_t mask = __ballot(take);
    const int at = count + lanes_before(mask);
    if (take) buf[at] = key;
    count += __popcll(mask);
  }
  // Merges the first 64 keys of the buffer, or what there is.
  __device__ __forceinline__ void settle() {
    const int lane = threadIdx.x & 63;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    const uint64_t first = lane < count ? buf[lane] : 0, rest = buf[64 + lane];
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    count = max(count - 64, 0);
    if (lane < count) buf[lane] = rest;
    absorb(first);
  }
  // Leaves the wavefront's candidates, at most 127, in the buffer; returns their number.
  __device__ __forceinline__ int finish() {
    if (!merged) return count;
    const int lane = threadIdx.x & 63;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    buf[lane] = list;
    return min(k, __popcll(__ballot(list != 0)));
  }
};

// How many of the n keys at p (16-byte aligned) are larger.
__device__ __forceinline__ int rank_among(const uint64_t* p, int n, uint64_t key) {
  auto two = [&](int j) {
    const u32x4 v = *reinterpret_cast<const u32x4*>(p + j);
    return int((uint64_t(v[1]) << 32 | v[0]) > key) + int((uint64_t(v[3]) << 32 | v[2]) > key);
  };
  int r = 0, j = 0;
  for (; j + 8 <= n; j += 8) r += (two(j) + two(j + 2)) + (two(j + 4) + two(j + 6));
  for (; j + 2 <= n; j += 2) r += two(j);
  if (j < n) r += p[j] > key;
  return r;
}

// ---------------------------------------------------------------- chunks

// The 16-byte word at element i of a row [first, last), masked outside it (a
// word that the row shares with others is read whole).
template <typename T>
__device__ __forceinline__ u32x4 edge_word(const T* p, int64_t i, int64_t first, int64_t last) {
  constexpr int kVec = 16 / sizeof(T);
  constexpr uint32_t masked = sizeof(T) == 4 ? 0xff800000u : __is_same(T, uint16_t) ? 0xff80ff80u : 0xfc00fc00u;
  u32x4 raw = {masked, masked, masked, masked};
  if (i + kVec <= first || i >= last) return raw;
  const u32x4 v = *reinterpret_cast<const u32x4*>(p + i);
  // Elements lo .. hi - 1 of the word belong to the row.
  const int lo = int(first > i ? first - i : 0), hi = int(last - i < kVec ? last - i : kVec);
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    uint32_t keep;
    if constexpr (sizeof(T) == 4)
      keep = (w >= lo && w < hi) ? ~0u : 0u;
    else
      keep = ((2 * w >= lo && 2 * w < hi) ? 0xffffu : 0u) |
             ((2 * w + 1 >= lo && 2 * w + 1 < hi) ? 0xffff0000u : 0u);
    raw[w] = (v[w] & keep) | (masked & ~keep);
  }
  return raw;
}

template <typename T>
struct Chunk {
  static constexpr int kVec = 16 / sizeof(T);     // elements of a 16-byte load
  static constexpr int kLane = 4 * kVec;          // elements of a lane
  static constexpr int kSize = 64 * kLane;
  u32x4 raw[4];

  // Element e of load l of a lane, as fp32.
  __device__ __forceinline__ float get(int l, int e) const {
    if constexpr (sizeof(T) == 4) {
      return __uint_as_float(raw[l][e]);
    } else {
      const uint32_t w = raw[l][e >> 1];
      if constexpr (__is_same(T, uint16_t))
        return __uint_as_float((e & 1) ? w & 0xffff0000u : w << 16);
      else
        return h2f(uint16_t((e & 1) ? w >> 16 : w & 0xffffu));
    }
  }
  // Element j of the lane, whose j is its own: registers cannot be indexed.
  __device__ __forceinline__ float pick(int j) const {
    const int w = sizeof(T) == 4 ? j : j >> 1;
    auto of_load = [&](const u32x4& v) {
      const uint32_t lo = (w & 1) ? v[1] : v[0], hi = (w & 1) ? v[3] : v[2];
      return (w & 2) ? hi : lo;
    };
    const uint32_t lo = (w & 4) ? of_load(raw[1]) : of_load(raw[0]), hi = (w & 4) ? of_load(raw[3]) : of_load(raw[2]);
    const uint32_t v = (w & 8) ? hi : lo;
    if constexpr (sizeof(T) == 4) {
      return __uint_as_float(v);
    } else {
      const uint32_t half = (j & 1) ? v >> 16 : v & 0xffffu;
      if constexpr (__is_same(T, uint16_t))
        return __uint_as_float(half << 16);
      else
        return h2f(uint16_t(half));
    }
  }
  // `p`: the row's 16-byte aligned origin; all of chunk c lies in the row.
  __device__ __forceinline__ void load(const T* p, int64_t c) {
    const T* q = p + c * kSize + (threadIdx.x & 63) * kVec;
#pragma unroll
    for (int l = 0; l < 4; ++l) raw[l] = *reinterpret_cast<const u32x4*>(q + l * 64 * kVec);
  }
  // The same where the chunk reaches past the row [first, last): masked there.
  __device__ void load_edge(const T* p, int64_t c, int64_t first, int64_t last) {
#pragma unroll
    for (int l = 0; l < 4; ++l)
      raw[l] = edge_word(p, c * kSize + (l * 64 + (threadIdx.x & 63)) * kVec, first, last);
  }
};

// One row as its 16-byte aligned origin and the range of it that the row holds.
template <typename T>
struct Row {
  const T* p;
  int64_t first, last;
  int chunks;
  __device__ __forceinline__ Row(const LogprobsArgs& a, int row) {
    const T* z = static_cast<const T*>(a.logits) + int64_t(row) * a.ld;
    first = (reinterpret_cast<uintptr_t>(z) & 15) / sizeof(T);
    p = z - first;
    last = first + a.vocab;
    chunks = int((last + Chunk<T>::kSize - 1) / Chunk<T>::kSize);
  }
  __device__ __forceinline__ void load(Chunk<T>& c, int i) const {
    if (int64_t(i) * Chunk<T>::kSize >= first && int64_t(i + 1) * Chunk<T>::kSize <= last)
      c.load(p, i);
    else
      c.load_edge(p, i, first, last);
  }
};

// A wavefront's sums: m is the same in every lane, the others are the lane's own.
struct Running {
  Sums a{kLowest, 0.0f, 0.0f, 0.0f};
  float scaled = 0.0f;  // M = m log2(e), rounded
  float delta = 0.0f;   // what the rounding took off: m log2(e) - M
  float fix = 1.0f;     // 2^-delta

  // The chunk's elements; `top` is its largest over all lanes.
  template <typename T>
  __device__ __forceinline__ void add(const Chunk<T>& c, float top) {
    constexpr int V = Chunk<T>::kVec;
    float s[4] = {}, f[4] = {}, t[4] = {};
    if (top >= a.m || fabsf(a.m) > kFarMaximum) {
      if (top > a.m) {
        rescale(a, top);
        scaled = a.m * kLog2e;
        delta = fmaf(a.m, kLog2e, -scaled);
        fix = exp2_raw(-delta);
      }
#pragma unroll
      for (int l = 0; l < 4; ++l)
#pragma unroll
        for (int e = 0; e < V; ++e) {
          const float d = c.get(l, e) - a.m, x = exp_of(d);
          s[e & 3] += x;
          f[e & 3] += __builtin_amdgcn_fractf(x);  // 0 where x is 1
          t[e & 3] = fmaf(x, fmaxf(d, kFar), t[e & 3]);
        }
      a.s += (s[0] + s[1]) + (s[2] + s[3]);
      a.f += (f[0] + f[1]) + (f[2] + f[3]);
      a.t += (t[0] + t[1]) + (t[2] + t[3]);
    } else {
#pragma unroll
      for (int l = 0; l < 4; ++l)
#pragma unroll
        for (int e = 0; e < V; ++e) {
          const float y = fmaf(c.get(l, e), kLog2e, -scaled), x = exp2_raw(y);
          s[e & 3] += x;
          t[e & 3] = fmaf(x, fmaxf(y, 2 * kFar), t[e & 3]);
        }
      const float sum = (s[0] + s[1]) + (s[2] + s[3]);
      const float weighted = fmaf(-delta, sum, (t[0] + t[1]) + (t[2] + t[3]));
      a.s = fmaf(sum, fix, a.s);
      a.f = fmaf(sum, fix, a.f);
      a.t = fmaf(weighted, fix * kLn2, a.t);
    }
  }
  __device__ __forceinline__ Sums total() const { return Sums{a.m, sum_wave(a.s), sum_wave(a.f), sum_wave(a.t)}; }
};

// Lane maxima of the four loads.
template <typename T>
__device__ __forceinline__ f32x4 tops_of(const Chunk<T>& c) {
  f32x4 top;
#pragma unroll
  for (int l = 0; l < 4; ++l) {
    top[l] = c.get(l, 0);
#pragma unroll
    for (int e = 1; e < Chunk<T>::kVec; ++e) top[l] = fmaxf(top[l], c.get(l, e));
  }
  return top;
}

// The chunk's elements that may be among the best.  A lane offers one at a
// time, from a copy of the chunk in LDS since registers cannot be indexed
// (read again from memory it would wait for the next chunk's loads as well).
// After the last chunk a list that has been started takes the rest of the
// buffer.
template <typename T>
__device__ __forceinline__ void offer_chunk(const Chunk<T>& c, const f32x4& tops, const Row<T>& row, int i, bool last,
                                            Best& best, u32x4 (*copy)[4]) {
  constexpr int V = Chunk<T>::kVec;
  const int lane = threadIdx.x & 63;
  uint32_t hits = 0;
#pragma unroll
  for (int l = 0; l < 4; ++l) {
    if (!__ballot(tops[l] >= best.above)) continue;
    copy[lane][l] = c.raw[l];
#pragma unroll
    for (int e = 0; e < V; ++e) hits |= uint32_t(c.get(l, e) >= best.above) << (l * V + e);
  }
  const int at0 = i * Chunk<T>::kSize + lane * V - int(row.first);  // token of the lane's element 0
  while (true) {
    const bool more = __ballot(hits != 0) != 0;
    if (more) {
      uint64_t key = 0;
      if (hits) {
        const int j = __builtin_ctz(hits);
        hits &= hits - 1;
        const float z = elem(reinterpret_cast<const T*>(copy[lane]), j);
        // Outside the row a chunk holds masked elements.
        if (z > -kInf) key = key_of(z, at0 + (j / V) * 64 * V + j % V);
      }
      best.offer(key);
    }
    if (best.count >= 64 || (!more && last && best.merged && best.count > 0))
      best.settle();
    else if (!more)
      break;
  }
}

// ---------------------------------------------------------------- results

__device__ __forceinline__ float log_sum(const Sums& a) { return a.s < 1.5f ? log1pf(a.f) : logf(a.s); }

// A row's log probabilities from its sums.
struct Answer {
  float m = 0.0f, log_s = 0.0f;
  bool bad = false, none = false;
  __device__ Answer() = default;
  __device__ __forceinline__ explicit Answer(const Sums& a)
      : m(a.m), log_s(0.0f), bad(a.s != a.s), none(a.s == 0.0f) {
    if (!none) log_s = log_sum(a);
  }
  __device__ __forceinline__ float logp(float z) const {
    return bad ? __builtin_nanf("") : z == -kInf ? z : (z - m) - log_s;
  }
};

// Given token j of a row and its logit, loaded ahead of the sums.
struct Given {
  int tok = -1;
  float z = 0.0f;
  template <typename T>
  __device__ __forceinline__ void load(const LogprobsArgs& a, const T*, int row, int j) {
    if (j >= a.n_tokens) return;
    tok = a.tokens[int64_t(row) * a.n_tokens + j];
    if (tok >= 0 && tok < a.vocab) z = elem(static_cast<const T*>(a.logits) + int64_t(row) * a.ld, tok);
  }
  __device__ __forceinline__ void write(const LogprobsArgs& a, int row, int j, const Answer& w) const {
    if (j < a.n_tokens)
      a.token_lp[int64_t(row) * a.n_tokens + j] =
          tok == -1 ? 0.0f : (tok < 0 || tok >= a.vocab) ? __builtin_nanf("") : w.logp(z);
  }
};

// One wavefront writes a row's entropy and given tokens; lane j has token j.
template <typename T>
__device__ __forceinline__ void write_row(const LogprobsArgs& a, int row, const Sums& sums, const Answer& w,
                                          const Given& given) {
  const int lane = threadIdx.x & 63;
  if (lane == 0 && a.entropy)
    a.entropy[row] = w.bad ? __builtin_nanf("") : w.none ? 0.0f : w.log_s - sums.t / sums.s;
  given.write(a, row, lane, w);
  for (int j = lane + 64; j < a.n_tokens; j += 64) {
    Given g;
    g.load(a, static_cast<const T*>(nullptr), row, j);
    g.write(a, row, j, w);
  }
}

// Alternative number `rank` of a row (key 0: none).
__device__ __forceinline__ void write_top(const LogprobsArgs& a, int row, int rank, uint64_t key, const Answer& w) {
  const int64_t o = int64_t(row) * a.top_k + rank;
  a.top_tokens[o] = key != 0 && !w.bad ? token_of(key) : -1;
  a.top_lp[o] = w.bad ? __builtin_nanf("") : key != 0 ? w.logp(value_of(key)) : -kInf;
}

__device__ __forceinline__ uint64_t* partial_keys(const LogprobsArgs& a, int64_t blocks) {
  return reinterpret_cast<uint64_t*>(static_cast<f32x4*>(a.part) + blocks);
}

// A value that at least k of four values of every lane reach; kLowest where
// fewer are not masked.
__device__ __forceinline__ float reached_by(const f32x4& v, int k) {
  uint32_t o[4], t = 0;
#pragma unroll
  for (int q = 0; q < 4; ++q) o[q] = order_of(v[q]);
  if (k <= 32) {
    // The k-th largest of the lanes' largest: 800 cycles.
    t = __builtin_amdgcn_readlane(sort_wave(max(max(o[0], o[1]), max(o[2], o[3]))), k - 1);
  } else {
    // The k-th largest of all to 16 bits, each step of which waits for the one
    // before: 2000 cycles, for 85 elements instead of 260 with k = 64.
#pragma unroll
    for (int b = 31; b >= 16; --b) {
      const uint32_t c = t | (1u << b);
      int n = 0;
#pragma unroll
      for (int q = 0; q < 4; ++q) n += __popcll(__ballot(o[q] >= c));
      if (n >= k) t = c;
    }
  }
  return t < order_of(kLowest) ? kLowest : value_of(uint64_t(t) << 32);
}

// What the lanes of a block of W wavefronts leave in LDS of the chunks: so many
// maxima each.  A wavefront with more chunks than its share of them takes
// several as one.  16 blocks of one wavefront fit a CU.
template <int W>
constexpr int kPeaks = W == 1 ? 32 : 64;

// Bit j: element j of the lane reaches `bound`.
template <typename T>
__device__ __forceinline__ uint32_t reaching(const Chunk<T>& c, float bound) {
  constexpr int V = Chunk<T>::kVec;
  uint32_t which = 0;
#pragma unroll
  for (int l = 0; l < 4; ++l)
#pragma unroll
    for (int e = 0; e < V; ++e) which |= uint32_t(c.get(l, e) >= bound) << (l * V + e);
  return which;
}

// Keys of the lanes' elements `which` of a chunk, whose element 0 of the lane is
// `token`, behind the n in buf; their new number, of which kBuffer are there.
template <typename T>
__device__ __forceinline__ int leave_keys(const Chunk<T>& c, uint32_t which, int64_t token, uint64_t* buf, int n) {
  constexpr int V = Chunk<T>::kVec;
  while (true) {  // nearly always one a lane
    const uint64_t mask = __ballot(which != 0);
    if (mask == 0) return n;
    const int at = n + lanes_before(mask);
    const int j = __builtin_ctz(which | 0x80000000u);
    const float z = c.pick(j);
    if (which && at < kBuffer) buf[at] = key_of(z, uint32_t(token + (j / V) * 64 * V + j % V));
    which &= which - 1;
    n += __popcll(mask);
  }
}

// Keys of the elements that reach `bound`, of the entries (lanes' maxima of
// `group` chunks) that do, into buf; their number, or more than kBuffer where
// they are too many (buf then holds nothing of use).
template <typename T, int W>
__device__ __forceinline__ int collect(const Row<T>& row, int begin, int end, int group, int entries, float bound,
                                       const float (*peaks)[64], uint16_t* hits, uint64_t* buf) {
  constexpr int V = Chunk<T>::kVec;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int found = 0, n = 0;
#pragma unroll 4
  for (int e = 0; e < entries; ++e) {
    const bool hit = peaks[e][lane] >= bound;
    const uint64_t mask = __ballot(hit);
    if (mask == 0) continue;
    const int at = found + lanes_before(mask);
    if (hit && at < kBuffer) hits[at] = uint16_t(e * 64 + lane);
    found += __popcll(mask);
  }
  if (found > kBuffer) return found;
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  for (int h = 0; h < found; h += 64) {
    const int hit = h + lane < found ? hits[h + lane] : -1;
    for (int g = 0; g < group; ++g) {
      const int c = begin + wave + W * ((hit >> 6) * group + g);
      const bool mine = hit >= 0 && c < end;
      const int64_t i0 = int64_t(c) * Chunk<T>::kSize + (hit & 63) * V;
      Chunk<T> words;
      uint32_t inside = 0;  // elements that the row holds
#pragma unroll
      for (int l = 0; l < 4; ++l) {
        const int64_t i = i0 + l * 64 * V;
        words.raw[l] = u32x4{0, 0, 0, 0};
        if (mine && i + V > row.first && i < row.last) {
          words.raw[l] = *reinterpret_cast<const u32x4*>(row.p + i);
          const int lo = int(max(row.first - i, int64_t(0))), hi = int(min(row.last - i, int64_t(V)));
          inside |= ((1u << hi) - (1u << lo)) << (l * V);
        }
      }
      n = leave_keys(words, reaching(words, bound) & inside, i0 - row.first, buf, n);
    }
  }
  return n;
}

// Block (split, row): W wavefronts take the split's chunks in turn.  SPLIT: the
// block's sums and its best keys, sorted, go to the workspace; else the row's
// results are written.
template <typename T, int W, bool SPLIT, bool TOP>
__global__ __launch_bounds__(64 * W) void logprobs_kernel(LogprobsArgs a, int splits) {
  constexpr int kOwn = kPeaks<W> / W;  // a wavefront's entries
  // The second look's copy of a chunk takes their place.
  static_assert(kOwn * 64 * sizeof(float) >= 64 * 4 * sizeof(u32x4), "peaks hold a chunk");
  __shared__ __attribute__((aligned(16))) uint64_t keys[TOP ? W : 1][kBuffer];
  __shared__ __attribute__((aligned(16))) float peaks[TOP ? kPeaks<W> : 1][64];
  __shared__ __attribute__((aligned(16))) float pool[TOP && W > 1 ? W * 64 : 4];
  __shared__ uint16_t hits[TOP ? W : 1][kBuffer];
  __shared__ f32x4 all_sums[W];
  __shared__ int counts[W];
  static_assert(W == 1 || W == 4, "four values of every lane make the bound");
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int r = SPLIT ? blockIdx.y : blockIdx.x;
  const Row<T> row(a, r);
  int begin = 0, end = row.chunks;
  if constexpr (SPLIT) {
    // Equal parts: the first ones take a chunk more.
    const uint32_t split = blockIdx.x, each = uint32_t(row.chunks) / uint32_t(splits);
    const uint32_t more = uint32_t(row.chunks) - each * uint32_t(splits);
    begin = int(each * split + min(split, more));
    end = begin + int(each) + int(split < more);
  }

  Running run;
  Given given;
  Chunk<T> c, next;
  int i = begin + wave;
  if (i < end) row.load(next, i);
  if (!SPLIT && wave == 0) given.load(a, row.p, r, lane);
  const int group = ((end - begin + W - 1) / W + kOwn - 1) / kOwn;
  float(*own)[64] = peaks + (TOP ? wave * kOwn : 0);
  f32x4 most = {-kInf, -kInf, -kInf, -kInf};
  float peak = -kInf;
  int entry = 0, in_group = 0;
  auto lane_top_of = [](const f32x4& t) { return fmaxf(fmaxf(t[0], t[1]), fmaxf(t[2], t[3])); };
  while (i < end) {
    c = next;
    if (i + W < end) row.load(next, i + W);
    const f32x4 tops = tops_of(c);
    const float lane_top = lane_top_of(tops);
    const float top = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(max_wave(lane_top))));
    if constexpr (TOP) {
      peak = in_group == 0 ? lane_top : fmaxf(peak, lane_top);
      own[entry][lane] = peak;
      if (++in_group == group) {
        in_group = 0;
        ++entry;
      }
      if constexpr (W == 1) {
#pragma unroll
        for (int l = 0; l < 4; ++l) most[l] = fmaxf(most[l], tops[l]);
      } else {
        most[0] = fmaxf(most[0], lane_top);
      }
    }
    run.add(c, top);
    i += W;
  }

  Sums sums = run.total();
  if (lane == 0) all_sums[wave] = f32x4{sums.m, sums.s, sums.f, sums.t};
  int n = 0;
  if constexpr (TOP) {
    if constexpr (W > 1) {
      pool[threadIdx.x] = most[0];
      __syncthreads();
      // One wavefront with a chunk is enough for 64 lanes' values.
#pragma unroll
      for (int w = 0; w < W; ++w) most[w] = pool[w * 64 + lane];
    }
    const float bound = reached_by(most, a.top_k);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    if (begin + W < end) {
      n = collect<T, W>(row, begin, end, group, entry + (in_group > 0), bound, own, hits[wave], keys[wave]);
    } else if (begin + wave < end) {
      // The wavefront's only chunk is still in registers.
      const int64_t at = int64_t(begin + wave) * Chunk<T>::kSize + lane * Chunk<T>::kVec;
      n = leave_keys(c, reaching(c, bound), at - row.first, keys[wave], 0);
    }
    if (n > kBuffer) {
      // Too many: all chunks once more.
      Best best;
      best.init(a.top_k, keys[wave]);
      best.bound(bound);
      u32x4(*copy)[4] = reinterpret_cast<u32x4(*)[4]>(own);
      for (i = begin + wave; i < end; i += W) {
        row.load(c, i);
        const f32x4 tops = tops_of(c);
        const float top = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(max_wave(lane_top_of(tops)))));
        const bool last = i + W >= end;
        if (top >= best.above || (last && best.merged)) offer_chunk(c, tops, row, i, last, best, copy);
      }
      n = best.finish();
    }
  }
  if (lane == 0) counts[wave] = n;
  __syncthreads();
  if constexpr (W > 1) {
    // Lane l takes wavefront l % 4's.
    const f32x4 o = all_sums[lane & 3];
    sums = Sums{o[0], o[1], o[2], o[3]};
    auto quad = [](float v, auto f) {
      v = f(v, xor_lane<1>(v));
      return f(v, xor_lane<2>(v));
    };
    auto add = [](float x, float y) { return x + y; };
    const float m = quad(sums.m, [](float x, float y) { return fmaxf(x, y); });
    rescale(sums, m);
    sums = Sums{m, quad(sums.s, add), quad(sums.f, add), quad(sums.t, add)};
  }
  const int64_t part = int64_t(r) * splits + blockIdx.x;  // SPLIT: the block's place
  Answer answer;
  if constexpr (SPLIT) {
    if (threadIdx.x == 0) static_cast<f32x4*>(a.part)[part] = f32x4{sums.m, sums.s, sums.f, sums.t};
  } else {
    answer = Answer(sums);
    if (wave == 0) write_row<T>(a, r, sums, answer, given);
  }
  if constexpr (TOP) {
    uint64_t* sorted = partial_keys(a, int64_t(a.rows) * splits) + part * a.top_k;
    auto put = [&](int rank, uint64_t key) {
      if constexpr (SPLIT)
        sorted[rank] = key;
      else
        write_top(a, r, rank, key, answer);
    };
    int total = 0;
#pragma unroll
    for (int w = 0; w < W; ++w) total += counts[w];
    // W lanes rank a key, each among one wavefront's.
    const int w = lane % W;
    for (int j0 = 0; j0 < n; j0 += 64 / W) {
      const int j = j0 + lane / W;
      const uint64_t key = keys[wave][min(j, kBuffer - 1)];
      int rank = j < n ? rank_among(keys[w], counts[w], key) : a.top_k;
      if constexpr (W > 1) {
        rank += xor_lane<1>(uint32_t(rank));
        rank += xor_lane<2>(uint32_t(rank));
      }
      if (w == 0 && rank < a.top_k) put(rank, key);
    }
    if (wave == 0 && lane >= total && lane < a.top_k) put(lane, 0);
  }
}

// A row's partial results.  Lane i of the last wavefront takes split i's sums; the
// others merge the splits' sorted keys, a fourth of the splits each, and the
// first of them what they have (a merge is six stages, some 300 cycles).
constexpr int kMergers = 4;

template <typename T, bool TOP>
__global__ __launch_bounds__(64 * (TOP ? kMergers + 1 : 1)) void join_kernel(LogprobsArgs a, int splits) {
  __shared__ uint64_t lists[kMergers][64];
  __shared__ f32x4 shared;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = blockIdx.x;
  const int64_t base = int64_t(r) * splits;
  uint64_t list = 0;
  if (!TOP || wave == kMergers) {
    Sums sums{kLowest, 0.0f, 0.0f, 0.0f};
    if (lane < splits) {
      const f32x4 v = static_cast<const f32x4*>(a.part)[base + lane];
      sums = Sums{v[0], v[1], v[2], v[3]};
    }
    Given given;
    given.load(a, static_cast<const T*>(nullptr), r, lane);
    const float m = max_wave(sums.m);
    rescale(sums, m);
    sums = Sums{m, sum_wave(sums.s), sum_wave(sums.f), sum_wave(sums.t)};
    const Answer answer(sums);
    write_row<T>(a, r, sums, answer, given);
    if (TOP && lane == 0) shared = f32x4{answer.m, answer.log_s, float(answer.bad), float(answer.none)};
  } else if constexpr (TOP) {
    const uint64_t* src = partial_keys(a, int64_t(a.rows) * splits) + base * a.top_k;
    // The best key of a split is a list's first, or its last where it is merged into another.
    auto key = [&](int split, int i) { return split < splits && i < a.top_k ? src[split * a.top_k + i] : 0; };
    constexpr int kAhead = 4;
    uint64_t next[kAhead];
    list = key(wave, lane);
#pragma unroll
    for (int q = 0; q < kAhead; ++q) next[q] = key(wave + kMergers * (q + 1), 63 - lane);
    for (int s = wave + kMergers; s < splits; s += kMergers * kAhead) {
#pragma unroll
      for (int q = 0; q < kAhead; ++q) {
        if (s + kMergers * q >= splits) break;
        list = merge_stages<32>(list > next[q] ? list : next[q], true);
        next[q] = key(s + kMergers * (q + kAhead), 63 - lane);
      }
    }
    lists[wave][lane] = list;
  }
  if constexpr (TOP) {
    __syncthreads();
    if (wave != 0) return;
    for (int w = 1; w < min(kMergers, splits); ++w) {
      const uint64_t other = lists[w][63 - lane];
      list = merge_stages<32>(list > other ? list : other, true);
    }
    Answer answer;
    answer.m = shared[0];
    answer.log_s = shared[1];
    answer.bad = shared[2] != 0.0f;
    answer.none = shared[3] != 0.0f;
    if (lane < a.top_k) write_top(a, r, lane, list, answer);
  }
}

template <typename T, bool TOP>
hipError_t launch(const LogprobsArgs& a, int cus, hipStream_t s) {
  const LogprobsShape p = logprobs_shape(a.rows, a.vocab, sizeof(T), cus);
  if (p.splits > 1) {
    hipLaunchKernelGGL((logprobs_kernel<T, 4, true, TOP>), dim3(p.splits, a.rows), dim3(256), 0, s, a, p.splits);
    hipLaunchKernelGGL((join_kernel<T, TOP>), dim3(a.rows), dim3(TOP ? 64 * (kMergers + 1) : 64), 0, s, a, p.splits);
  } else if (p.waves == 1) {
    hipLaunchKernelGGL((logprobs_kernel<T, 1, false, TOP>), dim3(a.rows), dim3(64), 0, s, a, 1);
  } else {
    hipLaunchKernelGGL((logprobs_kernel<T, 4, false, TOP>), dim3(a.rows), dim3(256), 0, s, a, 1);
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_logprobs(const LogprobsArgs& a, int cus, hipStream_t s) {
  if (a.rows < 1) return hipSuccess;
  const bool top = a.top_k > 0;
  switch (a.type) {
    case HS_TYPE_F32: return top ? launch<float, true>(a, cus, s) : launch<float, false>(a, cus, s);
    case HS_TYPE_BF16: return top ? launch<uint16_t, true>(a, cus, s) : launch<uint16_t, false>(a, cus, s);
    case HS_TYPE_F16: return top ? launch<_Float16, true>(a, cus, s) : launch<_Float16, false>(a, cus, s);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace hs
