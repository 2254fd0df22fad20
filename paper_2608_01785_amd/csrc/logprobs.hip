// Log probabilities of given tokens, entropy and top alternatives of rows of
// logits z, in one read of them:
//   m = max z,  S = sum e^(z - m),  log p[t] = z[t] - m - log S,
//   H = log S - T / S,  T = sum e^(z - m) (z - m)
// Alternatives are ordered by logit, equal ones by the lower token.
//
// Every lane keeps a running (m, S, F, T) of its elements; F is S without the
// largest element's own 1, so that log S = log1p(F) keeps its digits where
// one token has nearly all the probability.  A 4 KB chunk of a row sits in
// one wavefront's registers: its maximum first, then one rescaling of the
// sums, then e^(z - m) of each element.
//
// Alternatives: a wavefront keeps its 64 best keys (order of the value, then
// the lower token) sorted over its lanes.  A chunk whose maximum does not
// exceed the k-th best is done; otherwise the elements that do go to a buffer
// in LDS, and every 64 of them are sorted and merged.  The first chunk's lane
// maxima give a first bound: their k-th largest.
#include "answer_device.h"
#include "answer_kernels.h"

namespace hs {
namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLowest = -3.4028234663852886e38f;  // running maximum before any element
constexpr float kInf = __builtin_inff();
constexpr float kFar = -200.0f;  // e^-200 is 0 in fp32: differences are clamped here where 0 * -inf could arise

// ---------------------------------------------------------------- running sums

struct Sums {
  float m, s, f, t;  // maximum, S, S without the maximum's own 1, T
};

__device__ __forceinline__ float exp_of(float d) { return exp2_raw(d * kLog2e); }

__device__ __forceinline__ Sums join(const Sums& a, const Sums& b) {
  Sums r;
  r.m = fmaxf(a.m, b.m);
  const float da = fmaxf(a.m - r.m, kFar), db = fmaxf(b.m - r.m, kFar);
  const float fa = exp_of(da), fb = exp_of(db);
  const float sa = a.s * fa, sb = b.s * fb;
  r.s = sa + sb;
  r.f = (a.m < r.m ? sa : a.f) + (b.m < r.m ? sb : b.f);
  r.t = fmaf(sa, da, fa * a.t) + fmaf(sb, db, fb * b.t);
  return r;
}

// ---------------------------------------------------------------- lanes

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
__device__ __forceinline__ Sums join_lanes(const Sums& a) {
  return join(a, Sums{xor_lane<J>(a.m), xor_lane<J>(a.s), xor_lane<J>(a.f), xor_lane<J>(a.t)});
}
__device__ __forceinline__ Sums join_wave(Sums a) {
  a = join_lanes<1>(a);
  a = join_lanes<2>(a);
  a = join_lanes<4>(a);
  a = join_lanes<8>(a);
  a = join_lanes<16>(a);
  return join_lanes<32>(a);
}

// One stage of a bitonic network over the 64 lanes: lane pairs J apart, the
// larger value to the lower lane where `down`.
template <int J, typename V>
__device__ __forceinline__ V stage(V v, bool down) {
  const V o = xor_lane<J>(v);
  const bool keep_large = ((threadIdx.x & J) == 0) == down;
  return (v > o) == keep_large ? v : o;
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

constexpr int kBuffer = 128;  // candidates of a wavefront in LDS: 63 left over and 64 new

// One wavefront's best keys.
struct Best {
  uint64_t list = 0;   // lane i: the i-th best so far
  uint64_t kth;        // a candidate's key must exceed this
  float above;         // so its value must be at least this
  int count = 0;       // candidates in the buffer
  int k;
  uint64_t* buf;

  __device__ __forceinline__ void init(int top_k, uint64_t* lds) {
    k = top_k;
    buf = lds;
    kth = key_of(-kInf, 0);  // above every masked token
    above = kLowest;
  }
  // Elements still to come have higher tokens than those in the list, so one
  // that only equals the k-th value loses: the next value up is the least to look at.
  __device__ __forceinline__ void bound(uint64_t key) {
    if (key > kth) {
      kth = key;
      above = value_of(key + (uint64_t(1) << 32));
    }
  }
  // The k-th largest of the first chunk's lane maxima: k elements are at least that.
  __device__ __forceinline__ void seed(float lane_max) {
    const float s = sort_wave(lane_max);
    const float v = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(s), k - 1));
    if (v > -kInf) {
      kth = (uint64_t(order_of(v)) << 32) - 1;
      above = v;
    }
  }
  __device__ __forceinline__ uint64_t kth_of_list() const {
    return (uint64_t(__builtin_amdgcn_readlane(uint32_t(list >> 32), k - 1)) << 32) |
           uint32_t(__builtin_amdgcn_readlane(uint32_t(list), k - 1));
  }
  __device__ __forceinline__ void absorb(uint64_t key) {
    list = merge_lists(list, sort_wave(key));
    bound(kth_of_list());
  }
  // Every lane offers a key (0: none).
  __device__ __forceinline__ void offer(uint64_t key) {
    const int lane = threadIdx.x & 63;
    const bool take = key > kth;
    const uint64_t mask = __ballot(take);
    if (mask == 0) return;
    const int at = count + __popcll(mask & ((uint64_t(1) << lane) - 1));
    if (take) buf[at] = key;
    count += __popcll(mask);
    if (count >= 64) {
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      const uint64_t first = buf[lane], rest = buf[64 + lane];
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      count -= 64;
      if (lane < count) buf[lane] = rest;
      absorb(first);
    }
  }
  __device__ __forceinline__ void finish() {
    const int lane = threadIdx.x & 63;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    if (count) absorb(lane < count ? buf[lane] : 0);
    count = 0;
  }
};

// ---------------------------------------------------------------- chunks

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
  // `p`: the row's 16-byte aligned origin; all of chunk c lies in the row.
  __device__ __forceinline__ void load(const T* p, int64_t c) {
    const T* q = p + c * kSize + (threadIdx.x & 63) * kVec;
#pragma unroll
    for (int l = 0; l < 4; ++l) raw[l] = *reinterpret_cast<const u32x4*>(q + l * 64 * kVec);
  }
  // The same where the chunk reaches past the row [first, last): masked there.
  __device__ void load_edge(const T* p, int64_t c, int64_t first, int64_t last) {
#pragma unroll
    for (int l = 0; l < 4; ++l) {
      const int64_t i = c * kSize + (l * 64 + (threadIdx.x & 63)) * kVec;
      if (i >= first && i + kVec <= last) {
        raw[l] = *reinterpret_cast<const u32x4*>(p + i);
      } else {
        constexpr uint32_t masked = sizeof(T) == 4 ? 0xff800000u : __is_same(T, uint16_t) ? 0xff80u : 0xfc00u;
        uint32_t v[4];
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          if constexpr (sizeof(T) == 4) {
            v[w] = (i + w >= first && i + w < last) ? __float_as_uint(p[i + w]) : masked;
          } else {
            const int64_t a = i + 2 * w, b = a + 1;
            const uint16_t* u = reinterpret_cast<const uint16_t*>(p);
            v[w] = ((a >= first && a < last) ? u[a] : masked) | (((b >= first && b < last) ? u[b] : masked) << 16);
          }
        }
        raw[l] = u32x4{v[0], v[1], v[2], v[3]};
      }
    }
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

// One chunk's elements into the lane's sums; returns the lane's largest.
template <typename T>
__device__ __forceinline__ float accumulate(const Chunk<T>& c, Sums& a) {
  constexpr int V = Chunk<T>::kVec;
  float top = c.get(0, 0);
#pragma unroll
  for (int l = 0; l < 4; ++l)
#pragma unroll
    for (int e = 0; e < V; ++e) top = fmaxf(top, c.get(l, e));
  const float m = fmaxf(a.m, top);
  const float d0 = fmaxf(a.m - m, kFar), f0 = exp_of(d0), s0 = a.s * f0;
  a.f = a.m < m ? s0 : a.f;
  a.t = fmaf(s0, d0, f0 * a.t);
  a.m = m;
  float s[4] = {}, f[4] = {}, t[4] = {};
#pragma unroll
  for (int l = 0; l < 4; ++l)
#pragma unroll
    for (int e = 0; e < V; ++e) {
      const float d = c.get(l, e) - m, x = exp_of(d);
      s[e & 3] += x;
      f[e & 3] += __builtin_amdgcn_fractf(x);   // 0 where x is 1
      t[e & 3] = fmaf(x, fmaxf(d, kFar), t[e & 3]);
    }
  a.s = s0 + ((s[0] + s[1]) + (s[2] + s[3]));
  a.f += (f[0] + f[1]) + (f[2] + f[3]);
  a.t += (t[0] + t[1]) + (t[2] + t[3]);
  return top;
}

// The chunk's elements that may be among the best.  A lane offers one element
// at a time, read again from memory (the cache still has it) since registers
// cannot be indexed.
template <typename T>
__device__ __forceinline__ void offer_chunk(const Chunk<T>& c, const Row<T>& row, int i, Best& best) {
  constexpr int V = Chunk<T>::kVec;
  uint32_t hits = 0;
#pragma unroll
  for (int l = 0; l < 4; ++l)
#pragma unroll
    for (int e = 0; e < V; ++e) hits |= uint32_t(c.get(l, e) >= best.above) << (l * V + e);
  while (__ballot(hits != 0)) {
    uint64_t key = 0;
    if (hits) {
      const int j = __builtin_ctz(hits);
      hits &= hits - 1;
      const int64_t at = int64_t(i) * Chunk<T>::kSize + ((j / V) * 64 + int(threadIdx.x & 63)) * V + j % V;
      // Outside the row a chunk holds masked elements.
      if (at >= row.first && at < row.last) key = key_of(elem(row.p, at), uint32_t(at - row.first));
    }
    best.offer(key);
  }
}

// ---------------------------------------------------------------- results

__device__ __forceinline__ float log_sum(const Sums& a) { return a.s < 1.5f ? log1pf(a.f) : logf(a.s); }

// One wavefront writes a row's results from its sums and its best keys.
template <typename T>
__device__ __forceinline__ void write_row(const LogprobsArgs& a, int row, const Sums& sums, uint64_t best) {
  const int lane = threadIdx.x & 63;
  const bool bad = sums.s != sums.s, none = sums.s == 0.0f;
  const float nan = __builtin_nanf(""), log_s = none ? 0.0f : log_sum(sums);
  auto logp = [&](float z) { return bad ? nan : z == -kInf ? z : (z - sums.m) - log_s; };
  if (lane == 0 && a.entropy) a.entropy[row] = bad ? nan : none ? 0.0f : log_s - sums.t / sums.s;
  const T* z = static_cast<const T*>(a.logits) + int64_t(row) * a.ld;
  for (int j = lane; j < a.n_tokens; j += 64) {
    const int64_t o = int64_t(row) * a.n_tokens + j;
    const int tok = a.tokens[o];
    a.token_lp[o] = tok == -1 ? 0.0f : (tok < 0 || tok >= a.vocab) ? nan : logp(elem(z, tok));
  }
  if (lane < a.top_k) {
    const int64_t o = int64_t(row) * a.top_k + lane;
    const bool listed = best != 0 && !bad;
    a.top_tokens[o] = listed ? token_of(best) : -1;
    a.top_lp[o] = bad ? nan : listed ? logp(value_of(best)) : -kInf;
  }
}

__device__ __forceinline__ uint64_t* partial_keys(const LogprobsArgs& a, int64_t blocks) {
  return reinterpret_cast<uint64_t*>(static_cast<f32x4*>(a.part) + blocks);
}

// The block's wavefronts' sums and lists, joined in wavefront 0.
template <int W, bool TOP>
__device__ __forceinline__ void join_block(Sums& sums, uint64_t& list, f32x4* lds_sums, uint64_t (*lds_keys)[kBuffer]) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int half = W / 2; half > 0; half >>= 1) {
    if (wave >= half && wave < 2 * half) {
      if (lane == 0) lds_sums[wave] = f32x4{sums.m, sums.s, sums.f, sums.t};
      if (TOP) lds_keys[wave][lane] = list;
    }
    __syncthreads();
    if (wave < half) {
      const f32x4 o = lds_sums[wave + half];
      sums = join(sums, Sums{o[0], o[1], o[2], o[3]});
      if (TOP) list = merge_lists(list, lds_keys[wave + half][lane]);
    }
  }
}

// Block (row, split): W wavefronts take the split's chunks in turn.
template <typename T, int W, bool TOP>
__global__ __launch_bounds__(64 * W) void logprobs_kernel(LogprobsArgs a, int splits, int chunks_per_split) {
  __shared__ uint64_t keys[TOP ? W : 1][kBuffer];
  __shared__ f32x4 lds_sums[W];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t blocks = int64_t(a.rows) * splits;
  const int r = int(blockIdx.x / splits), split = int(blockIdx.x % splits);
  const Row<T> row(a, r);
  const int end = min(row.chunks, (split + 1) * chunks_per_split);

  Sums sums{kLowest, 0.0f, 0.0f, 0.0f};
  Best best;
  if (TOP) best.init(a.top_k, keys[wave]);
  int i = split * chunks_per_split + wave;
  bool first = true;
  Chunk<T> next;
  if (i < end) row.load(next, i);
  while (i < end) {
    const Chunk<T> c = next;
    if (i + W < end) row.load(next, i + W);
    const float top = accumulate(c, sums);
    if constexpr (TOP) {
      if (first) best.seed(top);
      if (__ballot(top >= best.above)) offer_chunk(c, row, i, best);
      first = false;
    }
    i += W;
  }
  if (TOP) best.finish();
  sums = join_wave(sums);
  join_block<W, TOP>(sums, best.list, lds_sums, keys);
  if (wave != 0) return;
  if (splits == 1) {
    write_row<T>(a, r, sums, TOP ? best.list : 0);
    return;
  }
  if (lane == 0) static_cast<f32x4*>(a.part)[blockIdx.x] = f32x4{sums.m, sums.s, sums.f, sums.t};
  if (TOP && lane < a.top_k) partial_keys(a, blocks)[int64_t(blockIdx.x) * a.top_k + lane] = best.list;
}

// A row's partial results: lane i takes split i's sums, the wavefronts the
// lists in turn.
template <typename T, bool TOP>
__global__ __launch_bounds__(256) void join_kernel(LogprobsArgs a, int splits) {
  __shared__ uint64_t keys[TOP ? 4 : 1][kBuffer];
  __shared__ f32x4 lds_sums[4];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = blockIdx.x;
  const int64_t base = int64_t(r) * splits;
  Sums sums{kLowest, 0.0f, 0.0f, 0.0f};
  if (wave == 0 && lane < splits) {
    const f32x4 v = static_cast<const f32x4*>(a.part)[base + lane];
    sums = Sums{v[0], v[1], v[2], v[3]};
  }
  sums = join_wave(sums);
  uint64_t list = 0;
  if (TOP) {
    const uint64_t* src = partial_keys(a, int64_t(a.rows) * splits) + base * a.top_k;
    for (int i = wave; i < splits; i += 4)
      list = merge_lists(list, lane < a.top_k ? src[int64_t(i) * a.top_k + lane] : 0);
  }
  join_block<4, TOP>(sums, list, lds_sums, keys);
  if (wave == 0) write_row<T>(a, r, sums, list);
}

template <typename T, bool TOP>
hipError_t launch(const LogprobsArgs& a, int cus, hipStream_t s) {
  const LogprobsShape p = logprobs_shape(a.rows, a.vocab, sizeof(T), cus);
  const unsigned grid = unsigned(a.rows) * unsigned(p.splits);
  if (p.waves == 1)
    hipLaunchKernelGGL((logprobs_kernel<T, 1, TOP>), dim3(grid), dim3(64), 0, s, a, p.splits, p.chunks_per_split);
  else
    hipLaunchKernelGGL((logprobs_kernel<T, 4, TOP>), dim3(grid), dim3(256), 0, s, a, p.splits, p.chunks_per_split);
  if (p.splits > 1) hipLaunchKernelGGL((join_kernel<T, TOP>), dim3(a.rows), dim3(256), 0, s, a, p.splits);
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
