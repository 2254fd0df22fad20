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
#include "logits_scan.h"

namespace hs {
namespace {

using namespace scan;

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
