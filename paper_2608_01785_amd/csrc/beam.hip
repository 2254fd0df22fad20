// The best continuations of a group of beams, over beams b and vocabulary t:
//   value(b, t) = score[b] + z[b, t] - log sum_j e^z[b, j]
// Order: the value, then the lower beam, then the lower token; within a row, the
// logit's own order, which its values share.
//
// Two launches.  The scan of hs_logprobs (logits_scan.h) reads every row once and
// leaves, for each block of it, the sums behind the logarithm and the keys of its
// `select` best logits: no continuation outside a row's `select` best can be among
// the group's.  The join, a block per group, takes the logarithm of each beam's sum and
// ranks the beams' candidates against each other: up to 256 as the splits left them,
// more after each beam's sorted lists have been merged to one.  Ended and empty beams
// are not read.
//
// The read of the logits bounds a large call (512 rows of 131072 bf16: 27.5 us for the scan,
// 4.9 TB/s, and 5.2 for the join), the chain of each kernel a small one (4 rows of 32000
// fp32: 4.9 and 3.6; with merged lists the join took 6.2).
//
// Values are held in 64 bits from the sums of a row on: continuations of two beams
// that lie closer than the 2^-20 that fp32 resolves at -10 are common among the many
// near a selection's border, and their order decides whole sequences.
#include "decoding_kernels.h"
#include "logits_scan.h"

namespace hs {
namespace {

using namespace scan;

constexpr int kJoinWaves = 16;

// log sum e^z of a row from its splits' partial results, the same bits in every lane;
// NaN or -inf where the row has no distribution (NaN, +inf, all masked).
__device__ __forceinline__ double log_sum_of(Sums sums) {
  // The splits' sums against the row's maximum; F without the elements at it.
  const float m = max_wave(sums.m);
  const float f = exp_of(fmaxf(sums.m - m, kFar));
  // (No product is left for the sums to contract with: every lane adds the same.)
  double s = double(sums.s * f), rest = sums.m < m ? s : double(sums.f);
  s = reduce_wave(s, [](double x, double y) { return x + y; });
  rest = reduce_wave(rest, [](double x, double y) { return x + y; });
  if (!(s > 0.0)) return -double(kInf);
  return double(m) + (s < 1.5 ? log1p(rest) : log(s));
}

__device__ __forceinline__ void write_selected(const BeamArgs& a, int64_t group, int rank, double value, int beam,
                                               int token) {
  const int64_t o = group * a.select + rank;
  a.out_scores[o] = float(value);
  a.out_parents[o] = beam;
  a.out_tokens[o] = token;
  if (a.out_finished)
    a.out_finished[o] =
        beam >= 0 && ((a.finished && a.finished[group * a.beams + beam] != 0) || (a.end_token >= 0 && token == a.end_token));
}

// Few candidates: the splits' keys of all beams, as they were left, are ranked against
// each other.  Block: one group, a thread or more for each of its n candidates;
// wavefronts take the beams' sums in turn.
constexpr int kFewCandidates = 256;

__global__ __launch_bounds__(64 * kJoinWaves) void beam_few_kernel(BeamArgs a, LogprobsArgs scanned, int splits) {
  __shared__ double values[kFewCandidates];
  __shared__ uint64_t keys[kFewCandidates];
  __shared__ double log_sums[kBeamMaxBeams];
  __shared__ int total;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
  const int per_beam = splits * a.select, n = a.beams * per_beam;
  const int64_t row0 = int64_t(blockIdx.x) * a.beams;
  const int c = threadIdx.x;
  uint64_t key = 0;
  float score = -kInf;
  bool ended = false;
  const int beam = c / per_beam;
  if (c < n) {
    key = partial_keys(scanned, int64_t(scanned.rows) * splits)[row0 * per_beam + c];
    score = a.scores[row0 + beam];
    ended = a.finished && a.finished[row0 + beam] != 0;
  }
  for (int b = wave; b < a.beams; b += waves) {
    Sums sums{kLowest, 0.0f, 0.0f, 0.0f};
    if (lane < splits) {
      const f32x4 v = static_cast<const f32x4*>(a.part)[(row0 + b) * splits + lane];
      sums = Sums{v[0], v[1], v[2], v[3]};
    }
    const double l = log_sum_of(sums);  // (of an unscanned row: anything, not used)
    if (lane == 0) log_sums[b] = l;
  }
  if (threadIdx.x == 0) total = 0;
  __syncthreads();
  double value = -double(kInf);
  if (c < n && score > -kInf) {
    if (ended) {
      if (c == beam * per_beam) {
        value = double(score);
        key = key_of(0.0f, uint32_t(a.end_token));
      }
    } else if (key != 0 && log_sums[beam] > -double(kInf)) {
      value = double(score) + (double(value_of(key)) - log_sums[beam]);
    }
  }
  if (c < kFewCandidates) {
    values[c] = value;
    keys[c] = key;
  }
  const int here = __popcll(__ballot(value > -double(kInf)));
  if (lane == 0 && here) atomicAdd(&total, here);
  __syncthreads();
  // Eight lanes count what goes before a candidate.
  const int o = threadIdx.x & 7;
  for (int c0 = 0; c0 < n; c0 += blockDim.x / 8) {
    const int me = c0 + int(threadIdx.x >> 3);
    const double v = me < n ? values[me] : -double(kInf);
    uint32_t rank = 0;
    if (v > -double(kInf)) {
      int same = 0;  // as large, the candidate itself among them
#pragma unroll 8
      for (int j = o; j < n; j += 8) {
        const double w = values[j];
        rank += w > v;
        same += w == v;
      }
      if (same > int(((me ^ o) & 7) == 0)) {
        const uint64_t mine = keys[me];
        const int first = me / per_beam * per_beam;
        for (int j = o; j < n; j += 8)
          if (values[j] == v) rank += j < first || (j < first + per_beam && keys[j] > mine);
      }
    }
    rank += xor_lane<1>(rank);
    rank += xor_lane<2>(rank);
    rank += xor_lane<4>(rank);
    if (o == 0 && v > -double(kInf) && rank < uint32_t(a.select))
      write_selected(a, blockIdx.x, rank, v, me / per_beam, token_of(keys[me]));
  }
  for (int r = total + int(threadIdx.x); r < a.select; r += blockDim.x)
    write_selected(a, blockIdx.x, r, -double(kInf), -1, -1);
}

// Block: one group.  `team` wavefronts share a beam.
__global__ __launch_bounds__(64 * kJoinWaves) void beam_join_kernel(BeamArgs a, LogprobsArgs scanned, int splits,
                                                                    int team, int span) {
  __shared__ uint64_t lists[kJoinWaves][64];
  __shared__ int counts[kBeamMaxBeams];
  extern __shared__ double values[];                                   // [beams][select]
  int32_t* tokens = reinterpret_cast<int32_t*>(values + a.beams * a.select);  // [beams][select]
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int teams = int(blockDim.x >> 6) / team, member = wave % team;
  const int k = a.select;
  const int64_t row0 = int64_t(blockIdx.x) * a.beams;
  for (int b0 = 0; b0 < a.beams; b0 += teams) {
    const int b = b0 + wave / team;
    const bool mine = b < a.beams;
    const int64_t row = row0 + min(b, a.beams - 1);
    // Everything the beam needs is asked for at once; a beam that was not scanned has
    // left nothing, and nothing of it is used.
    const float score = a.scores[row];
    const bool ended = a.finished && a.finished[row] != 0;
    const uint64_t* src = partial_keys(scanned, int64_t(scanned.rows) * splits) + row * splits * k;
    // The best key of a split is a list's first, or its last where it is merged into another.
    auto key = [&](int split, int i) { return split < splits && i < k ? src[int64_t(split) * k + i] : 0; };
    uint64_t list = key(member, lane), next = key(member + team, 63 - lane);
    Sums sums{kLowest, 0.0f, 0.0f, 0.0f};
    if (lane < splits) {
      const f32x4 v = static_cast<const f32x4*>(a.part)[row * splits + lane];
      sums = Sums{v[0], v[1], v[2], v[3]};
    }
    for (int s = member + team; s < splits; s += team) {
      const uint64_t other = next;
      next = key(s + team, 63 - lane);
      list = merge_stages<32>(list > other ? list : other, true);
    }
    if (team > 1) {
      lists[wave][lane] = list;
      __syncthreads();
    }
    if (mine && member == 0) {
      int n = 0;
      if (!ended && score > -kInf) {
        for (int w = 1; w < min(team, splits); ++w) {
          const uint64_t other = lists[wave + w][63 - lane];
          list = merge_stages<32>(list > other ? list : other, true);
        }
        const double log_sum = log_sum_of(sums);
        n = log_sum > -double(kInf) ? __popcll(__ballot(lane < k && list != 0)) : 0;
        if (lane < n) {
          values[b * k + lane] = double(score) + (double(value_of(list)) - log_sum);
          tokens[b * k + lane] = token_of(list);
        }
      } else if (ended && score > -kInf) {
        n = 1;
        if (lane == 0) {
          values[b * k] = double(score);
          tokens[b * k] = a.end_token;
        }
      }
      if (lane == 0) counts[b] = n;
    }
    __syncthreads();
  }
  // The lists are sorted: a candidate's rank is its place in its own and, by
  // bisection, the number of larger values in each other (of equal ones, those of
  // lower beams).  A lane takes one of the other lists; `span` lanes, a power of two,
  // a candidate.
  const int o = threadIdx.x & (span - 1);
  for (int c0 = 0; c0 < a.beams * k; c0 += blockDim.x / span) {
    const int c = c0 + threadIdx.x / span;
    const int b = c / k, i = c - b * k;
    const bool there = b < a.beams && i < counts[min(b, a.beams - 1)];
    const double v = there ? values[c] : 0.0;
    int rank = 0;
    if (there && o < a.beams) {
      int hi = counts[o];
      if (o == b) {
        rank = i;
      } else {
        while (rank < hi) {
          const int mid = (rank + hi) >> 1;
          const double w = values[o * k + mid];
          if (w > v || (w == v && o < b))
            rank = mid + 1;
          else
            hi = mid;
        }
      }
    }
    for (int d = 1; d < span; d <<= 1) rank += __shfl_xor(rank, d, 64);
    if (!there || o != 0 || rank >= k) continue;
    write_selected(a, blockIdx.x, rank, v, b, tokens[c]);
  }
  if (wave != 0) return;
  int total = lane < a.beams ? counts[lane] : 0;
  for (int d = 1; d < 64; d <<= 1) total += __shfl_xor(total, d, 64);
  for (int r = total + lane; r < k; r += 64) write_selected(a, blockIdx.x, r, -double(kInf), -1, -1);
}

template <typename T>
hipError_t launch(const BeamArgs& a, int cus, hipStream_t s) {
  BeamScanArgs p{};
  p.logits = a.logits;
  p.type = a.type;
  p.ld = a.ld;
  p.rows = a.groups * a.beams;
  p.vocab = a.vocab;
  p.top_k = a.select;
  p.part = a.part;
  p.scores = a.scores;
  p.finished = a.finished;
  const LogprobsShape shape = beam_shape(p.rows, p.vocab, sizeof(T), cus);
  if (shape.waves == 1)
    hipLaunchKernelGGL((logprobs_kernel<T, 1, true, true, BeamScanArgs>), dim3(p.rows * shape.splits), dim3(64), 0, s, p,
                       shape.splits);
  else
    hipLaunchKernelGGL((logprobs_kernel<T, 4, true, true, BeamScanArgs>), dim3(p.rows * shape.splits), dim3(256), 0, s, p,
                       shape.splits);
  const int candidates = a.beams * shape.splits * a.select;
  if (candidates <= kFewCandidates) {
    const int threads = 8 * candidates <= 256 ? 256 : 8 * candidates <= 512 ? 512 : 1024;
    hipLaunchKernelGGL(beam_few_kernel, dim3(a.groups), dim3(threads), 0, s, a, p, shape.splits);
    return hipGetLastError();
  }
  int span = 1;
  while (span < a.beams) span *= 2;
  int team = a.beams < kJoinWaves ? kJoinWaves / a.beams : 1;
  if (team > shape.splits) team = shape.splits;
  const int waves = a.beams * team < kJoinWaves ? a.beams * team : kJoinWaves / team * team;
  hipLaunchKernelGGL(beam_join_kernel, dim3(a.groups), dim3(64 * waves), size_t(a.beams) * a.select * 12, s, a, p,
                     shape.splits, team, span);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_beam_select(const BeamArgs& a, int cus, hipStream_t s) {
  if (a.groups < 1) return hipSuccess;
  switch (a.type) {
    case HS_TYPE_F32: return launch<float>(a, cus, s);
    case HS_TYPE_BF16: return launch<uint16_t>(a, cus, s);
    case HS_TYPE_F16: return launch<_Float16>(a, cus, s);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace hs
