// 8-bit integer products with one scale per token and per channel for gfx950:
//   out[m, n] = a_scale[m] * w_scale[n] * sum_k a[m, k] w[n, k] + bias[n]
// The sum is exact (32-bit accumulators, k <= 131071); the conversion of the
// sum, the product of the scales, their product and the bias are one fp32
// rounding each, and the result is rounded once to the output's type.  So the
// bits depend on no tile, split or budget.
//
// The MFMA is issued as C^T = W A^T: every lane of a 32 x 32 accumulator owns
// one row of a and four consecutive channels per register group.
//
// A block of WN x WM waves computes tiles of 32 NS WN channels x 32 MT WM rows.
// K advances in stages of 64 bytes; half of the waves fetch the channels, half
// the rows, with 16-byte loads into a ring of registers:
//   stage t is loaded during stage t - 4, written to LDS buffer t % 2 in the
//   first half of stage t - 1 and multiplied during stage t.
// One barrier per stage, between its two 32-wide halves, after each wave's
// writes of stage t + 1 and fragment reads of stage t have completed: it makes
// the writes visible to the second half's reads of stage t + 1 and retires
// every read of the buffer that the next stage overwrites.  Stages past the
// end of k, up to a multiple of four, are zeros.
//
// The grid is persistent and the stages of a block's tiles form one sequence:
// the last four stages of a tile already fetch the next one's first four, and
// its epilogue runs under those loads.  An epilogue reads no memory: a tile's
// scales and bias come into LDS during the epilogue before it (stores count
// against the same completion counter as loads, so a load between them would
// wait for them; with such loads an epilogue took 18 us).
#include "answer_kernels.h"
#include "horizon.h"
#include "hs_device.h"

#include <type_traits>

namespace hs {
namespace {

typedef int32_t i32x4 __attribute__((ext_vector_type(4)));
typedef int32_t i32x16 __attribute__((ext_vector_type(16)));

constexpr int BK = 64;      // bytes of K per stage: 4 chunks of 16
constexpr int kUnroll = 4;  // stages per loop body
constexpr int kGroupM = 4;

__device__ __forceinline__ i32x16 mfma32_i8(const u32x4& a, const u32x4& b, const i32x16& c) {
  return __builtin_amdgcn_mfma_i32_32x32x32_i8(__builtin_bit_cast(i32x4, a), __builtin_bit_cast(i32x4, b), c, 0, 0, 0);
}

// 16-byte chunk c of tile row r sits at physical chunk c ^ swz(r).  A 16-lane
// pass of fragment reads covers rows r0 .. r0 + 15 at one logical chunk;
// (r & 3, c ^ swz(r)) is then distinct for all 16 rows, so the pass touches
// each of the 64 banks once.
__device__ __forceinline__ int swz(int r) { return ((r >> 1) ^ (r >> 2)) & 3; }

// ---------------------------------------------------------------- epilogue

template <int TYPE>
struct OutOf {
  using T = float;
};
template <>
struct OutOf<HS_TYPE_BF16> {
  using T = __bf16;
};
template <>
struct OutOf<HS_TYPE_F16> {
  using T = _Float16;
};

// The documented roundings of one output, none of them fused.
__device__ __forceinline__ float output(int32_t sum, float a_scale, float w_scale, bool with_bias, float bias) {
#pragma clang fp contract(off)
  const float s = a_scale * w_scale;
  const float v = float(sum) * s;
  return with_bias ? v + bias : v;
}

// Four consecutive values from p on, of which the first `left` exist.
template <typename T>
__device__ __forceinline__ void store_each(T* p, const float (&v)[4], int left) {
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (e < left) p[e] = T(v[e]);
}

template <typename T>
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  typedef T T2 __attribute__((ext_vector_type(2)));
  typedef float f2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((f2{lo, hi}), T2));
}

// Channels 0 .. 15 of a 16-channel run of one row, of which the first `left`
// exist: the low lane of the pair (lane, lane + 32) holds 0 .. 3 in `lo` and
// 8 .. 11 in `hi`, the high lane (h = 1) the four after each.  WIDE: p is
// aligned to 16 bytes; 16-bit values change lanes so that each lane stores 16
// bytes.  Both lanes of the pair must be active.
template <typename T, bool WIDE>
__device__ __forceinline__ void store_run(T* p, int h, const float (&lo)[4], const float (&hi)[4], int left) {
  if constexpr (sizeof(T) == 2) {
    if (WIDE && left >= 16) {
      const uint32_t a[2] = {pack2<T>(lo[0], lo[1]), pack2<T>(lo[2], lo[3])};
      const uint32_t b[2] = {pack2<T>(hi[0], hi[1]), pack2<T>(hi[2], hi[3])};
      u32x4 v;
#pragma unroll
      for (int d = 0; d < 2; ++d) {
        // Lanes 32 .. 63 of the first operand against lanes 0 .. 31 of the second.
        const auto s = __builtin_amdgcn_permlane32_swap(a[d], b[d], false, false);
        v[d] = s[0];
        v[2 + d] = s[1];
      }
      *reinterpret_cast<u32x4*>(p + 8 * h) = v;
      return;
    }
  } else if (WIDE && left >= 16) {
    *reinterpret_cast<f32x4*>(p + 4 * h) = f32x4{lo[0], lo[1], lo[2], lo[3]};
    *reinterpret_cast<f32x4*>(p + 8 + 4 * h) = f32x4{hi[0], hi[1], hi[2], hi[3]};
    return;
  }
  store_each(p + 4 * h, lo, left - 4 * h);
  store_each(p + 8 + 4 * h, hi, left - 8 - 4 * h);
}

// ---------------------------------------------------------------- tiles

// One wave's share of an operand's rows: the 16-byte chunk (lane & 3) of rows
// row0 + (lane >> 2) + 16 l.
//   ALIGNED: base, row stride and k are multiples of 16.  A buffer resource
//   over the rows: what lies past the last row or past k reads zero.
//   Otherwise: byte addresses, rows past the last read it again (they are
//   never stored) and the chunk that holds the end of k is read from 16 bytes
//   before that end and shifted.
template <bool ALIGNED, int L>
struct Operand {
  const int8_t* base;
  __amdgpu_buffer_rsrc_t res;
  uint32_t off[ALIGNED ? 1 : L];

  __device__ __forceinline__ void set(const int8_t* p, int64_t ld, int row0, int rows, int k) {
    const int r = (threadIdx.x & 63) >> 2, c = threadIdx.x & 3;
    if constexpr (ALIGNED) {
      // A wave without rows keeps one (never stored).
      const int first = min(row0, rows - 1), span = min(rows - first, 16 * L);
      base = p + int64_t(first) * ld;
      res = make_rsrc(base, uint32_t(span - 1) * uint32_t(ld) + uint32_t(k));
      off[0] = uint32_t(r) * uint32_t(ld) + uint32_t(c * 16);
    } else {
      base = p;
      const int first = min(row0, rows - 1);
      base = p + int64_t(first) * ld;
#pragma unroll
      for (int l = 0; l < L; ++l) off[l] = uint32_t(min(r + 16 * l, rows - 1 - first)) * uint32_t(ld) + uint32_t(c * 16);
    }
  }
  __device__ __forceinline__ u32x4 load(int l, int stage, int64_t ld, int k) const {
    const int whole = k / BK;  // stages without the end of k
    if constexpr (ALIGNED) {
      uint32_t v = off[0];
      // Past k: an offset outside the resource, which reads zero.
      if (stage >= whole && stage * BK + int(threadIdx.x & 3) * 16 >= k) v = 0x80000000u;
      const uint32_t s = uint32_t(min(stage, (k - 1) / BK)) * BK + uint32_t(16 * l) * uint32_t(ld);
      return __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(res, v, s, 0));
    } else {
      u32x4 v = {0, 0, 0, 0};
      const int8_t* p = base + int64_t(stage) * BK;
      if (stage < whole) {
        __builtin_memcpy(&v, p + off[l], 16);
        return v;
      }
      const int n = k - stage * BK - (int(threadIdx.x) & 3) * 16;  // bytes of the chunk that k holds
      if (n >= 16) {
        __builtin_memcpy(&v, p + off[l], 16);
      } else if (n > 0 && k >= 16) {
        __builtin_memcpy(&v, p + off[l] - (16 - n), 16);
        // Bytes 16 - n .. 15 are the chunk's first n.
        const int words = (16 - n) >> 2, bytes = (16 - n) & 3;
        uint32_t w[5] = {v[0], v[1], v[2], v[3], 0};
        for (int i = 0; i < words; ++i) {
          w[0] = w[1];
          w[1] = w[2];
          w[2] = w[3];
          w[3] = 0;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = __builtin_amdgcn_alignbyte(w[i + 1], w[i], bytes);
      } else if (n > 0) {
        uint32_t w[4] = {0, 0, 0, 0};
        for (int i = 0; i < n; ++i) {
          const uint32_t b = uint32_t(uint8_t(p[off[l] + i])) << (8 * (i & 3));
#pragma unroll
          for (int j = 0; j < 4; ++j) w[j] |= (i >> 2) == j ? b : 0u;
        }
        v = u32x4{w[0], w[1], w[2], w[3]};
      }
      return v;
    }
  }
};

template <int TYPE, bool ALIGNED, bool WIDE, int WN, int WM, int NS, int MT>
__global__ __launch_bounds__(WN * WM * 64, WN * WM == 8 ? 1 : 2) void linear_kernel(LinearI8Args a) {
  constexpr int kWaves = WN * WM, kHalf = kWaves / 2;
  constexpr int BN = 32 * NS * WN, BM = 32 * MT * WM;
  static_assert(BN == BM && BN % (16 * kHalf) == 0, "tile split");
  constexpr int L = BN / (16 * kHalf);  // 1 KB loads per wave and stage
  constexpr int kTile = BN * BK;
  constexpr int kStage = 2 * kTile;     // channels, then rows
  __shared__ __attribute__((aligned(1024))) uint8_t smem[2 * kStage];
  // w_scale, bias and a_scale of a tile; the next tile's beside it.
  constexpr int kFactors = 2 * BN + BM, kThreads = kWaves * 64, kPer = (kFactors + kThreads - 1) / kThreads;
  __shared__ __attribute__((aligned(16))) float factors[2][kFactors];
  using T = typename OutOf<TYPE>::T;

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wn = wave % WN, wm = wave / WN;
  const int fr = lane & 31, fh = lane >> 5;

  // Tiles in groups of kGroupM row tiles, rows fastest; a unit is a tile, or
  // half its rows where MT is even:
  //   - the tiles of a last row of tiles that holds at most half of them come
  //     after all others, as one half unit each;
  //   - when the last round of the others would leave more than half of the
  //     blocks idle (counting those halves), its tiles are split into two.
  const int tiles_m = (a.m + BM - 1) / BM, tiles_n = (a.n + BN - 1) / BN, G = gridDim.x;
  constexpr bool kHalves = MT % 2 == 0;
  const bool short_last = kHalves && a.m - (tiles_m - 1) * BM <= BM / 2;
  const int whole_m = short_last ? tiles_m - 1 : tiles_m;
  const int n_whole = whole_m * tiles_n, n_short = short_last ? tiles_n : 0;
  const int full_units = n_whole / G * G, tail = n_whole - full_units;
  const bool split_tail = kHalves && tail > 0 && 2 * tail + n_short <= G;
  const int n_first = split_tail ? full_units + 2 * tail : n_whole, n_units = n_first + n_short;
  const int per_group = kGroupM * tiles_n;
  struct Unit {
    int tm, tn, half;  // half: -1 the whole tile, else its first or second half
  };
  auto unit_at = [&](int u) {
    if (u >= n_first) return Unit{tiles_m - 1, u - n_first, 0};
    const bool split = split_tail && u >= full_units;
    const int t = split ? full_units + (u - full_units) / 2 : u;
    const int first_m = t / per_group * kGroupM;
    const int gsize = min(whole_m - first_m, kGroupM);
    return Unit{first_m + t % per_group % gsize, t % per_group / gsize, split ? (u - full_units) % 2 : -1};
  };
  // Round r gives block b unit r G + b, in odd rounds r G + G - 1 - b: the
  // blocks left without a full unit take the first halves.  The blocks of an
  // XCD stay on a contiguous range.
  const int b = xcd_remap(blockIdx.x, G);
  auto unit_of = [&](int r) { return r * G + ((r & 1) ? G - 1 - b : b); };
  int round = 0;
  if (unit_of(0) >= n_units) return;
  Unit unit = unit_at(unit_of(0));

  const int KP = ((a.k + BK - 1) / BK + kUnroll - 1) / kUnroll * kUnroll;  // stages of a tile
  // The first half of the waves loads channels, the second rows.
  const bool w_wave = wave < kHalf;
  const int8_t* src = w_wave ? a.w : a.a;
  const int64_t ld = w_wave ? a.ldw : a.lda;
  const int rows = w_wave ? a.n : a.m, wave_row = wave % kHalf * 16 * L;
  Operand<ALIGNED, L> op;
  auto set_op = [&](const Unit& u) {
    int row0 = w_wave ? u.tn * BN + wave_row : u.tm * BM + wave_row;
    if (!w_wave && u.half >= 0) row0 = wave_row < BM / 2 ? row0 + u.half * (BM / 2) : rows;
    op.set(src, ld, row0, rows, a.k);
  };
  set_op(unit);

  u32x4 ring[kUnroll][L];  // stage t in slot t % 4
  const uint32_t st_off = (w_wave ? 0u : uint32_t(kTile)) + uint32_t((wave_row + (lane >> 2)) * BK) +
                          uint32_t(((lane & 3) ^ swz(lane >> 2)) * 16);
  auto put = [&](int buf, int slot, int l) {
    *reinterpret_cast<u32x4*>(smem + buf * kStage + l * 16 * BK + st_off) = ring[slot][l];
  };
  struct Frag {
    u32x4 w[NS], a[MT];
  };
  Frag f[2];
  // Fragment x (rows first) of 32-wide half kk, with JT row subtiles per wave.
  auto read = [&](auto jt, int buf, int kk, int x, Frag& d) {
    constexpr int JT = decltype(jt)::value;
    const uint8_t* p = smem + buf * kStage + fr * BK + (((kk * 2 + fh) ^ swz(fr)) * 16);
    if (x < JT)
      d.a[x < JT ? x : 0] = *reinterpret_cast<const u32x4*>(p + kTile + (wm * JT + x) * 32 * BK);
    else
      d.w[x < JT ? 0 : x - JT] = *reinterpret_cast<const u32x4*>(p + (wn * NS + x - JT) * 32 * BK);
  };

  // Factor tid + kThreads i of a unit's tile.
  auto factor = [&](const Unit& u, int i) {
    const int x = tid + kThreads * i;
    if (x < BN) return a.w_scale[min(u.tn * BN + x, a.n - 1)];
    if (x < 2 * BN) return a.bias ? bf2f(a.bias[min(u.tn * BN + x - BN, a.n - 1)]) : 0.0f;
    return x < kFactors ? a.a_scale[min(u.tm * BM + x - 2 * BN, a.m - 1)] : 0.0f;
  };
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const float v = factor(unit, i);
    if (tid + kThreads * i < kFactors) factors[0][tid + kThreads * i] = v;
  }

#pragma unroll
  for (int t = 0; t < kUnroll; ++t)
#pragma unroll
    for (int l = 0; l < L; ++l) ring[t][l] = op.load(l, t, ld, a.k);
#pragma unroll
  for (int l = 0; l < L; ++l) put(0, 0, l);
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");

  int parity = 0;
  while (true) {
    i32x16 acc[NS][MT];
#pragma unroll
    for (int i = 0; i < NS; ++i)
#pragma unroll
      for (int j = 0; j < MT; ++j)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[i][j][r] = 0;
    const bool more = unit_of(round + 1) < n_units;
    const Unit next_unit = more ? unit_at(unit_of(round + 1)) : unit;
    auto k_loop = [&](auto jt) {
      constexpr int JT = decltype(jt)::value;
      constexpr int NM = NS * JT, NR = NS + JT, HB = NM > 1 ? NM / 2 : 1;
#pragma unroll
      for (int x = 0; x < NR; ++x) read(jt, 0, 0, x, f[0]);
      for (int kt = 0; kt < KP; kt += kUnroll) {
        const bool last = kt + kUnroll == KP;
        if (last && more) set_op(next_unit);
        // Past a unit's last stage come the next one's first four; after the
        // last unit its own again (in bounds, never used).
        const int kl = last ? 0 : kt + kUnroll;
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
          // A wave issues in order: every MFMA is pinned to its share of the
          // LDS accesses and loads, writes before loads since the barrier
          // waits for them.
#pragma unroll
          for (int q = 0; q < NM; ++q) {
#pragma unroll
            for (int x = q * NR / NM; x < (q + 1) * NR / NM; ++x) read(jt, u & 1, 1, x, f[1]);
            if (q < HB) {
#pragma unroll
              for (int x = q * L / HB; x < (q + 1) * L / HB; ++x) put((u + 1) & 1, (u + 1) & 3, x);
            }
            acc[q / JT][q % JT] = mfma32_i8(f[0].w[q / JT], f[0].a[q % JT], acc[q / JT][q % JT]);
            if (q >= NM - HB) {
#pragma unroll
              for (int x = (q - NM + HB) * L / HB; x < (q - NM + HB + 1) * L / HB; ++x)
                ring[u][x] = op.load(x, kl + u, ld, a.k);
            }
            __builtin_amdgcn_sched_barrier(0);
          }
          asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
          __builtin_amdgcn_s_barrier();
          asm volatile("" ::: "memory");
#pragma unroll
          for (int q = 0; q < NM; ++q) {
            if (u + 1 < kUnroll || !last) {
#pragma unroll
              for (int x = q * NR / NM; x < (q + 1) * NR / NM; ++x) read(jt, (u + 1) & 1, 0, x, f[0]);
            }
            acc[q / JT][q % JT] = mfma32_i8(f[1].w[q / JT], f[1].a[q % JT], acc[q / JT][q % JT]);
            __builtin_amdgcn_sched_barrier(0);
          }
        }
      }
    };
    if (!kHalves || unit.half < 0)
      k_loop(std::integral_constant<int, MT>{});
    else
      k_loop(std::integral_constant<int, kHalves ? MT / 2 : MT>{});

    // The factors were written before a barrier of this tile's stages, and
    // the other half was last read before them.
    float next[kPer];
#pragma unroll
    for (int i = 0; i < kPer; ++i) next[i] = more ? factor(next_unit, i) : 0.0f;
    const int n0 = unit.tn * BN + wn * NS * 32, nj = unit.half < 0 ? MT : MT / 2;
    const int row0 = (unit.half < 0 ? 0 : unit.half * (BM / 2)) + wm * nj * 32 + fr;  // within the tile
    const float* fac = factors[parity] + wn * NS * 32 + 4 * fh;
#pragma unroll
    for (int j = 0; j < MT; ++j) {
      const int m = unit.tm * BM + row0 + j * 32;
      if (j < nj && m < a.m) {
        const float a_scale = factors[parity][2 * BN + row0 + j * 32];
        T* row = static_cast<T*>(a.out) + int64_t(m) * a.ldo + n0;
#pragma unroll
        for (int i = 0; i < NS; ++i)
#pragma unroll
          for (int p = 0; p < 2; ++p) {
            float v[2][4];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const f32x4 ws = *reinterpret_cast<const f32x4*>(fac + i * 32 + 16 * p + 8 * h);
              const f32x4 bs = *reinterpret_cast<const f32x4*>(fac + BN + i * 32 + 16 * p + 8 * h);
#pragma unroll
              for (int e = 0; e < 4; ++e)
                v[h][e] = output(acc[i][j][8 * p + 4 * h + e], a_scale, ws[e], a.bias != nullptr, bs[e]);
            }
            store_run<T, WIDE>(row + i * 32 + 16 * p, fh, v[0], v[1], a.n - (n0 + i * 32 + 16 * p));
          }
      }
    }
    if (!more) break;
    parity ^= 1;
#pragma unroll
    for (int i = 0; i < kPer; ++i)
      if (tid + kThreads * i < kFactors) factors[parity][tid + kThreads * i] = next[i];
    unit = next_unit;
    ++round;
  }
}

template <int TYPE, bool ALIGNED, bool WIDE, int WN, int WM, int NS, int MT>
hipError_t launch_tiles(const LinearI8Args& a, int blocks, hipStream_t s) {
  constexpr int BN = 32 * NS * WN, BM = 32 * MT * WM;
  const int64_t tiles = int64_t((a.m + BM - 1) / BM) * ((a.n + BN - 1) / BN);
  if (tiles > (int64_t(1) << 30)) return hipErrorInvalidValue;
  const int grid = int(tiles < blocks ? tiles : blocks);
  hipLaunchKernelGGL((linear_kernel<TYPE, ALIGNED, WIDE, WN, WM, NS, MT>), dim3(grid), dim3(WN * WM * 64), 0, s, a);
  return hipGetLastError();
}

template <int TYPE>
hipError_t launch_type(const LinearI8Args& a, int cus, hipStream_t s) {
  constexpr size_t size = sizeof(typename OutOf<TYPE>::T);
  const uintptr_t in = reinterpret_cast<uintptr_t>(a.a) | reinterpret_cast<uintptr_t>(a.w) | uintptr_t(a.lda) |
                       uintptr_t(a.ldw) | uintptr_t(a.k);
  const uintptr_t out = reinterpret_cast<uintptr_t>(a.out) | uintptr_t(a.ldo) * size;
  const bool aligned = in % 16 == 0, wide = out % 16 == 0;
  if (!aligned) return launch_tiles<TYPE, false, false, 2, 2, 2, 2>(a, 2 * cus, s);
  if (!wide) return launch_tiles<TYPE, true, false, 2, 2, 2, 2>(a, 2 * cus, s);
  const int64_t big = int64_t((a.m + 255) / 256) * ((a.n + 255) / 256);
  if (big >= 2 * cus) return launch_tiles<TYPE, true, true, 2, 4, 4, 2>(a, cus, s);
  const int64_t mid = int64_t((a.m + 127) / 128) * ((a.n + 127) / 128);
  if (mid >= cus) return launch_tiles<TYPE, true, true, 2, 2, 2, 2>(a, 2 * cus, s);
  return launch_tiles<TYPE, true, true, 2, 2, 1, 1>(a, 4 * cus, s);
}

}  // namespace

hipError_t launch_linear_i8(const LinearI8Args& a, int cus, hipStream_t s) {
  if (a.m < 1 || a.n < 1) return hipSuccess;
  switch (a.out_type) {
    case HS_TYPE_F32: return launch_type<HS_TYPE_F32>(a, cus, s);
    case HS_TYPE_BF16: return launch_type<HS_TYPE_BF16>(a, cus, s);
    case HS_TYPE_F16: return launch_type<HS_TYPE_F16>(a, cus, s);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace hs
