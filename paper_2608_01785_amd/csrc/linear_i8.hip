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
// K advances in stages of 128 bytes, one cache line of every row (loads that
// take 64 bytes of twice the rows cost the address unit as much for half the
// data: 1024 x 8192 x 8192 in 128 x 128 tiles 88 us against 77).  Half of the
// waves fetch the channels, half the rows, with 16-byte loads into a ring of D
// stages' registers:
//   stage t is loaded during stage t - D, written to LDS buffer t % 2 during
//   stage t - 1 and multiplied during stage t, in four steps of 32.
// One barrier per stage, before its last step, after each wave's writes of
// stage t + 1 and fragment reads of stage t have completed: it makes the writes
// visible to the last step's reads of stage t + 1 and retires every read of the
// buffer that the next stage overwrites.  Stages past the end of k, up to a
// multiple of D, are zeros.  Small tiles, whose stages are short against
// memory's latency, have registers for D = 4: 128 x 4608 x 3584 11.4 us against 14.0.
//
// The grid is persistent and the stages of a block's tiles form one sequence:
// the last D stages of a tile already fetch the next one's first D (four of the 64
// x 64 tiles, two of the others), and its epilogue runs under those loads.  An
// epilogue reads no memory: a tile's scales and bias come into LDS during the
// epilogue before it (stores count against the same completion counter as loads,
// so a load between them would wait for them; with such loads an epilogue took 18
// us).
//
// Large products are bound by power: 8192^3 takes 460 to 490 us (2.3 PFLOP/s)
// with normally distributed values and 354 with zeros.
#include "answer_kernels.h"
#include "horizon.h"
#include "hs_device.h"

#include <type_traits>

namespace hs {
namespace {

typedef int32_t i32x4 __attribute__((ext_vector_type(4)));
typedef int32_t i32x16 __attribute__((ext_vector_type(16)));

constexpr int kGroupM = 4;

__device__ __forceinline__ i32x16 mfma32_i8(const u32x4& a, const u32x4& b, const i32x16& c) {
  return __builtin_amdgcn_mfma_i32_32x32x32_i8(__builtin_bit_cast(i32x4, a), __builtin_bit_cast(i32x4, b), c, 0, 0, 0);
}

// A stage holds one 128-byte line of K of every row, in 16-byte chunks; a load of
// 64 lanes takes eight rows of it.
constexpr int kLine = kLinearI8Line, kChunks = kLine / 16, kLoadRows = 64 / kChunks;

// Chunk c of row r of an LDS image of lines sits at physical chunk phys(r, c), so
// that a pass of 16 lanes, which reads one logical chunk of 16 consecutive rows,
// touches each of the 64 banks once: odd rows start on bank 32, so bits 1 .. 3 of
// r permute the chunks, and bit 0 keeps the writes of two rows in different halves.
__device__ __forceinline__ int phys(int r, int c) { return c ^ ((r >> 1) & 7) ^ ((r & 1) << 2); }

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
// 8 .. 11 in `hi`, the high lane (h = 1) the four after each.  16-bit values
// change lanes so that each lane stores 16 bytes, which need no more alignment
// than an element.  Both lanes of the pair must be active.
template <typename T>
__device__ __forceinline__ void store_run(T* p, int h, const float (&lo)[4], const float (&hi)[4], int left) {
  if (left < 16) {
    store_each(p + 4 * h, lo, left - 4 * h);
    store_each(p + 8 + 4 * h, hi, left - 8 - 4 * h);
  } else if constexpr (sizeof(T) == 2) {
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
    __builtin_memcpy(p + 8 * h, &v, 16);
  } else {
    __builtin_memcpy(p + 4 * h, lo, 16);
    __builtin_memcpy(p + 8 + 4 * h, hi, 16);
  }
}

// ---------------------------------------------------------------- tiles

// One wave's share of an operand's rows: load l of a stage takes chunk lane % 8 of
// row row0 + lane / 8 + 8 l.
//   ALIGNED: base, row stride and k are multiples of 16.  A buffer resource
//   over the rows: what lies past the last row or past k reads zero
//   (linear_i8_load).
//   Otherwise (k >= 16): byte addresses, rows past the last read it again (they
//   are never stored).  The chunk that holds the end of k is read from 16 bytes
//   before that end, chunks past it from the row's start, and settle() shifts
//   and clears them once they are there, so that no load waits for another.
template <bool ALIGNED, int L>
struct Operand {
  const int8_t* base;
  __amdgpu_buffer_rsrc_t res;
  uint32_t off[ALIGNED ? 1 : L];

  __device__ __forceinline__ void set(const int8_t* p, int64_t ld, int row0, int rows, int k) {
    if constexpr (ALIGNED) {
      // A wave without rows keeps one (never stored).
      const int first = min(row0, rows - 1), span = min(rows - first, kLoadRows * L);
      base = p + int64_t(first) * ld;
      res = make_rsrc(base, linear_i8_records(span, ld, k));
      off[0] = linear_i8_offset(threadIdx.x & 63, ld);
    } else {
      const int first = min(row0, rows - 1), r = (threadIdx.x & 63) / kChunks;
      base = p + int64_t(first) * ld;
#pragma unroll
      for (int l = 0; l < L; ++l) off[l] = uint32_t(min(r + kLoadRows * l, rows - 1 - first)) * uint32_t(ld);
    }
  }
  __device__ __forceinline__ u32x4 load(int l, int stage, int64_t ld, int k) const {
    if constexpr (ALIGNED) {
      const LinearI8Load at = linear_i8_load(off[0], threadIdx.x & 63, l, stage, ld, k);
      return __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(res, at.vector, at.scalar, 0));
    } else {
      const int at = stage * kLine + int(threadIdx.x % kChunks) * 16;
      u32x4 v;
      __builtin_memcpy(&v, base + (off[l] + uint32_t(at + 16 <= k ? at : at < k ? k - 16 : 0)), 16);
      return v;
    }
  }
  // Whether a stage's chunks need settle().
  __device__ __forceinline__ static bool ends(int stage, int k) { return !ALIGNED && stage >= k / kLine; }
  // The chunk as its stage holds it, from what load() brought.
  __device__ __forceinline__ u32x4 settle(u32x4 v, int stage, int k) const {
    if constexpr (ALIGNED) {
      return v;
    } else {
      const int n = k - stage * kLine - int(threadIdx.x % kChunks) * 16;  // bytes of the chunk that k holds
      if (n <= 0) return u32x4{0, 0, 0, 0};
      if (n >= 16) return v;
      // The chunk's n bytes came last.
      const int gone = 16 - n;
      if (gone & 8) v = u32x4{v[2], v[3], 0, 0};
      if (gone & 4) v = u32x4{v[1], v[2], v[3], 0};
      return u32x4{__builtin_amdgcn_alignbyte(v[1], v[0], gone & 3), __builtin_amdgcn_alignbyte(v[2], v[1], gone & 3),
                   __builtin_amdgcn_alignbyte(v[3], v[2], gone & 3), __builtin_amdgcn_alignbyte(0u, v[3], gone & 3)};
    }
  }
};

template <int TYPE, bool ALIGNED, int D, int WN, int WM, int NS, int MT>
__global__ __launch_bounds__(WN * WM * 64, WN * WM == 8 ? 1 : NS * MT == 1 ? 4 : 2) void linear_kernel(LinearI8Args a) {
  constexpr int kWaves = WN * WM, kHalf = kWaves / 2;
  constexpr int BN = 32 * NS * WN, BM = 32 * MT * WM;
  constexpr int BK = kLine, kSteps = BK / 32;  // bytes of K per stage, and its steps
  constexpr int kUnroll = D;                  // stages in flight, and per loop body
  static_assert(D % 2 == 0, "a body's buffers alternate");
  static_assert(BN == BM && BN % (16 * kHalf) == 0, "tile split");
  constexpr int L = BN / (kLoadRows * kHalf);  // 1 KB loads per wave and stage
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
  // The XCD of a block is blockIdx % 8.  Full rounds give every XCD a range of
  // units side by side, which share operands in its L2, and so does the last
  // round with its fewer units: each XCD gets an eighth of them (896 x 5120 x
  // 2048 in 64 x 64 tiles, whose last round has 96 of 1024: 29.2 us with those
  // on one XCD).  The blocks without a unit there take the first short units.
  auto of_xcd = [](int count, int x) { return (count - x + kNumXcd - 1) / kNumXcd; };
  auto before_xcd = [](int count, int x) { return x * (count / kNumXcd) + min(x, count % kNumXcd); };
  const int xcd = blockIdx.x % kNumXcd, pos = blockIdx.x / kNumXcd;
  const int full_rounds = n_first / G, rest = n_first % G;
  const bool busy = pos < of_xcd(rest, xcd);
  const int block = before_xcd(G, xcd) + pos, busy_at = before_xcd(rest, xcd) + pos;
  const int short_at = busy ? G - rest + busy_at : block - before_xcd(rest, xcd) - of_xcd(rest, xcd);
  auto unit_of = [&](int r) {
    if (r < full_rounds) return r * G + block;
    r -= full_rounds;
    if (busy && r == 0) return full_rounds * G + busy_at;
    const int u = (r - (busy ? 1 : 0)) * G + short_at;
    return u < n_short ? n_first + u : n_units;
  };
  int round = 0;
  if (unit_of(0) >= n_units) return;
  Unit unit = unit_at(unit_of(0));

  const int KP = ((a.k + BK - 1) / BK + kUnroll - 1) / kUnroll * kUnroll;  // stages of a tile
  // The first half of the waves loads channels, the second rows.
  const bool w_wave = wave < kHalf;
  const int8_t* src = w_wave ? a.w : a.a;
  const int64_t ld = w_wave ? a.ldw : a.lda;
  const int rows = w_wave ? a.n : a.m, wave_row = wave % kHalf * kLoadRows * L;
  Operand<ALIGNED, L> op;
  auto set_op = [&](const Unit& u) {
    int row0 = w_wave ? u.tn * BN + wave_row : u.tm * BM + wave_row;
    if (!w_wave && u.half >= 0) row0 = wave_row < BM / 2 ? row0 + u.half * (BM / 2) : rows;
    op.set(src, ld, row0, rows, a.k);
  };
  set_op(unit);
  // Stages of one row of tiles may come in any order (the sums are exact).
  // Where no other block reads the same channels, each tile starts at another
  // one: rows a power of two apart would otherwise keep all blocks on the same
  // memory channels.
  auto turn_of = [&](const Unit& u) { return tiles_m == 1 ? u.tn * 11 % KP : 0; };
  int turn = turn_of(unit);
  auto turned = [&](int stage, int by) { return stage + by < KP ? stage + by : stage + by - KP; };

  u32x4 ring[kUnroll][L];  // stage t in slot t % kUnroll
  // Load l holds image rows wave_row + 8 l + lane / 8; phys() repeats with 16 of
  // them.
  const int put_row = wave_row + lane / kChunks;
  const uint32_t put_at = (w_wave ? 0u : uint32_t(kTile)) + uint32_t(put_row * BK);
  const uint32_t put_chunk[2] = {uint32_t(phys(put_row, lane % kChunks) * 16),
                                 uint32_t(phys(put_row + kLoadRows, lane % kChunks) * 16)};
  auto put = [&](int buf, int l, const u32x4& v) {
    *reinterpret_cast<u32x4*>(smem + buf * kStage + l * kLoadRows * BK + put_at +
                              put_chunk[l & 1]) = v;
  };
  // Over what put() wrote of a stage that holds the end of k: one branch a
  // stage (with one for every chunk 777 x 5001 x 2047 took 34 us, not 31).
  auto put_end = [&](int buf, int slot, int stage) {
    if (op.ends(stage, a.k)) {
#pragma unroll
      for (int l = 0; l < L; ++l) put(buf, l, op.settle(ring[slot][l], stage, a.k));
    }
  };
  struct Frag {
    u32x4 w[NS], a[MT];
  };
  Frag f[2];
  // Fragment x (rows first) of step kk, with JT row subtiles per wave.
  auto read = [&](auto jt, int buf, int kk, int x, Frag& d) {
    constexpr int JT = decltype(jt)::value;
    const uint8_t* p = smem + buf * kStage + fr * BK + phys(fr, kk * 2 + fh) * 16;
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
    for (int l = 0; l < L; ++l) ring[t][l] = op.load(l, turned(t, turn), ld, a.k);
#pragma unroll
  for (int l = 0; l < L; ++l) put(0, l, ring[0][l]);
  put_end(0, 0, turn);
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
    const int next_turn = turn_of(next_unit);
    auto k_loop = [&](auto jt) {
      constexpr int JT = decltype(jt)::value;
      constexpr int NM = NS * JT, NR = NS + JT;
#pragma unroll
      for (int x = 0; x < NR; ++x) read(jt, 0, 0, x, f[0]);
      for (int kt = 0; kt < KP; kt += kUnroll) {
        const bool last = kt + kUnroll == KP;
        if (last && more) set_op(next_unit);
        // Past a unit's last stage come the next one's first ones; after the
        // last unit its own again (in bounds, never used).
        const int kl = last ? 0 : kt + kUnroll, kl_turn = last ? next_turn : turn;
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
          const int buf = u & 1;
#pragma unroll
          for (int kk = 0; kk < kSteps; ++kk) {
            // A wave issues in order: every MFMA is pinned to its share of the
            // LDS accesses and loads.  The steps before the barrier write
            // stage t + 1 first, then load into the registers that held stage t.
            constexpr int kSlots = (kSteps - 1) * NM, kPutEnd = kSlots / 2, kLoadBegin = kSlots - kPutEnd;
#pragma unroll
            for (int q = 0; q < NM; ++q) {
              const int slot = kk * NM + q;
              if (kk + 1 < kSteps) {
#pragma unroll
                for (int x = q * NR / NM; x < (q + 1) * NR / NM; ++x) read(jt, buf, kk + 1, x, f[(kk + 1) & 1]);
                if (slot < kPutEnd) {
#pragma unroll
                  for (int x = slot * L / kPutEnd; x < (slot + 1) * L / kPutEnd; ++x)
                    put(1 - buf, x, ring[(u + 1) % kUnroll][x]);
                }
              } else if (u + 1 < kUnroll || !last) {
#pragma unroll
                for (int x = q * NR / NM; x < (q + 1) * NR / NM; ++x) read(jt, 1 - buf, 0, x, f[0]);
              }
              acc[q / JT][q % JT] = mfma32_i8(f[kk & 1].w[q / JT], f[kk & 1].a[q % JT], acc[q / JT][q % JT]);
              if (kk + 1 < kSteps && slot >= kLoadBegin) {
                constexpr int kN = kSlots - kLoadBegin;
#pragma unroll
                for (int x = (slot - kLoadBegin) * L / kN; x < (slot - kLoadBegin + 1) * L / kN; ++x)
                  ring[u][x] = op.load(x, turned(kl + u, kl_turn), ld, a.k);
              }
              __builtin_amdgcn_sched_barrier(0);
            }
            if (kk + 2 == kSteps) {
              put_end(1 - buf, (u + 1) % kUnroll,
                      u + 1 < kUnroll || !last ? turned(kt + u + 1, turn) : next_turn);
              asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
              __builtin_amdgcn_s_barrier();
              asm volatile("" ::: "memory");
            }
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
            store_run(row + i * 32 + 16 * p, fh, v[0], v[1], a.n - (n0 + i * 32 + 16 * p));
          }
      }
    }
    if (!more) break;
    parity ^= 1;
#pragma unroll
    for (int i = 0; i < kPer; ++i)
      if (tid + kThreads * i < kFactors) factors[parity][tid + kThreads * i] = next[i];
    unit = next_unit;
    turn = next_turn;
    ++round;
  }
}

// ---------------------------------------------------------------- few rows

// Few rows, in groups of 32 MT: what counts is reading w once, as fast as memory
// gives it.  A block takes 32 NT channels and its eight waves share K, wave v the
// 128 bytes of stages v, v + 8, ...: one cache line of every row to a load's eight
// lanes, two stages of loads in flight per wave.  Each wave turns its lines
// into MFMA operands through an LDS image of its own, so nothing in the loop
// waits for another wave; their sums meet in LDS at the end.
constexpr int kFewWaves = 8;

template <int TYPE, bool ALIGNED, int MT, int NT>
__global__ __launch_bounds__(kFewWaves * 64, MT == 1 && ALIGNED ? 4 : 2) void few_kernel(LinearI8Args a) {
  constexpr int kRow = 128, kImage = (NT + MT) * 32 * kRow;
  constexpr int D = 2;  // stages of loads in flight
  __shared__ __attribute__((aligned(1024))) uint8_t smem[kFewWaves * kImage];
  using T = typename OutOf<TYPE>::T;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int fr = lane & 31, fh = lane >> 5;
  const int n0 = blockIdx.x * 32 * NT;

  Operand<ALIGNED, 4 * NT> wop;
  Operand<ALIGNED, 4 * MT> aop;
  wop.set(a.w, a.ldw, n0, a.n, a.k);
  const int m0 = blockIdx.y * 32 * MT;
  aop.set(a.a, a.lda, m0, a.m, a.k);
  u32x4 w[D][4 * NT], x[D][4 * MT];
  auto load = [&](int slot, int stage) {
#pragma unroll
    for (int l = 0; l < 4 * NT; ++l) w[slot][l] = wop.load(l, stage, a.ldw, a.k);
#pragma unroll
    for (int l = 0; l < 4 * MT; ++l) x[slot][l] = aop.load(l, stage, a.lda, a.k);
  };
  uint8_t* image = smem + wave * kImage;
  // Load l holds rows 8 l + lane / 8, and phys() repeats with 16 rows.
  const uint32_t put_off = (lane >> 3) * kRow + phys(lane >> 3, lane & 7) * 16;
  const uint32_t put_odd = (lane >> 3) * kRow + phys(8 + (lane >> 3), lane & 7) * 16;

  i32x16 acc[NT][MT];
#pragma unroll
  for (int i = 0; i < NT; ++i)
#pragma unroll
    for (int j = 0; j < MT; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[i][j][r] = 0;
  const int stages = (a.k + kRow - 1) / kRow, rounds = (stages + kFewWaves - 1) / kFewWaves;
  // As in linear_kernel, every block starts at another round.
  const int turn = blockIdx.x * 3 % rounds;
  auto stage_of = [&](int i) {
    const int round = i + turn < rounds ? i + turn : i + turn - rounds;
    return i < rounds ? wave + round * kFewWaves : stages + 1;
  };
#pragma unroll
  for (int d = 0; d < D; ++d) load(d, stage_of(d));
  // At the end wave v has the groups of four channels v, v + 8, ... of a lane:
  // group 4 (MT i + j) + g is number g of channel subtile i and row subtile j.
  // Their factors come behind the first stages.
  constexpr int kGroups = 4 * MT * NT, kOwn = (kGroups + kFewWaves - 1) / kFewWaves;
  auto row_of = [&](int o) { return m0 + (wave + kFewWaves * o) / 4 % MT * 32 + fr; };
  auto channel_of = [&](int o) { return n0 + (wave + kFewWaves * o) / (4 * MT) * 32 + 8 * (wave & 3) + 4 * fh; };
  auto mine = [&](int o) { return wave + kFewWaves * o < kGroups && row_of(o) < a.m && channel_of(o) < a.n; };
  float a_scale[kOwn] = {}, w_scale[kOwn][4] = {}, bias[kOwn][4] = {};
#pragma unroll
  for (int o = 0; o < kOwn; ++o) {
    if (!mine(o)) continue;
    a_scale[o] = a.a_scale[row_of(o)];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int c = min(channel_of(o) + e, a.n - 1);
      w_scale[o][e] = a.w_scale[c];
      if (a.bias) bias[o][e] = bf2f(a.bias[c]);
    }
  }
  for (int i = 0; i < rounds; i += D) {
#pragma unroll
    for (int d = 0; d < D; ++d) {
      const int stage = stage_of(i + d);
      auto put = [&](int l, const u32x4& v) {
        *reinterpret_cast<u32x4*>(image + l * 8 * kRow + ((l & 1) ? put_odd : put_off)) = v;
      };
      if (wop.ends(stage, a.k)) {
#pragma unroll
        for (int l = 0; l < 4 * NT; ++l) w[d][l] = wop.settle(w[d][l], stage, a.k);
#pragma unroll
        for (int l = 0; l < 4 * MT; ++l) x[d][l] = aop.settle(x[d][l], stage, a.k);
      }
#pragma unroll
      for (int l = 0; l < 4 * NT; ++l) put(l, w[d][l]);
#pragma unroll
      for (int l = 0; l < 4 * MT; ++l) put(4 * NT + l, x[d][l]);
      load(d, stage_of(i + d + D));  // zeros past the end of k
      // The image is this wave's alone, and LDS serves one wave in order.
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
      for (int kk = 0; kk < 4; ++kk) {
        const uint8_t* p = image + fr * kRow + phys(fr, 2 * kk + fh) * 16;
        u32x4 wf[NT], af[MT];
#pragma unroll
        for (int i = 0; i < NT; ++i) wf[i] = *reinterpret_cast<const u32x4*>(p + i * 32 * kRow);
#pragma unroll
        for (int j = 0; j < MT; ++j) af[j] = *reinterpret_cast<const u32x4*>(p + (NT + j) * 32 * kRow);
#pragma unroll
        for (int i = 0; i < NT; ++i)
#pragma unroll
          for (int j = 0; j < MT; ++j) acc[i][j] = mfma32_i8(wf[i], af[j], acc[i][j]);
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
  }

  // Sums of four channels and one row per lane.
  __syncthreads();
  int32_t* part = reinterpret_cast<int32_t*>(smem);
#pragma unroll
  for (int i = 0; i < NT; ++i)
#pragma unroll
    for (int j = 0; j < MT; ++j)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        *reinterpret_cast<i32x4*>(part + (((4 * (MT * i + j) + g) * kFewWaves + wave) * 64 + lane) * 4) =
            i32x4{acc[i][j][4 * g], acc[i][j][4 * g + 1], acc[i][j][4 * g + 2], acc[i][j][4 * g + 3]};
  __syncthreads();
#pragma unroll
  for (int o = 0; o < kOwn; ++o) {
    if (!mine(o)) continue;
    const int32_t* from = part + ((wave + kFewWaves * o) * kFewWaves * 64 + lane) * 4;
    i32x4 sum = {0, 0, 0, 0};
#pragma unroll
    for (int v = 0; v < kFewWaves; ++v) sum += *reinterpret_cast<const i32x4*>(from + v * 64 * 4);
    float v[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = output(sum[e], a_scale[o], w_scale[o][e], a.bias != nullptr, bias[o][e]);
    const int n = channel_of(o);
    T* p = static_cast<T*>(a.out) + int64_t(row_of(o)) * a.ldo + n;
    if (n + 4 > a.n) {
      store_each(p, v, a.n - n);
    } else if constexpr (sizeof(T) == 4) {
      __builtin_memcpy(p, v, 16);
    } else {
      const u32x2 two = {pack2<T>(v[0], v[1]), pack2<T>(v[2], v[3])};
      __builtin_memcpy(p, &two, 8);
    }
  }
}

// Rows of fewer than 16 bytes that are not aligned: one thread an output.
template <int TYPE>
__global__ __launch_bounds__(256) void short_kernel(LinearI8Args a) {
  using T = typename OutOf<TYPE>::T;
  const int64_t outputs = int64_t(a.m) * a.n;
  for (int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x; i < outputs; i += int64_t(gridDim.x) * 256) {
    const int m = int(i / a.n), n = int(i % a.n);
    int32_t sum = 0;
    for (int k = 0; k < a.k; ++k) sum += int32_t(a.a[int64_t(m) * a.lda + k]) * a.w[int64_t(n) * a.ldw + k];
    static_cast<T*>(a.out)[int64_t(m) * a.ldo + n] =
        T(output(sum, a.a_scale[m], a.w_scale[n], a.bias != nullptr, a.bias ? bf2f(a.bias[n]) : 0.0f));
  }
}

template <int TYPE, bool ALIGNED, int D, int WN, int WM, int NS, int MT>
hipError_t launch_tiles(const LinearI8Args& a, int blocks, hipStream_t s) {
  constexpr int BN = 32 * NS * WN, BM = 32 * MT * WM;
  const int64_t tiles = int64_t((a.m + BM - 1) / BM) * ((a.n + BN - 1) / BN);
  if (tiles > (int64_t(1) << 30)) return hipErrorInvalidValue;
  const int grid = int(tiles < blocks ? tiles : blocks);
  hipLaunchKernelGGL((linear_kernel<TYPE, ALIGNED, D, WN, WM, NS, MT>), dim3(grid), dim3(WN * WM * 64), 0, s, a);
  return hipGetLastError();
}

template <int TYPE, bool ALIGNED>
hipError_t launch_choice(const LinearI8Args& a, int choice, int cus, hipStream_t s) {
  const int few_rows = choice == kLinearI8Few32 ? 32 : 64, few_channels = choice == kLinearI8Few64x64 ? 64 : 32;
  const dim3 few((a.n + few_channels - 1) / few_channels, (a.m + few_rows - 1) / few_rows);
  switch (choice) {
    case kLinearI8Few32:
      hipLaunchKernelGGL((few_kernel<TYPE, ALIGNED, 1, 1>), few, dim3(kFewWaves * 64), 0, s, a);
      return hipGetLastError();
    case kLinearI8Few64:
      hipLaunchKernelGGL((few_kernel<TYPE, ALIGNED, 2, 1>), few, dim3(kFewWaves * 64), 0, s, a);
      return hipGetLastError();
    case kLinearI8Few64x64:
      if constexpr (!ALIGNED) return hipErrorInvalidValue;
      hipLaunchKernelGGL((few_kernel<TYPE, true, 2, 2>), few, dim3(kFewWaves * 64), 0, s, a);
      return hipGetLastError();
    case kLinearI8Tile64: return launch_tiles<TYPE, ALIGNED, 4, 2, 2, 1, 1>(a, 4 * cus, s);
    case kLinearI8Tile128: return launch_tiles<TYPE, ALIGNED, 2, 2, 2, 2, 2>(a, 2 * cus, s);
    default:
      if constexpr (ALIGNED) return launch_tiles<TYPE, ALIGNED, 2, 2, 4, 4, 2>(a, cus, s);
      return hipErrorInvalidValue;
  }
}

template <int TYPE>
hipError_t launch_type(const LinearI8Args& a, int cus, hipStream_t s) {
  const uintptr_t in = reinterpret_cast<uintptr_t>(a.a) | reinterpret_cast<uintptr_t>(a.w) | uintptr_t(a.lda) |
                       uintptr_t(a.ldw) | uintptr_t(a.k);
  const int choice = linear_i8_choice(a.m, a.n, a.k, cus, in % 16 == 0);
  if (in % 16 == 0) return launch_choice<TYPE, true>(a, choice, cus, s);
  if (a.k >= 16) return launch_choice<TYPE, false>(a, choice, cus, s);
  const int64_t blocks = (int64_t(a.m) * a.n + 255) / 256;
  hipLaunchKernelGGL(short_kernel<TYPE>, dim3(unsigned(blocks < 16 * cus ? blocks : 16 * cus)), dim3(256), 0, s, a);
  return hipGetLastError();
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
