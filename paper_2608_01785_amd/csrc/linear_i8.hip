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
// A block of WN x WM waves computes tiles of 32 NS WN channels x 32 MT WM rows;
// K advances in stages of 128 bytes, one cache line of every row, through two
// LDS buffers, fetched two to three stages ahead into registers.  The grid is
// persistent and the stages of a block's tiles form one sequence: the last
// stages of a tile already fetch the next one's first, and its epilogue runs
// under those loads.
#include "answer_kernels.h"
#include "horizon.h"
#include "hs_device.h"

namespace hs {
namespace {

typedef int32_t i32x4 __attribute__((ext_vector_type(4)));
typedef int32_t i32x16 __attribute__((ext_vector_type(16)));

constexpr int BK = 128;       // bytes of K per stage: 8 chunks of 16
constexpr int kKk = BK / 32;  // MFMA steps per stage
constexpr int kGroupM = 4;

__device__ __forceinline__ i32x16 mfma32_i8(const u32x4& a, const u32x4& b, const i32x16& c) {
  return __builtin_amdgcn_mfma_i32_32x32x32_i8(__builtin_bit_cast(i32x4, a), __builtin_bit_cast(i32x4, b), c, 0, 0, 0);
}

// 16-byte chunk c of tile row r sits at physical chunk c ^ ...: a pass of 16
// lanes reads one logical chunk of eight even and eight odd rows, and odd rows
// start on bank 32, so bits 1 .. 3 of r permute the chunks; bit 0 keeps the
// writes of two rows in different halves.
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
__device__ __forceinline__ float scaled(int32_t sum, float a_scale, float w_scale) {
#pragma clang fp contract(off)
  const float s = a_scale * w_scale;
  return float(sum) * s;
}
__device__ __forceinline__ float biased(float v, uint16_t bias) {
#pragma clang fp contract(off)
  return v + bf2f(bias);
}

// Four consecutive channels n .. n + 3 of one row.  WIDE: the address of a
// multiple of four channels is aligned for one store.
template <int TYPE, bool WIDE>
__device__ __forceinline__ void store4(const LinearI8Args& a, int m, int n, const i32x4& sum, float a_scale,
                                       const f32x4& ws, const float* b) {
  using T = typename OutOf<TYPE>::T;
  T* p = static_cast<T*>(a.out) + int64_t(m) * a.ldo + n;
  float v[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
#pragma clang fp contract(off)
    v[e] = scaled(sum[e], a_scale, ws[e]);
    if (a.bias) v[e] = v[e] + b[e];
  }
  if (WIDE && n + 4 <= a.n) {
    typedef T T4 __attribute__((ext_vector_type(4)));
    *reinterpret_cast<T4*>(p) = T4{T(v[0]), T(v[1]), T(v[2]), T(v[3])};
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (n + e < a.n) p[e] = T(v[e]);
  }
}

// ---------------------------------------------------------------- tiles

// Operand rows of one tile: the 16-byte chunk (lane & 7) of rows
// (lane >> 3) + 8 (wave + WAVES l).
//   ALIGNED: base, row stride and k are multiples of 16.  A buffer resource
//   over the tile's rows: what lies past the last row or past k reads zero.
//   Otherwise: byte addresses, rows past the last read it again (they are
//   never stored) and the chunk that holds the end of k is read from 16 bytes
//   before that end and shifted.
template <bool ALIGNED, int WAVES, int L>
struct Operand {
  const int8_t* base;
  __amdgpu_buffer_rsrc_t res;
  uint32_t off, off_tail;  // ALIGNED: load 0's offset, and in the stage that holds the end of k
  uint32_t offs[ALIGNED ? 1 : L];

  __device__ __forceinline__ void set(const int8_t* p, int64_t ld, int row0, int rows, int k) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r = 8 * wave + (lane >> 3), c = lane & 7;
    const int left = rows - row0;
    base = p + int64_t(row0) * ld;
    if constexpr (ALIGNED) {
      const int span = min(left, 8 * WAVES * L);
      res = make_rsrc(base, uint32_t(span - 1) * uint32_t(ld) + uint32_t(k));
      off = uint32_t(r) * uint32_t(ld) + uint32_t(c * 16);
      off_tail = c * 16 < (k & (BK - 1)) ? off : 0x80000000u;
    } else {
#pragma unroll
      for (int l = 0; l < L; ++l) offs[l] = uint32_t(min(r + 8 * WAVES * l, left - 1)) * uint32_t(ld) + uint32_t(c * 16);
    }
  }
  __device__ __forceinline__ u32x4 load(int l, int stage, int64_t ld, int k) const {
    const int whole = k / BK;  // stages without the end of k
    if constexpr (ALIGNED) {
      const uint32_t v = stage < whole ? off : stage > whole ? 0x80000000u : off_tail;
      const uint32_t s = uint32_t(min(stage, (k - 1) / BK)) * BK + uint32_t(8 * WAVES * l) * uint32_t(ld);
      return __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(res, v, s, 0));
    } else {
      u32x4 v = {0, 0, 0, 0};
      const int8_t* p = base + int64_t(stage) * BK;
      if (stage < whole) {
        __builtin_memcpy(&v, p + offs[l], 16);
        return v;
      }
      const int n = k - stage * BK - (int(threadIdx.x) & 7) * 16;  // bytes of the chunk that k holds
      if (n >= 16) {
        __builtin_memcpy(&v, p + offs[l], 16);
      } else if (n > 0 && k >= 16) {
        __builtin_memcpy(&v, p + offs[l] - (16 - n), 16);
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
          const uint32_t b = uint32_t(uint8_t(p[offs[l] + i])) << (8 * (i & 3));
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
  constexpr int kWaves = WN * WM;
  constexpr int BN = 32 * NS * WN, BM = 32 * MT * WM;
  constexpr int kWBytes = BN * BK, kABytes = BM * BK;
  constexpr int kStage = kWBytes + kABytes;
  constexpr int WL = BN / (8 * kWaves), AL = BM / (8 * kWaves);  // 1 KB loads per wave and stage
  static_assert(WL * 8 * kWaves == BN && AL * 8 * kWaves == BM, "tile split");
  __shared__ __attribute__((aligned(1024))) uint8_t smem[2 * kStage];

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wn = wave % WN, wm = wave / WN;
  const int fr = lane & 31, fh = lane >> 5;

  // Tiles in groups of kGroupM row tiles, rows fastest; round r gives block b
  // tile r G + b, with the blocks of an XCD on a contiguous range.
  const int tiles_m = (a.m + BM - 1) / BM, tiles_n = (a.n + BN - 1) / BN;
  const int n_tiles = tiles_m * tiles_n, G = gridDim.x;
  const int per_group = kGroupM * tiles_n;
  auto coords = [&](int t, int& tm, int& tn) {
    const int first_m = t / per_group * kGroupM;
    const int gsize = min(tiles_m - first_m, kGroupM);
    tm = first_m + t % per_group % gsize;
    tn = t % per_group / gsize;
  };
  int tile = xcd_remap(blockIdx.x, G);
  if (tile >= n_tiles) return;

  const int KT = (a.k + BK - 1) / BK, KP = (KT + 1) & ~1;  // stages of a tile, to an even number
  // The stage to be loaded next: its tile's operands and its number in it.
  Operand<ALIGNED, kWaves, WL> wop;
  Operand<ALIGNED, kWaves, AL> aop;
  int load_tile = tile, load_kt = 0;
  auto set_ops = [&](int t) {
    int tm, tn;
    coords(t, tm, tn);
    wop.set(a.w, a.ldw, tn * BN, a.n, a.k);
    aop.set(a.a, a.lda, tm * BM, a.m, a.k);
  };
  set_ops(tile);
  // After a tile's last stage come the next tile's; past the last tile the
  // loads repeat its first stages (in bounds, never used).
  auto advance = [&] {
    if (++load_kt == KP) {
      load_kt = 0;
      if (load_tile + G < n_tiles) {
        load_tile += G;
        set_ops(load_tile);
      }
    }
  };

  constexpr int NM = NS * MT, NR = NS + MT, NL = WL + AL;
  u32x4 gr[2][NL];
  auto load = [&](int slot, int l) {
    gr[slot][l] = l < WL ? wop.load(l < WL ? l : 0, load_kt, a.ldw, a.k) : aop.load(l < WL ? 0 : l - WL, load_kt, a.lda, a.k);
  };
  const uint32_t st_row = 8 * wave + (lane >> 3);
  const uint32_t st_off = st_row * BK + phys(st_row, lane & 7) * 16;  // the row's bits 0 .. 3 are every load's
  auto put = [&](int buf, int slot, int l) {
    const uint32_t at = l < WL ? uint32_t(l * 8 * kWaves * BK) : uint32_t(kWBytes + (l - WL) * 8 * kWaves * BK);
    *reinterpret_cast<u32x4*>(smem + buf * kStage + at + st_off) = gr[slot][l];
  };
  struct Frag {
    u32x4 w[NS], a[MT];
  };
  Frag f[2];
  // Fragment x (0 .. NR - 1, rows first) of step kk.
  auto read = [&](int buf, int kk, int x, Frag& d) {
    const uint8_t* p = smem + buf * kStage + fr * BK + phys(fr, 2 * kk + fh) * 16;
    if (x < MT)
      d.a[x < MT ? x : 0] = *reinterpret_cast<const u32x4*>(p + kWBytes + (wm * MT + x) * 32 * BK);
    else
      d.w[x < MT ? 0 : x - MT] = *reinterpret_cast<const u32x4*>(p + (wn * NS + x - MT) * 32 * BK);
  };

  // Stages 0 and 1 into the register slots, 0 on to LDS, 2 into its slot.
#pragma unroll
  for (int t = 0; t < 2; ++t) {
#pragma unroll
    for (int l = 0; l < NL; ++l) load(t, l);
    advance();
  }
  __builtin_amdgcn_sched_barrier(0);
#pragma unroll
  for (int l = 0; l < NL; ++l) put(0, 0, l);
#pragma unroll
  for (int l = 0; l < NL; ++l) load(0, l);
  advance();
  __builtin_amdgcn_sched_barrier(0);
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
#pragma unroll
  for (int x = 0; x < NR; ++x) read(0, 0, x, f[0]);
  __builtin_amdgcn_sched_barrier(0);

  // Stage t multiplies buffer t % 2, writes stage t + 1 to the other one in its
  // first two steps and loads stage t + 3 into the registers that held it in
  // the middle two.  Each step's fragments are read during the step before.
  // One barrier per stage, inside the last step, whose fragments have been
  // read by then: it follows every wave's writes of stage t + 1 (whose first
  // fragments are read next) and its reads of buffer t % 2 (which the next
  // stage overwrites).  Every MFMA is issued with its share of the LDS accesses
  // and loads, pinned by scheduling barriers, since a wave issues in order.
  constexpr int H = (NL + 1) / 2, HB = NM / 2;
  while (true) {
    i32x16 acc[NS][MT];
#pragma unroll
    for (int i = 0; i < NS; ++i)
#pragma unroll
      for (int j = 0; j < MT; ++j)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[i][j][r] = 0;

    for (int kt = 0; kt < KP; kt += 2) {
#pragma unroll
      for (int u = 0; u < 2; ++u) {
#pragma unroll
        for (int kk = 0; kk < kKk; ++kk) {
          const bool last = kk + 1 == kKk;
          const int nw = kk == 0 ? H : kk == 1 ? NL - H : 0;  // writes: 0 .. H - 1, then the rest
          const int nl = kk == 1 ? H : kk == 2 ? NL - H : 0;  // loads likewise, one step later
#pragma unroll
          for (int q = 0; q < NM; ++q) {
            if (last && q == HB) {
              asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
              __builtin_amdgcn_s_barrier();
              asm volatile("" ::: "memory");
            }
            if (!last) {
#pragma unroll
              for (int x = q * NR / NM; x < (q + 1) * NR / NM; ++x) read(u, kk + 1, x, f[(kk + 1) & 1]);
            } else if (q >= HB) {
#pragma unroll
              for (int x = (q - HB) * NR / (NM - HB); x < (q - HB + 1) * NR / (NM - HB); ++x) read(1 - u, 0, x, f[0]);
            }
#pragma unroll
            for (int x = q * nw / NM; x < (q + 1) * nw / NM; ++x) put(1 - u, 1 - u, kk * H + x);
            const int i = q / MT, j = q % MT;
            acc[i][j] = mfma32_i8(f[kk & 1].w[i], f[kk & 1].a[j], acc[i][j]);
#pragma unroll
            for (int x = q * nl / NM; x < (q + 1) * nl / NM; ++x) load(1 - u, (kk - 1) * H + x);
            __builtin_amdgcn_sched_barrier(0);
          }
        }
        advance();
      }
    }

    int tm, tn;
    coords(tile, tm, tn);
    const int n0 = tn * BN + wn * NS * 32 + 4 * fh, m0 = tm * BM + wm * MT * 32 + fr;
    float a_scale[MT];
#pragma unroll
    for (int j = 0; j < MT; ++j) a_scale[j] = a.a_scale[min(m0 + j * 32, a.m - 1)];
#pragma unroll
    for (int i = 0; i < NS; ++i)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const int n = n0 + i * 32 + 8 * g;
        f32x4 ws;
        float b[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int c = min(n + e, a.n - 1);
          ws[e] = a.w_scale[c];
          b[e] = a.bias ? bf2f(a.bias[c]) : 0.0f;
        }
#pragma unroll
        for (int j = 0; j < MT; ++j) {
          const i32x16& c = acc[i][j];
          if (m0 + j * 32 < a.m)
            store4<TYPE, WIDE>(a, m0 + j * 32, n, i32x4{c[4 * g], c[4 * g + 1], c[4 * g + 2], c[4 * g + 3]},
                               a_scale[j], ws, b);
        }
      }
    tile += G;
    if (tile >= n_tiles) break;
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
  const size_t size = TYPE == HS_TYPE_F32 ? 4 : 2;
  const uintptr_t in = reinterpret_cast<uintptr_t>(a.a) | reinterpret_cast<uintptr_t>(a.w) | uintptr_t(a.lda) |
                       uintptr_t(a.ldw) | uintptr_t(a.k);
  const uintptr_t out = reinterpret_cast<uintptr_t>(a.out) | uintptr_t(a.ldo) * size;
  const bool aligned = in % 16 == 0, wide = out % (4 * size) == 0;
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
