// Attention of one row a sequence over a paged cache whose sequences share their
// first positions in groups:
//   o[i, h] = sum_p w[p] v[p] / sum_p w[p],  w[p] = e^(q[i, h] . k[p] / sqrt(dh))
// over the prefix of the row's group and the row's own positions behind it.
//
// Single-row attention reads a sequence's keys for the few query heads that share
// them.  Behind a shared prefix all rows of a group want the same keys, so the group's
// (row, query head) pairs of one key/value head become the columns of one product
// and the prefix is read once for them.  A block takes a tile of such columns and a
// range of keys, of a group's prefix or of what one row has to itself; it leaves
// the unnormalised output, the maximum and the sum of its columns, and a second
// launch joins what belongs to a row.
//
// The unit is that of single-row attention (decode_unit.h): wavefront w takes the
// 32-key tiles w, w + 4, ... of the range, loads them as whole lines a tile ahead and
// passes them through an LDS image of its own into MFMA layout, S^T = K Q^T and
// O^T = V^T P^T, with a running softmax.
//
// What the device arrays say is checked here: a slot outside the cache is read as
// zeros and makes its rows NaN, and no range leaves the table.
#include "answer_device.h"
#include "decode_policy.h"
#include "decoding_kernels.h"

namespace hs {
namespace {

constexpr int kThreads = 256;
constexpr int kTileKeys = kv_tile_keys;
constexpr float kInf = __builtin_inff();

struct Group {
  int lo, hi;   // its rows
  int prefix;   // its shared positions
  int tile;     // of the group's row tiles
};

__device__ __forceinline__ int clamped(int v, int lo, int hi) { return min(max(v, lo), hi); }

// Rows [lo, hi) and prefix of group g, inside what the arguments allow.
__device__ __forceinline__ Group group_at(const PrefixArgs& a, int g) {
  Group r;
  r.lo = clamped(a.offsets[g], 0, a.n_seqs);
  r.hi = clamped(a.offsets[g + 1], r.lo, a.n_seqs);
  r.prefix = a.prefix[g];
  r.tile = 0;
  return r;
}

__device__ __forceinline__ int first_lane(int v) { return __builtin_amdgcn_readfirstlane(v); }

// The group that holds row tile `t` (tiles of `rows` columns, `per_head` of them a
// row); lo == hi where there is none.  A wavefront looks at 64 groups at a time.
__device__ __forceinline__ Group group_of_tile(const PrefixArgs& a, int t, int rows, int per_head) {
  const int lane = threadIdx.x & 63;
  for (int g0 = 0; g0 < a.n_groups; g0 += 64) {
    Group r{0, 0, 0, 0};
    if (g0 + lane < a.n_groups) r = group_at(a, g0 + lane);
    const int tiles = int((int64_t(r.hi - r.lo) * per_head + rows - 1) / rows);
    int end = tiles;  // tiles up to and with this lane's group
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int below = __shfl_up(end, o, 64);
      if (lane >= o) end += below;
    }
    const uint64_t mask = __ballot(t < end);
    if (mask != 0) {
      const int w = __builtin_ctzll(mask);
      Group f;
      f.lo = __shfl(r.lo, w, 64);
      f.hi = __shfl(r.hi, w, 64);
      f.prefix = __shfl(r.prefix, w, 64);
      f.tile = t - __shfl(end - tiles, w, 64);
      return f;
    }
    t -= __shfl(end, 63, 64);
  }
  return Group{0, 0, 0, 0};
}

// The prefix of a row's group (0 where no group holds the row).
__device__ __forceinline__ int prefix_of_row(const PrefixArgs& a, int row) {
  const int lane = threadIdx.x & 63;
  for (int g0 = 0; g0 < a.n_groups; g0 += 64) {
    const int g = g0 + lane;
    const bool mine = g < a.n_groups && a.offsets[g] <= row && row < a.offsets[g + 1];
    const uint64_t mask = __ballot(mine);
    if (mask != 0) return a.prefix[first_lane(g0 + __builtin_ctzll(mask))];
  }
  return 0;
}

// Partial states: [split][row][query head], prefix splits first.
__device__ __forceinline__ int64_t part_index(const PrefixArgs& a, int split, int row, int head) {
  return (int64_t(split) * a.n_seqs + row) * a.hq + head;
}
__device__ __forceinline__ float* part_stats(const PrefixArgs& a, int splits) {
  return static_cast<float*>(a.part) + int64_t(splits) * a.n_seqs * a.hq * a.dh;
}

template <int DH, int NQ>
struct Smem {
  static constexpr int kTile = kTileKeys * DH * 2;  // bytes of a tile's keys, and of its values
  static constexpr int kCols = 16 * NQ;
  static constexpr int kPass = 64;                  // dimensions of a pass of the join of wavefronts
  union {
    uint8_t tile[4][kTile];
    float red_o[4][kPass][kCols + 1];
  };
  float red_m[4][kCols], red_l[4][kCols];
};

// Largest and total value over the four lanes that hold one column's keys.
__device__ __forceinline__ float quarter_max(float v) {
  v = fmaxf(v, xor_lane<16>(v));
  return fmaxf(v, xor_lane<32>(v));
}
__device__ __forceinline__ float quarter_sum(float v) {
  v += xor_lane<16>(v);
  return v + xor_lane<32>(v);
}

// Columns m0 .. m0 + n_cols - 1 of rows lo .. (column m: row lo + m / G, query head
// head * G + m % G) over keys [k_lo, k_hi) of sequence `owner`'s pages, as partial
// state `split`.
template <int DH, int NQ, typename T>
__device__ __forceinline__ void unit(const PrefixArgs& a, int lo, int m0, int n_cols, int head, int owner, int k_lo,
                                     int k_hi, int split, int splits, Smem<DH, NQ>& sm) {
  constexpr int TK = kTileKeys;
  constexpr int NKB = DH / 32, NDS = DH / 16;
  constexpr int kTile = Smem<DH, NQ>::kTile, NL = kTile / 1024;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = first_lane(tid >> 6);
  const int fr = lane & 15, fh = lane >> 4;
  const int G = a.hq / a.hkv;
  const int64_t head_elems = int64_t(a.page) * DH, slot_elems = head_elems * a.hkv;
  const int t0 = k_lo / TK, n_tiles = (k_hi + TK - 1) / TK - t0;
  const int my_tiles = n_tiles > wave ? (n_tiles - wave + 3) / 4 : 0;
  const int32_t* pages = a.table + int64_t(owner) * a.pages_per_seq;

  // The page of the wavefront's tile i (clamped to its last one) and the tile's
  // place in it.
  bool bad = false;
  auto slot_of = [&](int i) {
    const int key = (t0 + wave + 4 * min(i, my_tiles - 1)) * TK;
    return first_lane(pages[key / a.page]);
  };
  struct {
    u32x4 k[NL], v[NL];
  } tl;
  auto base_of = [&](int i, int slot, uint32_t& bytes) {
    const int key = (t0 + wave + 4 * i) * TK;
    bytes = i < my_tiles && slot >= 0 && slot < a.n_slots ? uint32_t(kTile) : 0u;
    return bytes ? slot * slot_elems + head * head_elems + int64_t(key % a.page) * DH : int64_t(0);
  };
  auto load = [&](u32x4 (&d)[NL], const uint16_t* store, int64_t at, uint32_t bytes) {
    const uint64_t p = reinterpret_cast<uint64_t>(store + at);
    const uint64_t u = (uint64_t(uint32_t(first_lane(int(p >> 32)))) << 32) | uint32_t(first_lane(int(p)));
    const __amdgpu_buffer_rsrc_t res = make_rsrc(reinterpret_cast<const void*>(u), bytes);
#pragma unroll
    for (int l = 0; l < NL; ++l)
      d[l] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(res, uint32_t(lane * 16 + l * 1024), 0, 0));
    __builtin_amdgcn_sched_barrier(0);
  };

  u32x4 qf[NQ][NKB];  // B operand of S^T = K Q^T
#pragma unroll
  for (int j = 0; j < NQ; ++j) {
    const int m = m0 + min(16 * j + fr, n_cols - 1);  // lanes past the last column repeat it
    const uint16_t* qp = static_cast<const uint16_t*>(a.q) + int64_t(lo + m / G) * a.ldq + (head * G + m % G) * DH;
#pragma unroll
    for (int kb = 0; kb < NKB; ++kb) {
      // bf16 values convert exactly but for magnitudes below 2^-14 or beyond fp16.
      uint16_t raw[8];
      __builtin_memcpy(raw, qp + kb * 32 + fh * 8, 16);
      qf[j][kb] = __builtin_bit_cast(u32x4, raw);
      if constexpr (sizeof(T) == 2 && __is_same(T, uint16_t)) qf[j][kb] = bf8_to_h8(qf[j][kb]);
    }
  }

  // The LDS image of a tile: chunk c (16 bytes) of key row r at c ^ kphys(r), of value
  // row d at c ^ vphys(d), as in decode_unit.h.
  uint8_t* ks = sm.tile[wave];
  auto kphys = [](int r, int c) {
    const int i = ((r >> 3) << 2) | (r & 3);
    return c ^ (DH == 128 ? i : (i >> 1));
  };
  auto vphys = [](int d, int c) { return c ^ ((d >> 2) & 3); };
  constexpr int KCH = DH / 8;
  constexpr int kPer = NL / 4;
  uint32_t kw[4], kr[NKB];
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const int ch = q * kPer * 64 + lane, r = ch / KCH, c = ch % KCH;
    kw[q] = uint32_t(r * DH * 2 + kphys(r, c) * 16);
  }
#pragma unroll
  for (int kb = 0; kb < NKB; ++kb) {
    const int r = 8 * (fr >> 2) + (fr & 3);
    kr[kb] = uint32_t(r * DH * 2 + kphys(r, 4 * kb + fh) * 16);
  }
  const uint32_t vw = uint32_t((lane >> 2) * 64 + vphys(lane >> 2, lane & 3) * 16);
  const uint32_t vr = uint32_t(fr * 64 + vphys(fr, fh) * 16);

  float m_run[NQ], l_run[NQ];
  f32x4 o[NQ][NDS];
#pragma unroll
  for (int j = 0; j < NQ; ++j) {
    m_run[j] = -kInf;
    l_run[j] = 0.0f;
#pragma unroll
    for (int i = 0; i < NDS; ++i) o[j][i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  }

  if (my_tiles > 0) {
    int slot = slot_of(0), slot_next = slot_of(1);
    uint32_t bytes;
    int64_t at = base_of(0, slot, bytes);
    bad |= bytes == 0;
    load(tl.k, a.k, at, bytes);
    load(tl.v, a.v, at, bytes);
    for (int i = 0; i < my_tiles; ++i) {
      const int kv0 = (t0 + wave + 4 * i) * TK;
      at = base_of(i + 1, slot_next, bytes);
      bad |= i + 1 < my_tiles && bytes == 0;
      slot_next = slot_of(i + 2);
      asm volatile("" ::: "memory");
#pragma unroll
      for (int l = 0; l < NL; ++l) *reinterpret_cast<u32x4*>(ks + kw[l / kPer] + (l % kPer) * 1024) = tl.k[l];
      asm volatile("" ::: "memory");
      load(tl.k, a.k, at, bytes);
      f32x4 sc[NQ][2];
#pragma unroll
      for (int j = 0; j < NQ; ++j)
#pragma unroll
        for (int st = 0; st < 2; ++st) sc[j][st] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int st = 0; st < 2; ++st)
#pragma unroll
        for (int kb = 0; kb < NKB; ++kb) {
          const u32x4 kf = *reinterpret_cast<const u32x4*>(ks + kr[kb] + st * 4 * DH * 2);
#pragma unroll
          for (int j = 0; j < NQ; ++j) sc[j][st] = mfma16(kf, qf[j][kb], sc[j][st]);
        }
      // Score row i of subtile st is key 8 (i / 4) + 4 st + i % 4: the lane holds keys
      // 8 fh .. 8 fh + 7.
      const bool edge = kv0 < k_lo || kv0 + TK > k_hi;
      const int first = k_lo - kv0 - 8 * fh, last = k_hi - kv0 - 8 * fh;
      u32x4 pf[NQ];
#pragma unroll
      for (int j = 0; j < NQ; ++j) {
        if (edge) {
#pragma unroll
          for (int st = 0; st < 2; ++st)
#pragma unroll
            for (int r = 0; r < 4; ++r)
              if (4 * st + r < first || 4 * st + r >= last) sc[j][st][r] = -kInf;
        }
        // Every tile holds a key of the range, so the new maximum is finite.
        float mx = fmaxf(sc[j][0][0], sc[j][1][0]);
#pragma unroll
        for (int r = 1; r < 4; ++r) mx = fmaxf(mx, fmaxf(sc[j][0][r], sc[j][1][r]));
        const float m_new = fmaxf(m_run[j], quarter_max(mx) * a.scale_log2);
        const float alpha = exp2_raw(m_run[j] - m_new);
        float psum = 0.0f;
#pragma unroll
        for (int st = 0; st < 2; ++st)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const float p = exp2_raw(fmaf(sc[j][st][r], a.scale_log2, -m_new));
            sc[j][st][r] = p;
            psum += p;
          }
        l_run[j] = l_run[j] * alpha + psum;
        m_run[j] = m_new;
#pragma unroll
        for (int d = 0; d < NDS; ++d)
#pragma unroll
          for (int r = 0; r < 4; ++r) o[j][d][r] *= alpha;
        // The weights, at most 1, become fp16 operands as all contractions do; their
        // sum stays that of the unrounded ones.
#pragma unroll
        for (int e = 0; e < 4; ++e)
          pf[j][e] = pack2h_rne(sc[j][e >> 1][2 * (e & 1)], sc[j][e >> 1][2 * (e & 1) + 1]);
      }
      __builtin_amdgcn_sched_barrier(0);
      asm volatile("" ::: "memory");
      if (edge) {
        // Values outside the range may be anything; 0 * NaN must not reach the sum.
        const int vfirst = k_lo - kv0 - 8 * (lane & 3), vlast = k_hi - kv0 - 8 * (lane & 3);
        u32x4 keep;
#pragma unroll
        for (int e = 0; e < 4; ++e)
          keep[e] = ((2 * e >= vfirst && 2 * e < vlast) ? 0x0000ffffu : 0u) |
                    ((2 * e + 1 >= vfirst && 2 * e + 1 < vlast) ? 0xffff0000u : 0u);
#pragma unroll
        for (int l = 0; l < NL; ++l) *reinterpret_cast<u32x4*>(ks + vw + l * 1024) = tl.v[l] & keep;
      } else {
#pragma unroll
        for (int l = 0; l < NL; ++l) *reinterpret_cast<u32x4*>(ks + vw + l * 1024) = tl.v[l];
      }
      asm volatile("" ::: "memory");
      load(tl.v, a.v, at, bytes);
#pragma unroll
      for (int d = 0; d < NDS; ++d) {
        const u32x4 vf = *reinterpret_cast<const u32x4*>(ks + vr + d * 1024);
#pragma unroll
        for (int j = 0; j < NQ; ++j) o[j][d] = mfma16(vf, pf[j], o[j][d]);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
  }

  // The wavefronts' states become one.
#pragma unroll
  for (int j = 0; j < NQ; ++j) {
    const float l_tot = quarter_sum(l_run[j]);
    if (fh == 0) {
      sm.red_m[wave][16 * j + fr] = m_run[j];
      sm.red_l[wave][16 * j + fr] = bad ? __builtin_nanf("") : l_tot;
    }
  }
  float* stats = part_stats(a, splits);
  constexpr int kPass = Smem<DH, NQ>::kPass;
  static_assert(kPass == 64, "the index arithmetic below");
#pragma unroll
  for (int pass = 0; pass < DH / kPass; ++pass) {
    __syncthreads();  // the states take the tiles' place, and the last pass's
#pragma unroll
    for (int j = 0; j < NQ; ++j)
#pragma unroll
      for (int d = 0; d < kPass / 16; ++d)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          sm.red_o[wave][16 * d + 4 * fh + r][16 * j + fr] = o[j][pass * (kPass / 16) + d][r];
    __syncthreads();
    for (int idx = tid; idx < n_cols * kPass; idx += kThreads) {
      const int q = idx / kPass, d = idx % kPass;
      const int m = m0 + q;
      float M = -kInf;
#pragma unroll
      for (int w = 0; w < 4; ++w) M = fmaxf(M, sm.red_m[w][q]);
      float num = 0.0f, den = 0.0f;
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const float sc = exp2_raw(sm.red_m[w][q] - M);
        num += sc * sm.red_o[w][d][q];
        den += sc * sm.red_l[w][q];
      }
      const int64_t p = part_index(a, split, lo + m / G, head * G + m % G);
      static_cast<float*>(a.part)[p * DH + pass * kPass + d] = num;
      if (pass == 0 && d == 0) {
        stats[2 * p] = M;
        stats[2 * p + 1] = den;
      }
    }
  }
}

// Blocks of the prefixes (key/value head, row tile, split), then those of what rows
// have to themselves (key/value head, row, split).
template <int DH, int NQ, typename T>
__global__ __launch_bounds__(kThreads, 2) void prefix_kernel(PrefixArgs a, PrefixShape s) {
  __shared__ __attribute__((aligned(16))) Smem<DH, NQ> sm;
  const int G = a.hq / a.hkv, splits = s.prefix_splits + s.rest_splits;
  const int64_t reach = int64_t(a.pages_per_seq) * a.page;  // positions that the table covers
  uint32_t id = blockIdx.x;
  const uint32_t prefix_blocks = uint32_t(s.prefix_tiles) * s.prefix_splits * a.hkv;
  const int head = id % a.hkv;
  if (id < prefix_blocks) {
    id /= a.hkv;
    const int split = id % s.prefix_splits, tile = id / s.prefix_splits;
    const Group g = group_of_tile(a, tile, 16 * NQ, G);
    const int m0 = g.tile * 16 * NQ, n_cols = min((g.hi - g.lo) * G - m0, 16 * NQ);
    const int prefix = int(min(int64_t(clamped(g.prefix, 0, a.max_prefix)), reach));
    const int k_lo = split * s.prefix_keys, k_hi = min(prefix, k_lo + s.prefix_keys);
    if (n_cols < 1 || k_hi <= k_lo) return;
    unit<DH, NQ, T>(a, g.lo, m0, n_cols, head, g.lo, k_lo, k_hi, split, splits, sm);
  } else {
    id = (id - prefix_blocks) / a.hkv;
    const int split = id % s.rest_splits, row = id / s.rest_splits;
    const int prefix = clamped(prefix_of_row(a, row), 0, a.max_prefix);
    const int64_t end = min(int64_t(a.lens[row]), min(int64_t(prefix) + a.max_rest, reach));
    const int64_t k_lo = int64_t(prefix) + int64_t(split) * s.rest_keys;
    const int64_t k_hi = min(end, k_lo + s.rest_keys);
    if (k_hi <= k_lo) return;
    for (int m0 = 0; m0 < G; m0 += 16 * NQ) {
      if (m0 > 0) __syncthreads();  // the last unit's states have been read
      unit<DH, NQ, T>(a, row, m0, min(G - m0, 16 * NQ), head, row, int(k_lo), int(k_hi), s.prefix_splits + split,
                      splits, sm);
    }
  }
}

// One wavefront a (row, query head).
template <int DH, typename T>
__global__ __launch_bounds__(kThreads) void prefix_join_kernel(PrefixArgs a, PrefixShape s) {
  const int lane = threadIdx.x & 63;
  const int64_t index = int64_t(blockIdx.x) * 4 + first_lane(threadIdx.x >> 6);
  if (index >= int64_t(a.n_seqs) * a.hq) return;
  const int row = int(index / a.hq), head = int(index % a.hq);
  const int prefix = prefix_of_row(a, row), len = a.lens[row];
  const int64_t reach = int64_t(a.pages_per_seq) * a.page;
  const bool wrong = prefix < 0 || prefix > a.max_prefix || len < prefix || len - prefix > a.max_rest || len > reach;
  const int splits = s.prefix_splits + s.rest_splits;
  const float* stats = part_stats(a, splits);
  const float* part = static_cast<const float*>(a.part);
  const int n_prefix = wrong ? 0 : (prefix + s.prefix_keys - 1) / s.prefix_keys;
  const int n_rest = wrong ? 0 : (len - prefix + s.rest_keys - 1) / s.rest_keys;
  constexpr int V = DH / 64;
  float M = -kInf, L = 0.0f, acc[V] = {};
  for (int i0 = 0; i0 < n_prefix + n_rest; i0 += 64) {
    // The row's partial state number i0 + lane.
    const int i = i0 + lane, n = min(n_prefix + n_rest - i0, 64);
    const int split = i < n_prefix ? i : s.prefix_splits + i - n_prefix;
    float m = -kInf, l = 0.0f;
    if (lane < n) {
      const int64_t p = part_index(a, split, row, head);
      m = stats[2 * p];
      l = stats[2 * p + 1];
    }
    const float top = fmaxf(M, reduce_wave(m, [](float x, float y) { return fmaxf(x, y); }));
    const float w = lane < n ? exp2_raw(m - top) : 0.0f, old = exp2_raw(M - top);
    L = L * old + reduce_wave(w * l, [](float x, float y) { return x + y; });
#pragma unroll
    for (int e = 0; e < V; ++e) acc[e] *= old;
    for (int k = 0; k < n; ++k) {
      const int sk = i0 + k < n_prefix ? i0 + k : s.prefix_splits + i0 + k - n_prefix;
      const float wk = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(w), k));
      const float* src = part + part_index(a, sk, row, head) * DH;
#pragma unroll
      for (int e = 0; e < V; ++e) acc[e] = fmaf(wk, src[e * 64 + lane], acc[e]);
    }
    M = top;
  }
  const bool none = n_prefix + n_rest == 0;
#pragma unroll
  for (int e = 0; e < V; ++e) {
    const float y = wrong ? __builtin_nanf("") : none ? 0.0f : acc[e] / L;
    const int d = head * DH + e * 64 + lane;
    if (a.out_k8_rows) {
      static_cast<uint16_t*>(a.out)[act_index(row, d, 0, a.out_k8_rows)] = f2h(y);
    } else if constexpr (__is_same(T, uint16_t)) {
      // bf16, to nearest even; NaN stays NaN.
      const uint32_t b = __float_as_uint(y);
      static_cast<uint16_t*>(a.out)[row * a.ldo + d] =
          y != y ? uint16_t(0x7fc0) : uint16_t((b + 0x7fffu + ((b >> 16) & 1)) >> 16);
    } else {
      static_cast<_Float16*>(a.out)[row * a.ldo + d] = _Float16(y);
    }
  }
}

template <int DH, typename T>
hipError_t launch(const PrefixArgs& a, int cus, hipStream_t st) {
  const PrefixShape s = prefix_shape(a.n_seqs, a.n_groups, a.max_prefix, a.max_rest, a.hq, a.hkv, cus);
  const int64_t blocks = prefix_blocks(s, a.n_seqs, a.hkv);
  if (blocks > 0) {
    if (s.prefix_rows == 16)
      hipLaunchKernelGGL((prefix_kernel<DH, 1, T>), dim3(uint32_t(blocks)), dim3(kThreads), 0, st, a, s);
    else
      hipLaunchKernelGGL((prefix_kernel<DH, 2, T>), dim3(uint32_t(blocks)), dim3(kThreads), 0, st, a, s);
  }
  const int64_t rows = int64_t(a.n_seqs) * a.hq;
  hipLaunchKernelGGL((prefix_join_kernel<DH, T>), dim3(uint32_t((rows + 3) / 4)), dim3(kThreads), 0, st, a, s);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_prefix_attention(const PrefixArgs& a, int cus, hipStream_t s) {
  if (a.n_seqs < 1) return hipSuccess;
  if (a.dh == 64) return a.type == HS_TYPE_BF16 ? launch<64, uint16_t>(a, cus, s) : launch<64, _Float16>(a, cus, s);
  return a.type == HS_TYPE_BF16 ? launch<128, uint16_t>(a, cus, s) : launch<128, _Float16>(a, cus, s);
}

}  // namespace hs
