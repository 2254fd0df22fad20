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
// Where a group has more columns than such a unit, the tile is that of prefill attention
// (attention_tile.h): 128 columns, 32 a wavefront, which share 64-key tiles in LDS.
//
// Memory bounds short groups and what rows have to themselves (45 rows of up to 2000 keys
// in 32 / 8 heads of 128: 31 us, 6.0 TB/s, and 4.8 for the join), the alternation of products
// and exponentials in a wavefront long prefixes (128 rows in the same heads: 57 us behind
// 16384 positions and 40 for each further 16384, 0.85 P/s; behind 16384, with up to 512 keys
// more, 73 us and 7), the chain of loads small calls (8 rows behind 8192 positions in 28 / 4
// heads: 10.3 and 4.5; behind 256, 9.6).  Times are a trace's, on one state.
//
// The kernel with wide tiles for heads of 128 takes all 256 registers, with one vector and
// 11 scalar ones spilled: the unit for what rows have to themselves is in it too.
//
// What the device arrays say is checked here: a slot outside the cache is read as
// zeros and makes its rows NaN, and no range leaves the table.
#include "answer_device.h"
#include "attention_tile.h"
#include "decode_policy.h"
#include "decoding_kernels.h"

namespace hs {
namespace {

constexpr int kThreads = 256;
constexpr int kTileKeys = kv_tile_keys;
constexpr float kInf = __builtin_inff();

__device__ __forceinline__ int clamped(int v, int lo, int hi) { return min(max(v, lo), hi); }
__device__ __forceinline__ int first_lane(int v) { return __builtin_amdgcn_readfirstlane(v); }

// m / per_head, by the product with its rounded-up inverse.
__device__ __forceinline__ int row_of(const PrefixArgs& a, int m) {
  return int(__umulhi(2u * uint32_t(m), a.per_head_inv));
}

struct Group {
  int lo, hi;   // its rows
  int prefix;   // its shared positions
  int tile;     // of the group's row tiles
};

// The group that holds row tile `t` (of COLS columns, per_head of them a row); lo == hi
// where there is none.  The tiles of group g have the numbers from
// offsets[g] per_head / COLS + g on, which leaves each group enough of them and needs
// no sum over the groups before.  A wavefront looks at 64 groups at a time.
template <int COLS>
__device__ __forceinline__ Group group_of_tile(const PrefixArgs& a, int t) {
  const int lane = threadIdx.x & 63, per_head = a.hq / a.hkv;
  Group f{0, 0, 0, 0};
  for (int g0 = 0; g0 < a.n_groups; g0 += 64) {
    const int g = min(g0 + lane, a.n_groups - 1);
    const int lo = clamped(a.offsets[g], 0, a.n_seqs), hi = clamped(a.offsets[g + 1], lo, a.n_seqs);
    const int prefix = a.prefix[g];
    const int start = int(uint32_t(lo) * uint32_t(per_head) / COLS) + g;
    const uint64_t mask = __ballot(g0 + lane < a.n_groups && start <= t);
    if (mask == 0) break;
    const int w = 63 - __builtin_clzll(mask);
    f.lo = __builtin_amdgcn_readlane(lo, w);
    f.hi = __builtin_amdgcn_readlane(hi, w);
    f.prefix = __builtin_amdgcn_readlane(prefix, w);
    f.tile = t - __builtin_amdgcn_readlane(start, w);
    if (w < 63) break;
  }
  return f;
}

// The prefix of a row's group (0 where no group holds the row).
__device__ __forceinline__ int prefix_of_row(const PrefixArgs& a, int row) {
  const int lane = threadIdx.x & 63;
  for (int g0 = 0; g0 < a.n_groups; g0 += 64) {
    const int g = min(g0 + lane, a.n_groups - 1);
    const int lo = a.offsets[g], hi = a.offsets[g + 1], prefix = a.prefix[g];
    const uint64_t mask = __ballot(g0 + lane < a.n_groups && lo <= row && row < hi);
    if (mask != 0) return __builtin_amdgcn_readlane(prefix, __builtin_ctzll(mask));
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
  static constexpr int kPass = NQ == 1 ? DH : 64;   // dimensions of a pass of the join of wavefronts
  union {
    uint8_t tile[4][kTile];
    float red_o[4][kCols][kPass + 4];  // 16 columns apart in banks
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

// A 32-key tile for one wavefront.
struct Tile {
  int slot, at;       // where its keys lie: slot (any value), position in it
  int first, last;    // keys [first, last) of the tile count
  int c_lo, c_hi;     // for these columns of the unit
  bool there;
};

// The wavefront's tiles of the keys [k_lo, k_hi) of one sequence: every fourth one.  Entries
// of the table are read a tile ahead, and none that no key needs.
struct Range {
  static constexpr bool kSomeColumns = false;
  const int32_t* pages;
  int page, kv0, k_lo, k_hi, left, no, at, slot;

  __device__ __forceinline__ Range(const PrefixArgs& a, int owner, int lo, int hi, int wave) {
    pages = a.table + int64_t(owner) * a.pages_per_seq;
    page = a.page;
    k_lo = lo;
    k_hi = hi;
    const int t0 = lo / kTileKeys, n = (hi + kTileKeys - 1) / kTileKeys - t0;
    left = n > wave ? (n - wave + 3) / 4 : 0;
    kv0 = (t0 + wave) * kTileKeys;
    no = left > 0 ? first_lane(kv0 / page) : 0;
    at = kv0 - no * page;
    slot = left > 0 ? pages[no] : -1;
  }
  __device__ __forceinline__ Tile next() {
    const Tile t{slot, at, k_lo - kv0, k_hi - kv0, 0, 0, left > 0};
    --left;
    kv0 += 4 * kTileKeys;
    at += 4 * kTileKeys;
    while (at >= page) {
      at -= page;
      ++no;
    }
    slot = left > 0 ? pages[no] : -1;
    return t;
  }
};

// The wavefront's tiles of everything that a unit's columns look at: the prefix of
// their group, for all of them, and what each of their rows (at most 16) has to
// itself, for the row's columns.
struct Everything {
  static constexpr bool kSomeColumns = true;
  const PrefixArgs& a;
  int lo, m0, n_cols, prefix, rows, row0;  // row0: the columns' first row, behind lo
  int owner, pos, segment, tiles;          // segment 0: the prefix, then the rows
  int end;                                 // lane r: where row r's keys end
  int start, stop;                         // keys of the segment
  Tile ahead;

  __device__ __forceinline__ Everything(const PrefixArgs& args, int lo_, int m0_, int n, int prefix_, int reach, int wave)
      : a(args), lo(lo_), m0(m0_), n_cols(n), prefix(min(prefix_, reach)) {
    row0 = row_of(a, m0);
    rows = row_of(a, m0 + n_cols - 1) - row0 + 1;
    const int lane = threadIdx.x & 63;
    const int len = a.lens[lo + row0 + min(lane, rows - 1)];
    end = int(min(int64_t(len), min(int64_t(prefix_) + a.max_rest, int64_t(reach))));
    segment = 0;
    start = 0;
    stop = prefix;
    tiles = (stop + kTileKeys - 1) / kTileKeys;
    pos = wave;
    look();
  }
  // Finds the tile at `pos` and asks for its entry of the table.
  __device__ __forceinline__ void look() {
    while (pos >= tiles && segment <= rows) {
      pos -= tiles;
      if (++segment > rows) break;
      start = prefix;
      stop = __builtin_amdgcn_readlane(end, segment - 1);
      tiles = stop > start ? (stop + kTileKeys - 1) / kTileKeys - start / kTileKeys : 0;
    }
    ahead = Tile{-1, 0, 0, 0, 0, 0, segment <= rows};
    if (!ahead.there) return;
    const int per_head = a.hq / a.hkv, row = lo + (segment ? row0 + segment - 1 : 0);
    const int kv0 = (start / kTileKeys + pos) * kTileKeys, no = first_lane(kv0 / a.page);
    ahead.at = kv0 - no * a.page;
    ahead.slot = a.table[int64_t(row) * a.pages_per_seq + no];
    ahead.first = start - kv0;
    ahead.last = stop - kv0;
    ahead.c_lo = segment ? (row0 + segment - 1) * per_head - m0 : 0;
    ahead.c_hi = segment ? ahead.c_lo + per_head : n_cols;
  }
  __device__ __forceinline__ Tile next() {
    const Tile t = ahead;
    pos += 4;
    look();
    return t;
  }
};

// Columns m0 .. m0 + n_cols - 1 of rows lo .. (column m: row lo + m / G, query head
// head * G + m % G) over the tiles of `steps`.  emit(q, d, sums, maximum, sum): column m0 + q's
// unnormalised outputs d .. d + 3.
template <int DH, int NQ, typename T, typename Steps, typename Emit>
__device__ __forceinline__ void unit(const PrefixArgs& a, int lo, int m0, int n_cols, int head, Steps steps,
                                     Smem<DH, NQ>& sm, Emit emit) {
  constexpr int NKB = DH / 32, NDS = DH / 16;
  constexpr int kTile = Smem<DH, NQ>::kTile, NL = kTile / 1024;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = first_lane(tid >> 6);
  const int fr = lane & 15, fh = lane >> 4;
  const int G = a.hq / a.hkv;
  const int64_t head_elems = int64_t(a.page) * DH, slot_elems = head_elems * a.hkv;
  bool bad = false;  // of the lane's columns
  struct {
    u32x4 k[NL], v[NL];
  } tl;
  // Tiles past the last one, and slots outside the cache, are read through an empty
  // resource: zeros, no traffic.
  auto base_of = [&](const Tile& t, uint32_t& bytes) {
    const int slot = first_lane(t.slot);
    bytes = t.there && slot >= 0 && slot < a.n_slots ? uint32_t(kTile) : 0u;
    return bytes ? slot * slot_elems + head * head_elems + int64_t(t.at) * DH : int64_t(0);
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
    const int i = row_of(a, m);
    const uint16_t* qp = static_cast<const uint16_t*>(a.q) + int64_t(lo + i) * a.ldq + (head * G + m - i * G) * DH;
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

  Tile tile = steps.next();
  if (tile.there) {
    uint32_t bytes;
    int64_t at = base_of(tile, bytes);
    bool lost = bytes == 0;
    load(tl.k, a.k, at, bytes);
    load(tl.v, a.v, at, bytes);
    while (tile.there) {
      const Tile next = steps.next();
      at = base_of(next, bytes);
      const bool mine = !Steps::kSomeColumns || (fr >= tile.c_lo && fr < tile.c_hi);
      bad |= lost && mine;
      lost = bytes == 0;
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
      const bool edge = tile.first > 0 || tile.last < kTileKeys;
      const int first = tile.first - 8 * fh, last = tile.last - 8 * fh;
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
        if constexpr (Steps::kSomeColumns) {
#pragma unroll
          for (int st = 0; st < 2; ++st)
#pragma unroll
            for (int r = 0; r < 4; ++r) sc[j][st][r] = mine ? sc[j][st][r] : -kInf;
        }
        float mx = fmaxf(sc[j][0][0], sc[j][1][0]);
#pragma unroll
        for (int r = 1; r < 4; ++r) mx = fmaxf(mx, fmaxf(sc[j][0][r], sc[j][1][r]));
        const float m_new = fmaxf(m_run[j], quarter_max(mx) * a.scale_log2);
        const float use = against(m_new);
        const float alpha = exp2_raw(m_run[j] - use);
        float psum = 0.0f;
#pragma unroll
        for (int st = 0; st < 2; ++st)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const float p = exp2_raw(fmaf(sc[j][st][r], a.scale_log2, -use));
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
        const int vfirst = tile.first - 8 * (lane & 3), vlast = tile.last - 8 * (lane & 3);
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
        for (int j = 0; j < NQ; ++j) {
          const f32x4 y = mfma16(vf, pf[j], o[j][d]);
          // Another row's values may be NaN, which 0 does not take out.
#pragma unroll
          for (int r = 0; r < 4; ++r) o[j][d][r] = mine ? y[r] : o[j][d][r];
        }
      }
      __builtin_amdgcn_sched_barrier(0);
      tile = next;
    }
  }

  // The wavefronts' states become one; a lane adds up four dimensions of a column.
#pragma unroll
  for (int j = 0; j < NQ; ++j) {
    const float l_tot = quarter_sum(l_run[j]);
    if (fh == 0) {
      sm.red_m[wave][16 * j + fr] = m_run[j];
      sm.red_l[wave][16 * j + fr] = bad ? __builtin_nanf("") : l_tot;
    }
  }
  constexpr int kPass = Smem<DH, NQ>::kPass;
  constexpr int kLanes = kPass / 4, kStep = 256 / kLanes;  // of a column; columns at a time
#pragma unroll
  for (int pass = 0; pass < DH / kPass; ++pass) {
    __syncthreads();  // the states take the tiles' place, and the last pass's
#pragma unroll
    for (int j = 0; j < NQ; ++j)
#pragma unroll
      for (int d = 0; d < kPass / 16; ++d)
        *reinterpret_cast<f32x4*>(&sm.red_o[wave][16 * j + fr][16 * d + 4 * fh]) = o[j][pass * (kPass / 16) + d];
    __syncthreads();
#pragma unroll
    for (int q0 = 0; q0 < 16 * NQ; q0 += kStep) {
      const int q = q0 + tid / kLanes, d = tid % kLanes * 4;
      if (q >= n_cols) break;
      float m[4], M = -kInf;
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        m[w] = sm.red_m[w][q];
        M = fmaxf(M, m[w]);
      }
      const float use = against(M);
      f32x4 num = {0.0f, 0.0f, 0.0f, 0.0f};
      float den = 0.0f;
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const float f = exp2_raw(m[w] - use);
        const f32x4 v = *reinterpret_cast<const f32x4*>(&sm.red_o[w][q][d]);
        den = fmaf(f, sm.red_l[w][q], den);
#pragma unroll
        for (int e = 0; e < 4; ++e) num[e] = fmaf(f, v[e], num[e]);
      }
      emit(q, pass * kPass + d, num, M, den);
    }
  }
}

// The unit over a range of one sequence's keys, as partial state `split`.
template <int DH, int NQ, typename T>
__device__ __forceinline__ void range_unit(const PrefixArgs& a, int lo, int m0, int n_cols, int head, int owner, int k_lo,
                                           int k_hi, int split, int splits, Smem<DH, NQ>& sm) {
  float* stats = part_stats(a, splits);
  const int G = a.hq / a.hkv;
  unit<DH, NQ, T>(a, lo, m0, n_cols, head, Range(a, owner, k_lo, k_hi, first_lane(threadIdx.x >> 6)), sm,
                  [&](int q, int d, const f32x4& num, float m, float sum) {
                    const int i = row_of(a, m0 + q);
                    const int64_t p = part_index(a, split, lo + i, head * G + m0 + q - i * G);
                    *reinterpret_cast<f32x4*>(static_cast<float*>(a.part) + p * DH + d) = num;
                    if (d == 0) *reinterpret_cast<float2*>(stats + 2 * p) = make_float2(m, sum);
                  });
}

template <bool C, typename A, typename B>
struct Choose {
  using type = A;
};
template <typename A, typename B>
struct Choose<false, A, B> {
  using type = B;
};

// The same for up to 128 columns: wavefront w takes columns 32 w .. 32 w + 31 over all
// keys, whose tiles of 64 pass through LDS for all of them.  k_lo is a tile's start.
template <int DH>
struct WideSmem {
  static constexpr int kTile = BKV * DH * 2;
  static constexpr int kRow = 64 + 4;  // a state's 64 dimensions; 16 columns apart in banks
  union {
    uint8_t tile[2][2][kTile];         // [stage][keys, values]
    float out[4][32][kRow];
  };
};

template <int DH, typename T>
__device__ __forceinline__ void wide_unit(const PrefixArgs& a, int lo, int m0, int n_cols, int head, int owner,
                                          int k_lo, int k_hi, int split, int splits, WideSmem<DH>& sm) {
  constexpr int KROW = DH * 2, KCH = DH / 8;
  constexpr int LOADS = BKV * KCH / kThreads;  // of a thread, keys and values alike
  constexpr int NDS = DH / 32;
  const int tid = threadIdx.x, lane = tid & 63, wave = first_lane(tid >> 6);
  const int fr = lane & 31, fh = lane >> 5;
  const int G = a.hq / a.hkv;
  const int64_t head_elems = int64_t(a.page) * DH, slot_elems = head_elems * a.hkv;
  const int n_tiles = (k_hi - k_lo + BKV - 1) / BKV;
  const int32_t* pages = a.table + int64_t(owner) * a.pages_per_seq;
  bool bad = false;

  u32x4 qf[DH / 16];
  {
    const int m = m0 + min(wave * 32 + fr, n_cols - 1);  // lanes past the last column repeat it
    const int i = row_of(a, m);
    const uint16_t* qp = static_cast<const uint16_t*>(a.q) + int64_t(lo + i) * a.ldq + (head * G + m - i * G) * DH;
#pragma unroll
    for (int kb = 0; kb < DH / 16; ++kb) {
      qf[kb] = *reinterpret_cast<const u32x4*>(qp + kb * 16 + fh * 8);
      if constexpr (__is_same(T, uint16_t)) qf[kb] = bf8_to_h8(qf[kb]);
    }
  }

  uint32_t koff[LOADS], voff[LOADS];
#pragma unroll
  for (int j = 0; j < LOADS; ++j) {
    const int idx = tid + j * kThreads, d = idx >> 3, c = idx & 7;
    koff[j] = uint32_t(idx * 16);
    voff[j] = uint32_t(((c >> 2) * kv_tile_keys * DH + d * kv_tile_keys + (c & 3) * 8) * 2);
  }
  u32x4 rk[LOADS], rv[LOADS];
  // The page of the next tile to load, and the tile's place in it.
  int page_no = first_lane(k_lo / a.page), page_at = k_lo - page_no * a.page;
  auto gload = [&](int slot) {
    const bool ok = slot >= 0 && slot < a.n_slots;
    bad |= !ok;
    const int64_t at = ok ? slot * slot_elems + head * head_elems + int64_t(page_at) * DH : int64_t(0);
    const uint32_t bytes = ok ? uint32_t(WideSmem<DH>::kTile) : 0u;
    auto res = [&](const uint16_t* store) {
      const uint64_t p = reinterpret_cast<uint64_t>(store + at);
      const uint64_t u = (uint64_t(uint32_t(first_lane(int(p >> 32)))) << 32) | uint32_t(first_lane(int(p)));
      return make_rsrc(reinterpret_cast<const void*>(u), bytes);
    };
    const __amdgpu_buffer_rsrc_t kres = res(a.k), vres = res(a.v);
#pragma unroll
    for (int j = 0; j < LOADS; ++j) rk[j] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(kres, koff[j], 0, 0));
#pragma unroll
    for (int j = 0; j < LOADS; ++j) rv[j] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(vres, voff[j], 0, 0));
    page_at += BKV;  // pages are whole tiles
    if (page_at == a.page) {
      page_at = 0;
      ++page_no;
    }
  };
  // Values past the range may be anything; 0 * NaN must not reach the sum.
  auto vmask = [&](int t) {
    if (k_lo + (t + 1) * BKV <= k_hi) return;
#pragma unroll
    for (int j = 0; j < LOADS; ++j) {
      const int left = k_hi - (k_lo + t * BKV + ((tid + j * kThreads) & 7) * 8);
#pragma unroll
      for (int e = 0; e < 4; ++e)
        rv[j][e] &= (2 * e < left ? 0x0000ffffu : 0u) | (2 * e + 1 < left ? 0xffff0000u : 0u);
    }
  };
  auto lstore = [&](int stage) {
    uint8_t* ks = sm.tile[stage][0];
    uint8_t* vs = sm.tile[stage][1];
#pragma unroll
    for (int j = 0; j < LOADS; ++j) {
      const int idx = tid + j * kThreads, row = idx / KCH, c = idx % KCH;
      *reinterpret_cast<u32x4*>(ks + row * KROW + kphys<DH>(row, c) * 16) = rk[j];
    }
#pragma unroll
    for (int j = 0; j < LOADS; ++j) {
      const int idx = tid + j * kThreads, d = idx >> 3, c = idx & 7;
      *reinterpret_cast<u32x4*>(vs + d * 128 + vphys(d, c) * 16) = rv[j];
    }
  };

  f32x16 o[NDS];
#pragma unroll
  for (int i = 0; i < NDS; ++i)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[i][r] = 0.0f;
  float m_run = -kInf, l_run = 0.0f;

  gload(pages[page_no]);
  int slot = n_tiles > 1 ? pages[page_no] : 0;  // a tile ahead; past the last one there may be no entry
  vmask(0);
  lstore(0);
  __syncthreads();
  const bool busy = wave * 32 < n_cols;
  for (int t = 0; t < n_tiles; ++t) {
    if (t + 1 < n_tiles) gload(slot);
    if (t + 2 < n_tiles) slot = pages[page_no];
    if (busy) {
      const uint8_t* ks = sm.tile[t & 1][0];
      const uint8_t* vs = sm.tile[t & 1][1];
      f32x16 sc[2];
#pragma unroll
      for (int st = 0; st < 2; ++st)
#pragma unroll
        for (int r = 0; r < 16; ++r) sc[st][r] = 0.0f;
      // Fragments are read a step ahead of the products that use them.
      auto kfrag = [&](int kb, int st) {
        const int row = 32 * st + perm32(fr);
        return *reinterpret_cast<const u32x4*>(ks + row * KROW + kphys<DH>(row, 2 * kb + fh) * 16);
      };
      u32x4 kf[2][2];
      kf[0][0] = kfrag(0, 0);
      kf[0][1] = kfrag(0, 1);
      __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
#pragma unroll
      for (int kb = 0; kb < DH / 16; ++kb) {
        if (kb + 1 < DH / 16) {
          kf[(kb + 1) & 1][0] = kfrag(kb + 1, 0);
          kf[(kb + 1) & 1][1] = kfrag(kb + 1, 1);
        }
        sc[0] = mfma32(kf[kb & 1][0], qf[kb], sc[0]);
        sc[1] = mfma32(kf[kb & 1][1], qf[kb], sc[1]);
        if (kb + 1 < DH / 16) {
          __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
          __builtin_amdgcn_sched_group_barrier(0x008, 2, 0);
        }
      }
      __builtin_amdgcn_sched_barrier(0);
      u32x4 pf[4];
      const int last = k_hi - 1 - (k_lo + t * BKV);  // the tile's last key
      softmax_tile<NDS>(sc, o, pf, m_run, l_run, a.scale_log2, last < BKV - 1, last - 8 * fh);
      auto vfrag = [&](int kb2, int i) {
        const int d = 32 * i + fr;
        return *reinterpret_cast<const u32x4*>(vs + d * 128 + vphys(d, 2 * kb2 + fh) * 16);
      };
      u32x4 vf[2][NDS];
#pragma unroll
      for (int i = 0; i < NDS; ++i) vf[0][i] = vfrag(0, i);
      __builtin_amdgcn_sched_group_barrier(0x100, NDS, 0);
#pragma unroll
      for (int kb2 = 0; kb2 < 4; ++kb2) {
        if (kb2 + 1 < 4) {
#pragma unroll
          for (int i = 0; i < NDS; ++i) vf[(kb2 + 1) & 1][i] = vfrag(kb2 + 1, i);
        }
#pragma unroll
        for (int i = 0; i < NDS; ++i) o[i] = mfma32(vf[kb2 & 1][i], pf[kb2], o[i]);
        if (kb2 + 1 < 4) {
          __builtin_amdgcn_sched_group_barrier(0x100, NDS, 0);
          __builtin_amdgcn_sched_group_barrier(0x008, NDS, 0);
        }
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    if (t + 1 < n_tiles) {
      vmask(t + 1);
      lstore((t + 1) & 1);
    }
    __syncthreads();
  }
  if (!busy) return;

  // A wavefront's states leave through its part of LDS as rows.
  const float l_tot = l_run + xor_lane<32>(l_run);
  float* stats = part_stats(a, splits);
  if (fh == 0 && wave * 32 + fr < n_cols) {
    const int m = m0 + wave * 32 + fr, i = row_of(a, m);
    const int64_t p = part_index(a, split, lo + i, head * G + m - i * G);
    *reinterpret_cast<float2*>(stats + 2 * p) = make_float2(m_run, bad ? __builtin_nanf("") : l_tot);
  }
  float(*mine)[WideSmem<DH>::kRow] = sm.out[wave];
#pragma unroll
  for (int pass = 0; pass < DH / 64; ++pass) {
    asm volatile("" ::: "memory");
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const f32x16& v = o[2 * pass + i];
        *reinterpret_cast<f32x4*>(&mine[fr][32 * i + 8 * g + 4 * fh]) =
            f32x4{v[4 * g], v[4 * g + 1], v[4 * g + 2], v[4 * g + 3]};
      }
    asm volatile("" ::: "memory");
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int col = 4 * j + (lane >> 4), d = (lane & 15) * 4;
      if (wave * 32 + col >= n_cols) continue;
      const int m = m0 + wave * 32 + col, i = row_of(a, m);
      const int64_t p = part_index(a, split, lo + i, head * G + m - i * G);
      *reinterpret_cast<f32x4*>(static_cast<float*>(a.part) + p * DH + 64 * pass + d) =
          *reinterpret_cast<const f32x4*>(&mine[col][d]);
    }
  }
}

// Blocks of the prefixes (key/value head, row tile, split), then those of what rows
// have to themselves (key/value head, row, split).
// WIDE: the prefixes' tiles are wide ones.
template <int DH, int NQ, bool WIDE, typename T>
__global__ __launch_bounds__(kThreads, 2) void prefix_kernel(PrefixArgs a, PrefixShape s) {
  union Lds {
    Smem<DH, 1> rest;
    typename Choose<WIDE, WideSmem<DH>, Smem<DH, NQ>>::type prefix;
  };
  __shared__ __attribute__((aligned(16))) Lds sm;
  constexpr int kCols = WIDE ? 128 : 16 * NQ;
  const int G = a.hq / a.hkv, splits = s.prefix_splits + s.rest_splits;
  const int64_t reach = int64_t(a.pages_per_seq) * a.page;  // positions that the table covers
  uint32_t id = blockIdx.x;
  const uint32_t prefix_blocks = uint32_t(s.prefix_tiles) * s.prefix_splits * a.hkv;
  const int head = id % a.hkv;
  if (id < prefix_blocks) {
    id /= a.hkv;
    const int split = id % s.prefix_splits, tile = id / s.prefix_splits;
    const Group g = group_of_tile<kCols>(a, tile);
    const int m0 = g.tile * kCols, n_cols = min((g.hi - g.lo) * G - m0, kCols);
    const int prefix = int(min(int64_t(clamped(g.prefix, 0, a.max_prefix)), reach));
    const int k_lo = split * s.prefix_keys, k_hi = min(prefix, k_lo + s.prefix_keys);
    if (n_cols < 1 || k_hi <= k_lo) return;
    if constexpr (WIDE)
      wide_unit<DH, T>(a, g.lo, m0, n_cols, head, g.lo, k_lo, k_hi, split, splits, sm.prefix);
    else
      range_unit<DH, NQ, T>(a, g.lo, m0, n_cols, head, g.lo, k_lo, k_hi, split, splits, sm.prefix);
  } else {
    id = (id - prefix_blocks) / a.hkv;
    const int split = id % s.rest_splits, row = id / s.rest_splits;
    const int prefix = clamped(prefix_of_row(a, row), 0, a.max_prefix);
    const int64_t end = min(int64_t(a.lens[row]), min(int64_t(prefix) + a.max_rest, reach));
    const int64_t k_lo = int64_t(prefix) + int64_t(split) * s.rest_keys;
    const int64_t k_hi = min(end, k_lo + s.rest_keys);
    if (k_hi <= k_lo) return;
    for (int m0 = 0; m0 < G; m0 += 16) {
      if (m0 > 0) __syncthreads();  // the last unit's states have been read
      range_unit<DH, 1, T>(a, row, m0, min(G - m0, 16), head, row, int(k_lo), int(k_hi), s.prefix_splits + split,
                           splits, sm.rest);
    }
  }
}

// Output d of (row, query head): fp16 as the products take it, or the type of q.
template <int DH, typename T>
__device__ __forceinline__ void write_out(const PrefixArgs& a, int row, int head, int e, float y) {
  const int d = head * DH + e;
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

__device__ __forceinline__ bool wrong_lengths(const PrefixArgs& a, int prefix, int len) {
  return prefix < 0 || prefix > a.max_prefix || len < prefix || len - prefix > a.max_rest ||
         len > int64_t(a.pages_per_seq) * a.page;
}

// Short ranges in one launch: a block takes 16 columns of a group over everything that
// they look at and writes their outputs.
template <int DH, typename T>
__global__ __launch_bounds__(kThreads, 2) void prefix_short_kernel(PrefixArgs a) {
  __shared__ __attribute__((aligned(16))) Smem<DH, 1> sm;
  const int G = a.hq / a.hkv, head = blockIdx.x % uint32_t(a.hkv), tile = blockIdx.x / uint32_t(a.hkv);
  const Group g = a.n_groups ? group_of_tile<16>(a, tile) : Group{0, a.n_seqs, 0, tile};
  const int m0 = g.tile * 16, n_cols = min((g.hi - g.lo) * G - m0, 16);
  if (n_cols < 1) return;
  const int prefix = clamped(g.prefix, 0, a.max_prefix);
  const int reach = int(min(int64_t(a.pages_per_seq) * a.page, int64_t(1) << 30));
  unit<DH, 1, T>(a, g.lo, m0, n_cols, head, Everything(a, g.lo, m0, n_cols, prefix, reach, first_lane(threadIdx.x >> 6)),
                 sm, [&](int q, int d, const f32x4& num, float, float sum) {
                   const int i = row_of(a, m0 + q), row = g.lo + i, len = a.lens[row];
#pragma unroll
                   for (int e = 0; e < 4; ++e)
                     write_out<DH, T>(a, row, head * G + m0 + q - i * G, d + e,
                                      wrong_lengths(a, g.prefix, len) ? __builtin_nanf("") : len == 0 ? 0.0f : num[e] / sum);
                 });
}

// W wavefronts a (row, query head): each adds up every W-th of its partial states, all
// of a batch's loads in flight, and the first what they have.
constexpr int kJoinBatch = 8;

template <int DH, int W, typename T>
__global__ __launch_bounds__(kThreads) void prefix_join_kernel(PrefixArgs a, PrefixShape s) {
  constexpr int V = DH / 64;
  typedef float Vec __attribute__((ext_vector_type(V)));
  __shared__ float sums[4][DH + 2];
  const int lane = threadIdx.x & 63, wave = first_lane(threadIdx.x >> 6), member = wave % W;
  const int64_t index = int64_t(blockIdx.x) * (4 / W) + wave / W;
  const bool mine = index < int64_t(a.n_seqs) * a.hq;
  const int row = mine ? int(index / a.hq) : 0, head = int(index % a.hq);
  const int len = a.lens[row], prefix = prefix_of_row(a, row);
  const bool wrong = wrong_lengths(a, prefix, len);
  const int splits = s.prefix_splits + s.rest_splits;
  const float* stats = part_stats(a, splits);
  const float* part = static_cast<const float*>(a.part);
  const int n_prefix = wrong || !mine ? 0 : (prefix + s.prefix_keys - 1) / s.prefix_keys;
  const int n = wrong || !mine ? 0 : n_prefix + (len - prefix + s.rest_keys - 1) / s.rest_keys;
  float M = -kInf, L = 0.0f;
  Vec acc = 0.0f;
  for (int i0 = member; i0 < n; i0 += W * kJoinBatch) {
    float m[kJoinBatch], l[kJoinBatch];
    Vec v[kJoinBatch];
#pragma unroll
    for (int j = 0; j < kJoinBatch; ++j) {
      const int i = min(i0 + j * W, n - 1);
      const int64_t p = part_index(a, i < n_prefix ? i : s.prefix_splits + i - n_prefix, row, head);
      const float2 ml = *reinterpret_cast<const float2*>(stats + 2 * p);
      m[j] = ml.x;
      l[j] = ml.y;
      v[j] = *reinterpret_cast<const Vec*>(part + p * DH + lane * V);
    }
    float top = M;
#pragma unroll
    for (int j = 0; j < kJoinBatch; ++j) top = fmaxf(top, i0 + j * W < n ? m[j] : -kInf);
    const float use = against(top), old = exp2_raw(M - use);
    L *= old;
    acc *= old;
#pragma unroll
    for (int j = 0; j < kJoinBatch; ++j) {
      const float w = i0 + j * W < n ? exp2_raw(m[j] - use) : 0.0f;
      if (i0 + j * W < n) {
        L = fmaf(w, l[j], L);
        acc += w * v[j];
      }
    }
    M = top;
  }
  if constexpr (W > 1) {
#pragma unroll
    for (int e = 0; e < V; ++e) sums[wave][lane * V + e] = acc[e];
    if (lane == 0) {
      sums[wave][DH] = M;
      sums[wave][DH + 1] = L;
    }
    __syncthreads();
    if (member != 0) return;
    float top = -kInf;
    for (int w = 0; w < min(W, n); ++w) top = fmaxf(top, sums[wave + w][DH]);
    const float use = against(top);
    acc = 0.0f;
    L = 0.0f;
    for (int w = 0; w < min(W, n); ++w) {
      const float f = exp2_raw(sums[wave + w][DH] - use);
      L = fmaf(f, sums[wave + w][DH + 1], L);
#pragma unroll
      for (int e = 0; e < V; ++e) acc[e] = fmaf(f, sums[wave + w][lane * V + e], acc[e]);
    }
  }
  if (!mine) return;
#pragma unroll
  for (int e = 0; e < V; ++e)
    write_out<DH, T>(a, row, head, lane * V + e, wrong ? __builtin_nanf("") : n == 0 ? 0.0f : acc[e] / L);
}

template <int DH, typename T>
hipError_t launch(const PrefixArgs& a, int cus, hipStream_t st) {
  if (prefix_short(a.n_seqs, a.max_prefix, a.max_rest, a.hq, a.hkv)) {
    hipLaunchKernelGGL((prefix_short_kernel<DH, T>), dim3(uint32_t(prefix_short_blocks(a.n_seqs, a.n_groups, a.hq, a.hkv))),
                       dim3(kThreads), 0, st, a);
    return hipGetLastError();
  }
  const PrefixShape s = prefix_shape(a.n_seqs, a.n_groups, a.max_prefix, a.max_rest, a.hq, a.hkv, cus);
  const int64_t blocks = prefix_blocks(s, a.n_seqs, a.hkv);
  if (blocks > 0) {
    if (s.prefix_rows == 16)
      hipLaunchKernelGGL((prefix_kernel<DH, 1, false, T>), dim3(uint32_t(blocks)), dim3(kThreads), 0, st, a, s);
    else if (s.prefix_rows == 128)
      hipLaunchKernelGGL((prefix_kernel<DH, 1, true, T>), dim3(uint32_t(blocks)), dim3(kThreads), 0, st, a, s);
    else
      hipLaunchKernelGGL((prefix_kernel<DH, 2, false, T>), dim3(uint32_t(blocks)), dim3(kThreads), 0, st, a, s);
  }
  const int64_t rows = int64_t(a.n_seqs) * a.hq;
  if (s.prefix_splits + s.rest_splits > 4 && rows <= 4 * int64_t(cus))
    hipLaunchKernelGGL((prefix_join_kernel<DH, 4, T>), dim3(uint32_t(rows)), dim3(kThreads), 0, st, a, s);
  else
    hipLaunchKernelGGL((prefix_join_kernel<DH, 1, T>), dim3(uint32_t((rows + 3) / 4)), dim3(kThreads), 0, st, a, s);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_prefix_attention(const PrefixArgs& a, int cus, hipStream_t s) {
  if (a.n_seqs < 1) return hipSuccess;
  if (a.dh == 64) return a.type == HS_TYPE_BF16 ? launch<64, uint16_t>(a, cus, s) : launch<64, _Float16>(a, cus, s);
  return a.type == HS_TYPE_BF16 ? launch<128, uint16_t>(a, cus, s) : launch<128, _Float16>(a, cus, s);
}

}  // namespace hs
