// Pieces of attention over 64-key tiles in LDS with 32-query MFMA columns, shared by
// the prefill kernel and the one behind shared prefixes: LDS placement, addressing of
// a cache's tiles, one step of the running softmax.
#pragma once

#include "hs_device.h"

namespace hs {
namespace {

constexpr int BKV = 64;

// LDS placement of 16-byte chunk c of key row r (DH * 2 bytes per row).  A
// 16-lane pass of fragment reads takes one logical chunk of 16 distinct rows
// (perm32 of 16 consecutive indices).  With 256-byte rows every row starts on
// bank 0, so the 16 rows need 16 different physical chunks (c ^ (r & 15));
// with 128-byte rows odd rows start on bank 32, so the chunks need only
// differ within each parity (c ^ ((r >> 1) & 7)).
template <int DH>
__device__ __forceinline__ int kphys(int r, int c) {
  return DH == 128 ? (c ^ (r & 15)) : (c ^ ((r >> 1) & 7));
}

// Chunk c (8 keys) of value row d (64 keys, 128 bytes): odd rows start on bank
// 32, so a pass over 16 consecutive rows needs distinct chunks per parity.
__device__ __forceinline__ int vphys(int d, int c) { return c ^ ((d >> 1) & 7); }

// Buffer resource over the cache array `base` from element `off` on: the
// 64-bit start is block-uniform, so it is moved to scalar registers; tile
// loads then take a per-lane constant offset plus a uniform tile offset and
// need no vector address arithmetic.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t cache_rsrc(const uint16_t* base, int64_t off) {
  const uint64_t addr = reinterpret_cast<uint64_t>(base + off);
  const uint32_t lo = __builtin_amdgcn_readfirstlane(uint32_t(addr));
  const uint32_t hi = __builtin_amdgcn_readfirstlane(uint32_t(addr >> 32));
  return __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<void*>((uint64_t(hi) << 32) | lo), 0, 0x7ffffff0,
                                           0x00020000);
}

// The reference maximum of the online softmax moves only when a tile's
// maximum exceeds it by more than this (log2 units): weights are then at
// most 2^8, well inside fp16, and the output rescale is skipped on almost
// every tile.  Any reference value gives the same softmax; only rounding
// differs.
constexpr float kLazyMax = 8.0f;

// One online-softmax step over a 64-key tile of scores held as two 32-key
// subtiles (register r of subtile st: key kv0 + 32 st + 16 (r / 8) + 8 fh +
// r % 8 of the lane's query).  `lim` = qpos - kv0 - 8 fh: keys with
// 32 st + 16 (r / 8) + r % 8 > lim are masked when `mask` is set.  The
// weights are left in `pf` as the B operand of O^T = V^T P^T.
template <int NDS>
__device__ __forceinline__ void softmax_tile(f32x16 (&s)[2], f32x16 (&o)[NDS], u32x4 (&pf)[4], float& m_run,
                                             float& l_run, float scale_log2, bool mask, int lim) {
  if (mask) {
#pragma unroll
    for (int st = 0; st < 2; ++st)
#pragma unroll
      for (int r = 0; r < 16; ++r)
        if (32 * st + 16 * (r >> 3) + (r & 7) > lim) s[st][r] = -INFINITY;
  }
  float mx = -INFINITY;
#pragma unroll
  for (int st = 0; st < 2; ++st)
#pragma unroll
    for (int r = 0; r < 16; ++r) mx = fmaxf(mx, s[st][r]);
  mx = fmaxf(mx, __shfl_xor(mx, 32, 64)) * scale_log2;
  // A row that has seen no key yet keeps -inf; its exponents are taken
  // against 0, which gives weight 0.
  const bool move = mx > m_run + kLazyMax;
  const float m_new = move ? mx : m_run;
  const float m_use = against(m_new);
  const float alpha = exp2_raw(m_run - m_use);
  m_run = m_new;
  float psum = 0.0f;
#pragma unroll
  for (int st = 0; st < 2; ++st)
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const float p = exp2_raw(fmaf(s[st][r], scale_log2, -m_use));
      s[st][r] = p;
      psum += p;
    }
  l_run = l_run * alpha + psum;
  if (__ballot(move) != 0) {
#pragma unroll
    for (int i = 0; i < NDS; ++i)
#pragma unroll
      for (int r = 0; r < 16; ++r) o[i][r] *= alpha;
  }
  // P^T fragments: key block kb2 (16 keys) = registers 8 (kb2 % 2) .. +8 of subtile kb2 / 2.
#pragma unroll
  for (int kb2 = 0; kb2 < 4; ++kb2) {
    const int st = kb2 >> 1, r0 = 8 * (kb2 & 1);
#pragma unroll
    for (int e = 0; e < 4; ++e) pf[kb2][e] = pack2h_rne(s[st][r0 + 2 * e], s[st][r0 + 2 * e + 1]);
  }
}

}  // namespace
}  // namespace hs
