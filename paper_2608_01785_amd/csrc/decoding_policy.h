// Splits and sizes of the kernels for decoding on a shared cache, shared by their
// launchers, the workspace sizes and the tests.  Pure C++; no HIP types.
#pragma once

#include <stddef.h>
#include <stdint.h>

#include "answer_policy.h"

namespace hs {

constexpr int kMaxCus = 256;  // of a device: no launch is sized for more
constexpr int64_t kMaxBlocks = (int64_t(1) << 24) - 1;  // of 256 threads: fewer than 2^32 in a grid

// hs_beam_select: beams of a group and selected continuations at most; the join
// holds beams * select candidates in LDS (48 KB at most) and its lists of keys
// cover a wavefront.
constexpr int kBeamMaxBeams = 64;
constexpr int kBeamMaxSelect = kLogprobsMaxTop;

// The scan's blocks: as hs_logprobs (see logprobs_shape), but the join is there in any
// case, so rows are split wherever CUs would idle: 85 rows of 50001 fp16 take 14.7 us in
// 3 blocks each and 16.2 whole.  Two or four blocks a CU cost the join what they save
// (32 rows of 65536 fp32: 12.7 us with one, 13.8 with two, 14.4 with four; the 85 rows 14.2
// with two).  Here and below, times are those of whole calls among others.
constexpr int kBeamPerCu = 1;
inline LogprobsShape beam_shape(int rows, int vocab, int elem_bytes, int cus) {
  const int chunk = 4096 / elem_bytes;
  const int chunks = int((int64_t(vocab) + 16 / elem_bytes - 1 + chunk - 1) / chunk);  // any row start
  if (int64_t(rows) >= 8 * int64_t(cus) || chunks < 2) return LogprobsShape{1, 1};
  int splits = rows < kBeamPerCu * cus ? kBeamPerCu * cus / rows : 1;
  if (splits > (chunks + 3) / 4) splits = (chunks + 3) / 4;
  if (splits > kLogprobsMaxSplits) splits = kLogprobsMaxSplits;
  return LogprobsShape{4, splits};
}

// Workspace bytes of a call of at most max_rows rows on any budget and type: a
// partial result for every block.
inline size_t beam_workspace(int64_t max_rows, int select) {
  const int64_t blocks = max_rows > kBeamPerCu * 256 ? max_rows : max_rows * kLogprobsMaxSplits < kBeamPerCu * 256
                                                                      ? max_rows * kLogprobsMaxSplits
                                                                      : kBeamPerCu * 256;
  return size_t(blocks) * logprobs_partial_bytes(select);
}

// hs_cache_copy: layers and copies of one launch (kernel arguments hold 4 KB), bytes of
// a block.  A head's run of so many value tiles (2^33 bytes at most) has copy_segments.
constexpr int kCopyLayers = 32;
constexpr int kCopyList = 200;
constexpr int kCopySegment = 8192;
constexpr int32_t copy_segments(int tiles, int dh) {
  return int32_t((int64_t(tiles) * 64 * dh + kCopySegment - 1) / kCopySegment);
}

// m / per_head = 2 m prefix_inverse(per_head) >> 32 for m < 2^31 / per_head: a launch
// has at most 2^25 columns, and at most this many query heads share a key/value head.
constexpr int kPrefixMaxPerHead = 64;
constexpr uint32_t prefix_inverse(int per_head) { return ((uint32_t(1) << 31) + per_head - 1) / per_head; }

// hs_prefix_attention: which rows go through one block together, and how the keys
// are split over blocks.
struct PrefixShape {
  int prefix_rows;    // rows (query heads of a group's sequences) of a block: 16, 32 or 128
  int prefix_tiles;   // row tiles of all groups together, at most
  int prefix_keys;    // keys of a block
  int prefix_splits;  // blocks over the longest prefix
  int rest_keys, rest_splits;
};

constexpr int kPrefixMaxSplits = 64;  // of a prefix, and of what a row has to itself
constexpr int kPrefixKeys = 128;      // a block's keys are a multiple: a tile for each wavefront

inline int64_t prefix_up(int64_t n, int64_t to) { return (n + to - 1) / to; }

// Keys of a block where `blocks` blocks share each split of `keys` keys.
inline int prefix_split_keys(int64_t keys, int64_t blocks, int cus, int per_cu) {
  if (keys < 1) return kPrefixKeys;
  int64_t splits = prefix_up(per_cu * int64_t(cus), blocks < 1 ? 1 : blocks);
  if (splits > kPrefixMaxSplits) splits = kPrefixMaxSplits;
  return int(prefix_up(prefix_up(keys, splits), kPrefixKeys) * kPrefixKeys);
}

// Tiles: up to 128 columns a group on average go in narrow ones, which read the keys
// again for every 32 (out of L2): 98 columns behind 8192 positions 15.9 us against 19.1
// in a wide one; 168 behind 30000 48.2 against 34.7 (28 / 4 heads of 128).
// Blocks a CU are counted for the groups' columns packed into whole tiles.  Groups that
// end inside a tile launch more: 5 groups of 36 columns are counted as 6 tiles and take 10.
// Wide tiles: two blocks a CU, whose products and exponentials overlap (128 rows in 32 / 8
// heads of 128 behind 16384 positions 62 us, with one 69; behind 32768, 99 and 125); one
// where the rows' own keys take more than about a fourth as long to read, which then share
// the CUs from the start (behind 16384 with up to 512 keys more 74 us against 79).
// Narrow tiles: one block a CU.  More leave more states than the shorter ranges save: 8
// rows in 28 / 4 heads behind 8192 positions, with up to 128 keys more, take 13.7 us with
// one, 18.3 with two; behind 30000, 20.3 and 28.3.
// What rows have to themselves: two blocks a CU beside the prefixes' (20 rows in 5 groups
// behind up to 1501 positions, with up to 700 keys more, in 32 / 8 heads 17.0 us against
// 19.7 with four), eight alone (45 rows of up to 2000 keys 34.5 us against 37.2 with two).
constexpr int kPrefixPerCu = 2;  // blocks over the prefixes, at most
constexpr int kRestPerCu = 8;    // blocks over what rows have to themselves, at most
inline PrefixShape prefix_shape(int n_seqs, int n_groups, int max_prefix, int max_rest, int hq, int hkv, int cus) {
  const int64_t per_head = hq / hkv, rows = int64_t(n_seqs) * per_head;
  PrefixShape s{};
  s.prefix_rows = max_prefix < 1 || rows <= 16 * int64_t(n_groups) ? 16 : rows <= 128 * int64_t(n_groups) ? 32 : 128;
  s.prefix_tiles = max_prefix > 0 ? int(rows / s.prefix_rows + n_groups) : 0;
  const bool wide = s.prefix_rows == 128, long_rest = 240 * int64_t(max_rest) > per_head * max_prefix;
  s.prefix_keys = prefix_split_keys(max_prefix, prefix_up(rows, s.prefix_rows) * hkv, cus,
                                  wide && !long_rest ? kPrefixPerCu : 1);
  s.prefix_splits = int(prefix_up(max_prefix, s.prefix_keys));
  const bool beside = int64_t(s.prefix_tiles) * s.prefix_splits * hkv >= cus / 2;
  s.rest_keys = prefix_split_keys(max_rest, int64_t(n_seqs) * hkv, cus, beside ? 2 : kRestPerCu);
  s.rest_splits = int(prefix_up(max_rest, s.rest_keys));
  return s;
}

// Whether one block takes 16 columns over all that they look at: so many tiles of 32 keys
// at most, for four wavefronts.
constexpr int kPrefixShortTiles = 16;
inline bool prefix_short(int n_seqs, int max_prefix, int max_rest, int hq, int hkv) {
  const int64_t touched = prefix_up(16, hq / hkv) + 1, rows = touched < n_seqs ? touched : n_seqs;
  return prefix_up(max_prefix, 32) + rows * (max_rest ? prefix_up(max_rest, 32) + 1 : 0) <= kPrefixShortTiles;
}

inline int64_t prefix_short_blocks(int n_seqs, int n_groups, int hq, int hkv) {
  return (int64_t(n_seqs) * (hq / hkv) / 16 + (n_groups > 0 ? n_groups : 1)) * hkv;
}

// Blocks of a launch: of the prefixes, then of what rows have to themselves.
inline int64_t prefix_blocks(const PrefixShape& s, int n_seqs, int hkv) {
  return (int64_t(s.prefix_tiles) * s.prefix_splits + int64_t(n_seqs) * s.rest_splits) * hkv;
}

// A partial state: dh unnormalised outputs, and the maximum and sum behind them.
inline size_t prefix_part_bytes(int dh) { return size_t(4 * dh + 8); }

// What a launch of this shape writes.
inline size_t prefix_states_bytes(const PrefixShape& s, int n_seqs, int hq, int dh) {
  return size_t(n_seqs) * hq * size_t(s.prefix_splits + s.rest_splits) * prefix_part_bytes(dh);
}

// Workspace bytes for at most n_seqs rows, on any budget.  Fewer rows or groups, a
// smaller bound and fewer CUs never take more partial states than this: `blocks` blocks
// share at most per_cu cus / blocks + 1 splits (per_cu: kPrefixPerCu and kRestPerCu at
// most), and each holds prefix_rows (at most 128; rest: per_head) states of a split.
inline size_t prefix_workspace(int n_seqs, int max_prefix, int max_rest, int hq, int hkv, int dh) {
  const int64_t rows = int64_t(n_seqs) * hq;
  auto states = [&](int64_t keys, int64_t of_block) {
    int64_t splits = prefix_up(keys, kPrefixKeys);
    if (splits > kPrefixMaxSplits) splits = kPrefixMaxSplits;
    const int64_t shared = kMaxCus * of_block + rows, each = rows * splits;
    return splits < 1 ? 0 : each < shared ? each : shared;
  };
  return size_t(states(max_prefix, kPrefixPerCu * 128) + states(max_rest, kRestPerCu * (hq / hkv))) *
         prefix_part_bytes(dh);
}

}  // namespace hs
