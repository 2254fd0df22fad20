// Host rules of the answering kernels (plain C++).
#pragma once

#include <stddef.h>
#include <stdint.h>

namespace hs {

constexpr int kLogprobsMaxTop = 64;       // alternatives a row can list: one per lane of a wavefront
constexpr int kLinearI8MaxK = 131071;     // (-128)^2 k stays below 2^31
constexpr int64_t kLinearI8MaxStride = int64_t(1) << 22;  // 256 rows of an operand stay within 32-bit offsets

// How hs_linear_i8 reads 16-byte aligned operands: in stages of one 128-byte
// line of K, eight rows to a load, 16 bytes to a lane, through a buffer resource
// that ends with the k bytes of the last of `span` rows.  The vector offset is
// what the resource's end is checked against; a scalar offset may or may not
// count.  So rows and what lies past k are told apart by the vector offset alone,
// and the scalar offset is the stage's, which stays inside the row.
struct LinearI8Load {
  uint32_t vector, scalar;  // byte offsets
};
constexpr int kLinearI8Line = 128;
constexpr uint32_t linear_i8_records(int span, int64_t ld, int k) {
  return uint32_t(span - 1) * uint32_t(ld) + uint32_t(k);
}
// A lane's place in load 0 of stage 0.
constexpr uint32_t linear_i8_offset(int lane, int64_t ld) {
  return uint32_t(lane / 8) * uint32_t(ld) + uint32_t(lane % 8 * 16);
}
// Load l (rows 8 l .. 8 l + 7) of a stage.  Past k it reads zeros: 2^31 is beyond
// any resource, with up to 63 rows of stride kLinearI8MaxStride on top as well.
constexpr LinearI8Load linear_i8_load(uint32_t offset, int lane, int l, int stage, int64_t ld, int k) {
  const bool past = stage >= k / kLinearI8Line && stage * kLinearI8Line + lane % 8 * 16 >= k;
  const int last = (k - 1) / kLinearI8Line;
  return LinearI8Load{(past ? 0x80000000u : offset) + uint32_t(8 * l) * uint32_t(ld),
                      uint32_t(stage < last ? stage : last) * uint32_t(kLinearI8Line)};
}

// The kernels of hs_linear_i8: for few rows (32 or 64 a block, by 32 or 64
// channels), and tiles.
enum LinearI8Choice {
  kLinearI8Few32,
  kLinearI8Few64,
  kLinearI8Few64x64,
  kLinearI8Tile64,
  kLinearI8Tile128,
  kLinearI8Tile256
};

// Which of them an [m, k] x [n, k]^T product takes on `cus` compute units.  All
// give the same bits, so the choice may follow the budget.  The times below
// are in us, fitted to some 80 products of 1 to 4096 rows on the whole chip.
//
// The kernels for few rows share K among a block's waves, so they need no
// channels to fill the chip; the tiles have less to read and to add up once
// there are many.  Few rows against the best tiles: 32 rows 4608 x 3584 6.5, 10.8;
// 3584 x 18944 18, 43; 65536 x 4096 65, 55.  128 rows: 1024 x 4096 7.5, 12; 3584 x
// 18944 26, 45; 14336 x 4096 34, 19.  32 rows a block where the blocks fit the
// chip, 64 where that halves the rounds: 64 rows 3584 x 18944 19 against 25, 100
// rows 4096 x 4096 10.7 against 9.3.  64 by 64 reads half as much a product and
// runs alone on its CU, for long sums of more rows: 192 rows 3584 x 18944 36
// against 49 and 51, and 45 in tiles; 100 rows 8192 x 8192 20 against 42, 30 and 23.
//
// A CU's time in tiles is the tiles it gets times a tile's 64-byte steps.  64 x
// 64 tiles, four on a CU at a time, hide their latency behind each other; of
// 128 x 128 tiles it runs two, which take little less than one after the other;
// a 256 x 256 step takes longer the more of the chip works, whose clock follows
// the power.  4096 x 8192 x 8192: 235 in 256s, 323 in 128s, 477 in 64s; 777 x
// 4096 x 4096: 44, 24, 30; 256 x 4608 x 3584: 39, 20, 17.  Over 143 products of 1
// to 1024 rows the rule loses 0.8 % against the fastest (192 x 37888 x 3584 most: 63
// in 128s, 48 in 256s).  The constants are those of 256 CUs, of which every CU
// is taken to have its share of memory's rate.  64 CUs reach half of it and not a
// fourth, so on part of the chip the rule loses more: 3 % on 128 CUs, 7 % on 64,
// there 48 x 14336 x 4096 47 for few rows against 27 in 64s.
//
// Rows that are not 16-byte aligned cost the address unit twice as much a load,
// which the kernels that use a load least feel most: 512 x 4608 x 3583 40 in 64s
// and 29 in 128s (22 and 21 aligned), 64 x 1024 x 1023 11 for few rows and 8 in
// 64s (6.7 and 6.2 aligned).  256s have no registers for their addresses, and 64 by
// 64 for few rows is behind the tiles (256 x 4096 x 4095 22, 18).
inline LinearI8Choice linear_i8_choice(int m, int n, int k, int cus, bool aligned) {
  auto up = [](int64_t a, int64_t b) { return (a + b - 1) / b; };
  auto larger = [](float a, float b) { return a > b ? a : b; };
  const float steps = float(up(k, 256)) * 4.0f, kf = float(k), fcus = float(cus), w_bytes = float(n) * kf / fcus;
  const int64_t tiles64 = up(m, 64) * up(n, 64), full64 = tiles64 / (4 * cus);
  const float rest64 = float(up(tiles64 - full64 * 4 * cus, cus)), slots64 = float(tiles64) / (4.0f * fcus);
  // The time of the channels' stream stretches where CUs get unequal numbers of
  // tiles, by a part of what the largest number is above the mean.
  auto stretch = [&](int64_t tiles, int64_t places, float part) {
    return 1.0f + part * (float(up(tiles, places) * places) / float(tiles) - 1.0f);
  };
  const float each64 = aligned ? 0.11f : 0.21f, alone64 = aligned ? 0.145f : 0.2f;
  float work64 = 2.5f + float(full64) * (4.0f * each64 * steps + 3.0f);
  if (rest64 > 0.0f) work64 += steps * larger(alone64, each64 * rest64) + 0.75f * rest64 + (full64 > 0 ? 1.0f : 0.0f);

  LinearI8Choice best = kLinearI8Tile64;
  // Rows of a tile take from the rate of the channels' stream.
  auto fill = [&](int tile, float part) { return 1.0f + part * float(m < tile ? m : tile); };
  float cost = larger(work64, 3.0f + stretch(tiles64, slots64 > 1.0f ? 4 * cus : cus, slots64 > 1.0f ? 0.5f : 0.2f) *
                                         fill(64, 0.003f) * w_bytes / 20700.0f);
  auto offer = [&](LinearI8Choice c, float t) {
    if (t < cost) {
      cost = t;
      best = c;
    }
  };
  // Tiles of both kinds: a last row of them that holds at most half its rows
  // costs half.
  const int64_t tm128 = up(m, 128), tn128 = up(n, 128);
  const bool short128 = m - (tm128 - 1) * 128 <= 64;
  const float rounds128 = (float(tm128) - (short128 ? 0.5f : 0.0f)) * float(tn128) / fcus;
  const float pairs = float(int64_t(0.5f * rounds128)), rest128 = rounds128 - 2.0f * pairs;
  const float step128 = aligned ? steps : 1.4f * steps;
  const float work128 = 3.0f + pairs * (0.6f * step128 + 2.5f) +
                        (rest128 > 1.0f ? 0.5f * step128 + 4.0f : rest128 > 0.0f ? 0.305f * step128 + 3.5f : 0.0f);
  offer(kLinearI8Tile128, larger(work128, 3.0f + stretch(tm128 * tn128, cus, 0.45f) * fill(128, 0.0018f) *
                                                     w_bytes / 20700.0f));
  const int64_t tm = up(m, 256), tn = up(n, 256);
  const bool short_last = m - (tm - 1) * 256 <= 128;
  const int64_t whole = (short_last ? tm - 1 : tm) * tn, halves = short_last ? tn : 0;
  const int64_t grid = tm * tn < cus ? tm * tn : cus, tail = whole % grid;
  float units = float(whole / grid);
  if (tail > 0 && 2 * tail + halves <= grid) {
    units += 0.6f;
  } else {
    units += tail > 0 ? 1.0f : 0.0f;
    const int64_t rest = halves - (tail > 0 ? grid - tail : 0);
    units += rest > 0 ? 0.6f * float(up(rest, grid)) : 0.0f;
  }
  if (aligned)
    offer(kLinearI8Tile256, larger(6.0f + units * ((0.45f + 0.38f * float(grid) / fcus) * steps + 8.0f),
                                   3.0f + stretch(tm * tn, cus, 0.4f) * fill(128, 0.0012f) * w_bytes / 20000.0f));
  // A grid's first dimension holds fewer than 2^32 threads, its second 65535
  // row groups.
  const int64_t few = up(n, 32);
  if (few < (1 << 23) && up(m, 32) <= 65535) {
    const float load = aligned ? 1.0f : 2.0f;
    const float rounds32 = float(up(few * up(m, 32), cus)), rounds64 = float(up(few * up(m, 64), cus));
    const float read32 = (rounds32 > 1.0f && m > 32 ? 1.6f : 1.0f) * fill(32, 0.008f) * w_bytes / 20700.0f;
    offer(kLinearI8Few32, larger(5.0f, 3.0f + load * larger(rounds32 * (0.00085f * kf + 0.2f), read32)));
    const float rounds6464 = float(up(up(n, 64) * up(m, 64), cus));
    if (m > 32 && aligned)
      offer(kLinearI8Few64x64, larger(rounds6464 * (0.00165f * kf + 5.0f),
                                      3.5f + stretch(tiles64, cus, 0.2f) * fill(64, 0.003f) * w_bytes / 20700.0f));
    if (m > 32)
      offer(kLinearI8Few64, larger(2.5f + rounds64 * load * (0.0013f * kf + 2.0f),
                                   2.0f + load * 0.0018f * kf * float(few) / fcus));
  }
  return best;
}

// hs_logprobs: a row's elements go through wavefronts in chunks of 4 KB (one
// wavefront's registers); `waves` wavefronts form a block, and a row is split
// over `splits` blocks whose partial results a second kernel joins.
//
// From 8 rows a CU on, a wavefront takes a row, since every block pays for its
// alternatives once: 4096 x 32000 bf16, top 20, 64 us against 83 with four a
// row.  Fewer rows take blocks of four (1024 x 131072: 60 us against 70 with
// one), and rows that leave CUs idle are split over them, where that saves more
// than the second kernel takes, about the time of 18 chunks of 16-bit logits
// for a block of four (25 of fp32).  64 x 131072, top 20: 21 us whole, 15 in 4
// splits, 16 in 8; 1 x 50001: 12.7 whole, 11.3 in 8; 8 x 32000, top 5: 10.2
// whole, 10.5 in 8; 128 x 32000 fp32: 11.5 whole, 12.7 in 2.
struct LogprobsShape {
  int waves;             // per block: 1 or 4
  int splits;            // blocks per row
};

constexpr int kLogprobsMaxSplits = 64;    // the join takes one partial state per lane

inline LogprobsShape logprobs_shape(int rows, int vocab, int elem_bytes, int cus) {
  const int chunk = 4096 / elem_bytes;
  const int chunks = int((int64_t(vocab) + 16 / elem_bytes - 1 + chunk - 1) / chunk);  // any row start
  if (int64_t(rows) >= 8 * int64_t(cus) || chunks < 2) return LogprobsShape{1, 1};
  int splits = rows < cus ? cus / rows : 1;
  if (splits > (chunks + 3) / 4) splits = (chunks + 3) / 4;
  if (splits > kLogprobsMaxSplits) splits = kLogprobsMaxSplits;
  const int join = elem_bytes == 4 ? 25 : 18;
  if (chunks - chunks / splits <= join) splits = 1;
  return LogprobsShape{4, splits};
}

// A block's partial result: 16 bytes of sums, then top_k 8-byte keys.
inline size_t logprobs_partial_bytes(int top_k) { return 16 + 8 * ((size_t(top_k) + 1) / 2 * 2); }

// Workspace bytes of a call of at most max_rows rows on any budget and type:
// rows x (256 / rows) blocks at most where rows are split, and at most one block
// per 4 chunks of a row.
inline size_t logprobs_workspace(int64_t max_rows, int64_t vocab, int top_k) {
  int64_t splits = ((vocab + 3 + 1023) / 1024 + 3) / 4;
  if (splits > kLogprobsMaxSplits) splits = kLogprobsMaxSplits;
  if (splits <= 1) return 0;
  const int64_t blocks = max_rows * splits < 256 ? max_rows * splits : 256;
  return size_t(blocks) * logprobs_partial_bytes(top_k);
}

}  // namespace hs
