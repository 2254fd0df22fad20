// Host rules of the answering kernels (plain C++).
#pragma once

#include <stddef.h>
#include <stdint.h>

namespace hs {

constexpr int kLogprobsMaxTop = 64;       // alternatives a row can list: one per lane of a wavefront
constexpr int kLinearI8MaxK = 131071;     // (-128)^2 k stays below 2^31
constexpr int64_t kLinearI8MaxStride = int64_t(1) << 22;  // 256 rows of an operand stay within 32-bit offsets

// The kernels of hs_linear_i8: for at most 32 or 64 rows, and tiles.
enum LinearI8Choice { kLinearI8Few32, kLinearI8Few64, kLinearI8Tile64, kLinearI8Tile128, kLinearI8Tile256 };

// Which of them an [m, k] x [n, k]^T product takes on `cus` compute units.  All
// give the same bits.
//
// Few rows: the kernels that share K among a block's waves need no channels to
// fill the chip, the tiles have less to read (and to add up) once there are
// many.  In us, us of the best tiles: 32 rows 4608 x 3584 6.4, 11.2; 3584 x
// 18944 18, 46; 37888 x 3584 29.5, 32.6; 65536 x 3584 58, 52.  64 rows: 8.6, 11.2;
// 26, 46; 14336 x 4096 18.6, 13.7; 65536 x 3584 82, 56.
//
// Tiles: a CU's time is the tiles it gets times a tile's 64-byte stages, in us
// as fitted to 44 products of 1 to 4096 rows.  Two 128 x 128 tiles side by side
// on a CU take as long as one after the other; a 256 x 256 stage takes longer the
// more of the chip works (its clock follows the power).  4096 x 8192 x 8192: 254
// us in 256s, 350 in 128s, 596 in 64s; 777 x 4096 x 4096: 49, 26, 35; 256 x 4608 x
// 3584: 41, 21, 16.
inline LinearI8Choice linear_i8_choice(int m, int n, int k, int cus) {
  if (m <= 32 && n <= 160 * int64_t(cus)) return kLinearI8Few32;
  if (m <= 64 && n <= 32 * int64_t(cus)) return m <= 32 ? kLinearI8Few32 : kLinearI8Few64;
  auto up = [](int64_t a, int64_t b) { return (a + b - 1) / b; };
  const float stages = float(up(k, 256)) * 4.0f;
  auto rounds = [&](int tile) { return float(up(up(m, tile) * up(n, tile), cus)); };
  const float t64 = 2.5f + rounds(64) * (0.14f * stages + 0.6f);
  const float t128 = 3.0f + rounds(128) * (0.335f * stages + 2.0f);
  // The 256s run in halves at the end (see linear_kernel).
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
  const float t256 = 6.0f + units * ((0.58f + 0.38f * float(grid) / float(cus)) * stages + 8.0f);
  if (t256 <= t128 && t256 <= t64) return kLinearI8Tile256;
  return t128 <= t64 ? kLinearI8Tile128 : kLinearI8Tile64;
}

// hs_logprobs: a row's elements go through wavefronts in chunks of 4 KB (one
// wavefront's registers); `waves` wavefronts form a block, and a row is split
// over `splits` blocks whose partial results a second kernel joins.
//
// Eight wavefronts per CU keep memory busy.  Rows enough for that take one
// wavefront each, since every wavefront pays for its alternatives once: 2048 x
// 131072 bf16, top 5, 122 us against 132 with four a row.  Fewer rows take
// blocks of four (1024 rows, top 20: 75 us against 93 with one a row and 127
// with eight), and as many blocks as make up the eight per CU: 32 x 65536 fp32,
// top 20, 13.7 us over 16 blocks a row, 15.0 over 8.
struct LogprobsShape {
  int waves;             // per block: 1 or 4
  int splits;            // blocks per row
  int chunks_per_split;
};

constexpr int kLogprobsMaxSplits = 64;    // the join takes one partial state per lane

inline LogprobsShape logprobs_shape(int rows, int vocab, int elem_bytes, int cus) {
  const int chunk = 4096 / elem_bytes;
  const int max_chunks = int((int64_t(vocab) + 16 / elem_bytes - 1 + chunk - 1) / chunk);  // any row start
  const int64_t want = (8 * int64_t(cus) + rows - 1) / (rows > 0 ? rows : 1);              // wavefronts per row
  const int per_row = int(want < max_chunks ? want : max_chunks);
  LogprobsShape s{1, 1, max_chunks};
  if (per_row > 1) {
    s.waves = 4;
    int splits = (per_row + 3) / 4;
    if (splits > kLogprobsMaxSplits) splits = kLogprobsMaxSplits;
    s.chunks_per_split = (max_chunks + splits - 1) / splits;
    s.splits = (max_chunks + s.chunks_per_split - 1) / s.chunks_per_split;
  }
  return s;
}

// A block's partial result: 16 bytes of sums, then top_k 8-byte keys.
inline size_t logprobs_partial_bytes(int top_k) { return 16 + 8 * ((size_t(top_k) + 1) / 2 * 2); }

// Workspace bytes of a call of at most max_rows rows on any budget and type: at
// most rows x ceil(512 / rows) < 512 + rows blocks where rows are split (256
// CUs, fewer than 512 rows), and at most one block per 4 chunks of a row.
inline size_t logprobs_workspace(int64_t max_rows, int64_t vocab, int top_k) {
  const int64_t rows = max_rows < 511 ? max_rows : 511;
  int64_t splits = ((vocab + 3 + 1023) / 1024 + 3) / 4;
  if (splits > kLogprobsMaxSplits) splits = kLogprobsMaxSplits;
  if (splits <= 1) return 0;
  const int64_t blocks = rows * splits < 512 + rows ? rows * splits : 512 + rows;
  return size_t(blocks) * logprobs_partial_bytes(top_k);
}

}  // namespace hs
