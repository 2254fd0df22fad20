// Host rules of the answering kernels (plain C++).
#pragma once

#include <stddef.h>
#include <stdint.h>

namespace hs {

constexpr int kLogprobsMaxTop = 64;       // alternatives a row can list: one per lane of a wavefront
constexpr int kLinearI8MaxK = 131071;     // (-128)^2 k stays below 2^31
constexpr int64_t kLinearI8MaxStride = int64_t(1) << 22;  // 256 rows of an operand stay within 32-bit offsets

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
