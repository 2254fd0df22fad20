// Launch interface of the kernels for decoding on a shared cache: selection over
// beams, copies within the cache, attention behind shared prefixes (internal to
// the library).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "decoding_policy.h"

namespace hs {

struct BeamArgs {
  const void* logits;      // [groups * beams, vocab] of `type`, row stride ld
  int type;                // HS_TYPE_*
  int64_t ld;
  int groups, beams, vocab;
  const float* scores;     // [groups, beams]
  const uint8_t* finished; // [groups, beams] or null
  int end_token;           // or -1
  int select;
  float* out_scores;       // [groups, select]
  int32_t* out_parents;
  int32_t* out_tokens;
  uint8_t* out_finished;   // or null
  void* part;              // beam_workspace() bytes
};
hipError_t launch_beam_select(const BeamArgs& a, int cus, hipStream_t s);

// One launch of copies: what it needs sits in the kernel's arguments, so that
// nothing is staged and a captured launch keeps its list.
struct CacheCopyArgs {
  struct Copy {
    int32_t src, dst, tiles;  // slots, value tiles (32 positions) to copy
    int32_t first;            // segments of a head's runs before this copy's
  };
  uint16_t* k[kCopyLayers];
  uint16_t* v[kCopyLayers];
  Copy copies[kCopyList];
  int32_t layers, n_copies, heads, dh;
  int32_t segments;           // of a head's runs, all copies together
  int64_t head_bytes;         // bytes of one head of a slot
};
static_assert(sizeof(CacheCopyArgs) <= 4096, "kernel arguments");
hipError_t launch_cache_copy(const CacheCopyArgs& a, int cus, hipStream_t s);

// Attention of one row a sequence (see prefix_attention.hip).
struct PrefixArgs {
  const void* q;            // [n_seqs, hq, dh], row stride ldq
  int type;                 // HS_TYPE_F16 or HS_TYPE_BF16, of q and out
  int64_t ldq;
  void* out;                // [n_seqs, hq * dh], row stride ldo, or (out_k8_rows > 0) fp16 k-group-major
  int64_t ldo;
  int out_k8_rows;
  const uint16_t* k;        // one layer's keys and values, cache layout (kv_tile_keys)
  const uint16_t* v;
  int n_slots, page;        // positions of a slot
  const int32_t* table;     // [n_seqs, pages_per_seq]
  int pages_per_seq;
  const int32_t* lens;      // [n_seqs] keys of each row
  int n_seqs;
  const int32_t* offsets;   // [n_groups + 1] rows of each group
  const int32_t* prefix;    // [n_groups] shared positions
  int n_groups;
  int max_prefix, max_rest; // bounds of the prefixes and of what the rows have to themselves
  int hq, hkv, dh;
  uint32_t per_head_inv;    // prefix_inverse(hq / hkv)
  float scale_log2;         // log2(e) / sqrt(dh)
  void* part;               // prefix_workspace() bytes
};
hipError_t launch_prefix_attention(const PrefixArgs& a, int cus, hipStream_t s);

}  // namespace hs
