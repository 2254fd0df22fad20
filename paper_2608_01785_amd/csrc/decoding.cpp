// Entry points of decoding on a shared cache: selection over beams, copies within
// the cache, attention behind shared prefixes.  Argument checks and launches.
#include <hip/hip_runtime.h>
#include <math.h>

#include <algorithm>
#include <new>
#include <vector>

#include "call_checks.h"
#include "decoding_kernels.h"

using namespace hs;

namespace {

constexpr int32_t kBeamMaxRows = 1 << 22;      // a block of 256 threads each, 64 splits or one: fewer than 2^32 threads
constexpr int64_t kMaxSlotBytes = int64_t(1) << 33;
constexpr int32_t kMaxSlots = 1 << 28;  // a cache's bytes stay below 2^62
constexpr int32_t kMaxKvHeads = 1024;

hs_status check_workspace(const void* workspace, size_t ws_bytes, size_t need) {
  if (!need) return HS_OK;
  if (!workspace) return fail(HS_ERR_WORKSPACE, "workspace is null");
  if (reinterpret_cast<uintptr_t>(workspace) % 16 != 0)
    return fail(HS_ERR_INVALID_ARG, "workspace is not aligned to 16 bytes");
  if (ws_bytes < need) return fail(HS_ERR_WORKSPACE, "workspace has %zu bytes, %zu needed", ws_bytes, need);
  return HS_OK;
}

hs_status check_aligned16(const char* name, const void* p) {
  if (reinterpret_cast<uintptr_t>(p) % 16 != 0) return fail(HS_ERR_INVALID_ARG, "%s is not aligned to 16 bytes", name);
  return HS_OK;
}

hs_status check_heads(int32_t hkv, int32_t dh) {
  if (hkv < 1) return fail(HS_ERR_INVALID_ARG, "%d key/value heads", hkv);
  if (hkv > kMaxKvHeads) return fail(HS_ERR_UNSUPPORTED, "%d key/value heads: at most %d", hkv, kMaxKvHeads);
  if (dh != 64 && dh != 128) return fail(HS_ERR_UNSUPPORTED, "head_dim %d must be 64 or 128", dh);
  return HS_OK;
}

hs_status check_pages(int32_t n_slots, int32_t page, int32_t hkv, int32_t dh) {
  if (n_slots < 1) return fail(HS_ERR_INVALID_ARG, "the cache has %d slots", n_slots);
  if (page < 64 || page % 64 != 0)
    return fail(HS_ERR_INVALID_ARG, "%d positions a slot: must be a positive multiple of 64", page);
  if (int64_t(page) * hkv * dh * 2 > kMaxSlotBytes)
    return fail(HS_ERR_UNSUPPORTED, "a slot of %d positions exceeds %lld bytes", page, (long long)kMaxSlotBytes);
  if (n_slots > kMaxSlots) return fail(HS_ERR_UNSUPPORTED, "%d slots: at most %d", n_slots, kMaxSlots);
  return HS_OK;
}

}  // namespace

extern "C" {

hs_status hs_beam_select_workspace_size(int32_t max_groups, int32_t beams, int32_t vocab, int32_t n_select,
                                        size_t* bytes) {
  clear_error();
  if (!bytes) return fail(HS_ERR_INVALID_ARG, "output pointer is null");
  if (max_groups < 0 || beams < 1 || vocab < 1 || n_select < 1)
    return fail(HS_ERR_INVALID_ARG, "%d groups of %d beams, vocabulary %d, %d selected", max_groups, beams, vocab,
                n_select);
  if (beams > kBeamMaxBeams || n_select > kBeamMaxSelect)
    return fail(HS_ERR_UNSUPPORTED, "%d beams, %d selected: at most %d and %d", beams, n_select, kBeamMaxBeams,
                kBeamMaxSelect);
  const int64_t rows = int64_t(max_groups) * beams;
  if (rows > kBeamMaxRows) return fail(HS_ERR_UNSUPPORTED, "%lld rows: at most %d", (long long)rows, kBeamMaxRows);
  *bytes = beam_workspace(rows, n_select);
  return HS_OK;
}

// Bytes of the partial results of one call on `cus` CUs, as internal.
uint64_t hs_beam_select_states(int32_t rows, int32_t vocab, int32_t elem_bytes, int32_t n_select, int32_t cus) {
  return uint64_t(rows) * beam_shape(rows, vocab, elem_bytes, cus).splits * logprobs_partial_bytes(n_select);
}

hs_status hs_beam_select(hs_context* ctx, const void* logits, int32_t type, int64_t ld, int32_t groups, int32_t beams,
                         int32_t vocab, const float* scores, const uint8_t* finished, int32_t end_token,
                         int32_t n_select, float* out_scores, int32_t* out_parents, int32_t* out_tokens,
                         uint8_t* out_finished, int32_t cu_budget, void* stream, void* workspace, size_t ws_bytes) {
  size_t need = 0;
  HS_TRY(hs_beam_select_workspace_size(groups, beams, vocab, n_select, &need));  // the shape's checks
  HS_TRY(check_type("logits", type));
  if (end_token < -1 || end_token >= vocab)
    return fail(HS_ERR_INVALID_ARG, "end_token %d outside [-1, %d)", end_token, vocab);
  if (finished && end_token < 0) return fail(HS_ERR_INVALID_ARG, "finished beams need an end_token");
  const int32_t rows = groups * beams;
  const Span sz = rows_of("logits", logits, rows, vocab, ld, type_size(type));
  const Span ss = rows_of("scores", scores, rows, 1, 1, 4);
  const Span sf = rows_of("finished", finished, rows, 1, 1, 1);
  const Span os = rows_of("out_scores", out_scores, groups, n_select, n_select, 4);
  const Span op = rows_of("out_parents", out_parents, groups, n_select, n_select, 4);
  const Span ot = rows_of("out_tokens", out_tokens, groups, n_select, n_select, 4);
  const Span of = rows_of("out_finished", out_finished, groups, n_select, n_select, 1);
  const Span sws = {"workspace", workspace, need};
  HS_TRY(check_matrix(sz, rows, vocab, ld, type_size(type)));
  HS_TRY(check_matrix(ss, rows, 1, 1, 4));
  for (const Span& out : {os, op, ot}) HS_TRY(check_matrix(out, groups, n_select, n_select, 4));
  const Span outs[] = {os, op, ot, of, sws};
  for (const Span& out : outs)
    for (const Span& in : {sz, ss, sf}) HS_TRY(check_disjoint(out, in));
  for (const Span& out : outs)
    for (const Span& other : outs)
      if (&other > &out) HS_TRY(check_disjoint(out, other));
  if (groups) HS_TRY(check_workspace(workspace, ws_bytes, need));
  if (cu_budget < 1) return fail(HS_ERR_BUDGET, "CU budget %d", cu_budget);  // sizes the launch below
  if (groups && hs_beam_select_states(rows, vocab, int32_t(type_size(type)), n_select, std::min(cu_budget, kMaxCus)) > need)
    return fail(HS_ERR_INTERNAL, "the launch's partial results exceed the workspace");
  BeamArgs a{logits,   type,       ld,          groups,     beams,        vocab,    scores,
             finished, end_token,  n_select,    out_scores, out_parents,  out_tokens, out_finished,
             workspace};
  return run(ctx, cu_budget, stream, groups == 0, HS_KERNEL_BEAM_SELECT,
             [&](hipStream_t s) { return launch_beam_select(a, cu_budget, s); });
}

hs_status hs_cache_copy(hs_context* ctx, const hs_kv_cache* kv, int32_t n_layers, int32_t n_kv_heads, int32_t head_dim,
                        const int32_t* src, const int32_t* dst, const int32_t* positions, int32_t n_copies,
                        int32_t cu_budget, void* stream) {
  clear_error();
  if (!kv || !kv->k || !kv->v) return fail(HS_ERR_INVALID_ARG, "the cache is null");
  if (n_layers < 1) return fail(HS_ERR_INVALID_ARG, "n_layers %d < 1", n_layers);
  HS_TRY(check_heads(n_kv_heads, head_dim));
  HS_TRY(check_pages(kv->n_slots, kv->max_ctx, n_kv_heads, head_dim));
  for (int32_t l = 0; l < n_layers; ++l) {
    if (!kv->k[l] || !kv->v[l]) return fail(HS_ERR_INVALID_ARG, "cache of layer %d is null", l);
    HS_TRY(check_aligned16("the cache", kv->k[l]));
    HS_TRY(check_aligned16("the cache", kv->v[l]));
  }
  if (n_copies < 0 || (n_copies > 0 && (!src || !dst)))
    return fail(HS_ERR_INVALID_ARG, "%d copies, or their slots are null", n_copies);
  for (int32_t i = 0; i < n_copies; ++i) {
    for (int32_t slot : {src[i], dst[i]})
      if (slot < 0 || slot >= kv->n_slots)
        return fail(HS_ERR_INVALID_ARG, "copy %d: slot %d outside [0, %d)", i, slot, kv->n_slots);
    if (positions && (positions[i] < 0 || positions[i] > kv->max_ctx))
      return fail(HS_ERR_INVALID_ARG, "copy %d: %d positions of %d", i, positions[i], kv->max_ctx);
  }
  try {
    // Copies run at the same time: what one writes no other may touch.
    std::vector<uint8_t> written(size_t(kv->n_slots), 0);
    for (int32_t i = 0; i < n_copies; ++i) {
      if (written[dst[i]]) return fail(HS_ERR_INVALID_ARG, "slot %d is the destination of two copies", dst[i]);
      written[dst[i]] = 1;
    }
    for (int32_t i = 0; i < n_copies; ++i)
      if (written[src[i]]) return fail(HS_ERR_INVALID_ARG, "slot %d is a source and a destination", src[i]);
  } catch (const std::bad_alloc&) {
    return fail(HS_ERR_INTERNAL, "out of host memory");
  }
  return run(ctx, cu_budget, stream, n_copies == 0, HS_KERNEL_CACHE_COPY, [&](hipStream_t s) {
    const int64_t position_bytes = 2 * int64_t(head_dim);
    CacheCopyArgs a{};
    a.heads = n_kv_heads;
    a.dh = head_dim;
    a.head_bytes = kv->max_ctx * position_bytes;
    for (int32_t i = 0; i < n_copies;) {
      a.n_copies = 0;
      a.segments = 0;
      for (; i < n_copies && a.n_copies < kCopyList; ++i) {
        const int64_t n = positions ? (int64_t(positions[i]) + 31) / 32 * 32 : kv->max_ctx;
        if (n == 0) continue;
        CacheCopyArgs::Copy& c = a.copies[a.n_copies];
        c.src = src[i];
        c.dst = dst[i];
        c.tiles = int32_t(n / 32);
        c.first = a.segments;
        const int32_t more = copy_segments(c.tiles, head_dim);
        if (a.n_copies > 0 && (int64_t(a.segments) + more) * n_kv_heads > kMaxBlocks) break;  // of the next launch
        a.segments += more;
        ++a.n_copies;
      }
      for (int32_t l = 0; l < n_layers; l += kCopyLayers) {
        a.layers = std::min(n_layers - l, kCopyLayers);
        for (int32_t j = 0; j < a.layers; ++j) {
          a.k[j] = static_cast<uint16_t*>(kv->k[l + j]);
          a.v[j] = static_cast<uint16_t*>(kv->v[l + j]);
        }
        const hipError_t e = launch_cache_copy(a, cu_budget, s);
        if (e != hipSuccess) return e;
      }
    }
    return hipSuccess;
  });
}

hs_status hs_prefix_attention_workspace_size(int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim, int32_t n_seqs,
                                             int32_t max_prefix, int32_t max_rest, size_t* bytes) {
  clear_error();
  if (!bytes) return fail(HS_ERR_INVALID_ARG, "output pointer is null");
  HS_TRY(check_heads(n_kv_heads, head_dim));
  if (n_q_heads < 1 || n_q_heads % n_kv_heads != 0)
    return fail(HS_ERR_INVALID_ARG, "%d query heads on %d key/value heads", n_q_heads, n_kv_heads);
  if (n_q_heads / n_kv_heads > kPrefixMaxPerHead)
    return fail(HS_ERR_UNSUPPORTED, "%d query heads per key/value head: at most %d", n_q_heads / n_kv_heads,
                kPrefixMaxPerHead);
  if (n_seqs < 0 || max_prefix < 0 || max_rest < 0)
    return fail(HS_ERR_INVALID_ARG, "%d rows, prefixes up to %d and %d keys more", n_seqs, max_prefix, max_rest);
  if (int64_t(max_prefix) + max_rest > (int64_t(1) << 30) || n_q_heads > (1 << 16) ||
      int64_t(n_seqs) * n_q_heads > (int64_t(1) << 25))
    return fail(HS_ERR_UNSUPPORTED, "%d rows of %d heads over %d + %d keys", n_seqs, n_q_heads, max_prefix, max_rest);
  *bytes = prefix_workspace(n_seqs, max_prefix, max_rest, n_q_heads, n_kv_heads, head_dim);
  return HS_OK;
}

// Bytes of the partial states of one call on `cus` CUs (see prefix_shape).  Internal to
// the library and its tests (not declared in horizon.h).
uint64_t hs_prefix_attention_states(int32_t n_seqs, int32_t n_groups, int32_t max_prefix, int32_t max_rest, int32_t hq,
                                    int32_t hkv, int32_t dh, int32_t cus) {
  return prefix_states_bytes(prefix_shape(n_seqs, n_groups, max_prefix, max_rest, hq, hkv, cus), n_seqs, hq, dh);
}

hs_status hs_prefix_attention(hs_context* ctx, const void* q, int32_t type, int64_t ldq, void* out, int64_t ldo,
                              int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim, const void* k, const void* v,
                              int32_t n_slots, int32_t page_positions, const int32_t* block_table,
                              int32_t pages_per_seq, const int32_t* lens, int32_t n_seqs,
                              const int32_t* group_offsets, const int32_t* prefix_lens, int32_t n_groups,
                              int32_t max_prefix, int32_t max_rest, int32_t cu_budget, void* stream, void* workspace,
                              size_t ws_bytes) {
  size_t need = 0;
  HS_TRY(hs_prefix_attention_workspace_size(n_q_heads, n_kv_heads, head_dim, n_seqs, max_prefix, max_rest, &need));
  if (type != HS_TYPE_F16 && type != HS_TYPE_BF16) return fail(HS_ERR_INVALID_ARG, "q has type %d", type);
  HS_TRY(check_pages(n_slots, page_positions, n_kv_heads, head_dim));
  if (pages_per_seq < 1) return fail(HS_ERR_INVALID_ARG, "pages_per_seq %d must be >= 1", pages_per_seq);
  if (n_groups < 0) return fail(HS_ERR_INVALID_ARG, "n_groups %d < 0", n_groups);
  HS_TRY(check_rows(n_groups, 1 << 25));
  const int64_t cols = int64_t(n_q_heads) * head_dim;
  const int64_t cache = int64_t(n_slots) * page_positions * n_kv_heads * head_dim;
  const Span sq = rows_of("q", q, n_seqs, cols, ldq, 2), so = rows_of("out", out, n_seqs, cols, ldo, 2);
  const Span sk = {"k", k, uint64_t(cache) * 2}, sv = {"v", v, uint64_t(cache) * 2};
  const Span st = rows_of("block_table", block_table, n_seqs, pages_per_seq, pages_per_seq, 4);
  const Span sl = rows_of("lens", lens, n_seqs, 1, 1, 4);
  const Span sg = rows_of("group_offsets", group_offsets, n_groups ? int64_t(n_groups) + 1 : 0, 1, 1, 4);
  const Span sp = rows_of("prefix_lens", prefix_lens, n_groups, 1, 1, 4);
  const Span sws = {"workspace", workspace, need};
  HS_TRY(check_matrix(sq, n_seqs, cols, ldq, 2));
  HS_TRY(check_matrix(so, n_seqs, cols, ldo, 2));
  if (n_seqs > 0) {
    HS_TRY(check_aligned16("q", q));
    if (n_seqs > 1 && ldq % 8 != 0) return fail(HS_ERR_INVALID_ARG, "q: row stride %lld is not a multiple of 8", (long long)ldq);
    if (!k || !v) return fail(HS_ERR_INVALID_ARG, "the cache is null");
    HS_TRY(check_aligned16("k", k));
    HS_TRY(check_aligned16("v", v));
  }
  HS_TRY(check_matrix(st, n_seqs, 1, 1, 4));
  HS_TRY(check_matrix(sl, n_seqs, 1, 1, 4));
  HS_TRY(check_matrix(sg, n_groups, 1, 1, 4));
  HS_TRY(check_matrix(sp, n_groups, 1, 1, 4));
  for (const Span& written : {so, sws})
    for (const Span& in : {sq, sk, sv, st, sl, sg, sp}) HS_TRY(check_disjoint(written, in));
  HS_TRY(check_disjoint(so, sws));
  if (n_seqs) HS_TRY(check_workspace(workspace, ws_bytes, need));
  if (cu_budget < 1) return fail(HS_ERR_BUDGET, "CU budget %d", cu_budget);  // sizes the launch below
  const int32_t shared = n_groups ? max_prefix : 0;
  HS_TRY(check_prefix_launch(n_seqs, n_groups, shared, max_rest, n_q_heads, n_kv_heads, head_dim, cu_budget, need));
  PrefixArgs a{};
  a.q = q;
  a.type = type;
  a.ldq = ldq;
  a.out = out;
  a.ldo = ldo;
  a.k = static_cast<const uint16_t*>(k);
  a.v = static_cast<const uint16_t*>(v);
  a.n_slots = n_slots;
  a.page = page_positions;
  a.table = block_table;
  a.pages_per_seq = pages_per_seq;
  a.lens = lens;
  a.n_seqs = n_seqs;
  a.offsets = group_offsets;
  a.prefix = prefix_lens;
  a.n_groups = n_groups;
  a.max_prefix = shared;
  a.max_rest = max_rest;
  a.hq = n_q_heads;
  a.hkv = n_kv_heads;
  a.dh = head_dim;
  a.per_head_inv = prefix_inverse(n_q_heads / n_kv_heads);
  a.scale_log2 = 1.4426950408889634f / sqrtf(float(head_dim));
  a.part = workspace;
  return run(ctx, cu_budget, stream, n_seqs == 0, HS_KERNEL_PREFIX_ATTN,
             [&](hipStream_t s) { return launch_prefix_attention(a, cu_budget, s); });
}

}  // extern "C"
