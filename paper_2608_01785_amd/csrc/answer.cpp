// Entry points that answer from the residual stream: row quantisation with
// RMSNorm, 8-bit products, log probabilities.  Argument checks and launches.
#include <hip/hip_runtime.h>
#include <math.h>

#include "answer_kernels.h"
#include "call_checks.h"

using namespace hs;

namespace {

constexpr int32_t kLogprobsMaxRows = 1 << 25;     // a wavefront each: a grid holds fewer than 2^32 threads

}  // namespace

extern "C" {

hs_status hs_quantize_rows(hs_context* ctx, const void* x, int32_t x_type, int64_t ldx, const void* gain, float eps,
                           int32_t rows, int32_t d, void* q, int64_t ldq, float* scale, int32_t cu_budget,
                           void* stream) {
  hs::clear_error();
  HS_TRY(check_type("x", x_type));
  if (rows < 0 || d < 1) return hs::fail(HS_ERR_INVALID_ARG, "shape [%d, %d]", rows, d);
  HS_TRY(check_rows(rows, kMaxRows));
  const Span sx = rows_of("x", x, rows, d, ldx, type_size(x_type)), sq = rows_of("q", q, rows, d, ldq, 1);
  const Span ss = rows_of("scale", scale, rows, 1, 1, 4), sg = rows_of("gain", gain, 1, d, d, 2);
  HS_TRY(check_matrix(sx, rows, d, ldx, type_size(x_type)));
  HS_TRY(check_matrix(sq, rows, d, ldq, 1));
  HS_TRY(check_matrix(ss, rows, 1, 1, 4));
  if (gain) {
    HS_TRY(check_matrix(sg, 1, d, d, 2));
    if (!(eps > 0.0f) || !isfinite(eps)) return hs::fail(HS_ERR_INVALID_ARG, "eps %g must be positive", double(eps));
  }
  for (const Span& out : {sq, ss})
    for (const Span& in : {sx, sg}) HS_TRY(check_disjoint(out, in));
  HS_TRY(check_disjoint(sq, ss));
  hs::QuantizeArgs a{x, x_type, ldx, static_cast<const uint16_t*>(gain), eps, rows, d, static_cast<int8_t*>(q), ldq,
                     scale};
  return run(ctx, cu_budget, stream, rows == 0, HS_KERNEL_QUANTIZE,
             [&](hipStream_t s) { return hs::launch_quantize(a, cu_budget, s); });
}

hs_status hs_linear_i8(hs_context* ctx, const void* a, int64_t lda, const float* a_scale, const void* w, int64_t ldw,
                       const float* w_scale, const void* bias, void* out, int32_t out_type, int64_t ldo, int32_t m,
                       int32_t n, int32_t k, int32_t cu_budget, void* stream) {
  hs::clear_error();
  HS_TRY(check_type("out", out_type));
  if (m < 0 || n < 0 || k < 1) return hs::fail(HS_ERR_INVALID_ARG, "m %d, n %d, k %d", m, n, k);
  if (k > hs::kLinearI8MaxK)
    return hs::fail(HS_ERR_UNSUPPORTED, "k %d: 32-bit sums hold %d products", k, hs::kLinearI8MaxK);
  if (lda > hs::kLinearI8MaxStride || ldw > hs::kLinearI8MaxStride)
    return hs::fail(HS_ERR_UNSUPPORTED, "row strides %lld and %lld: operands allow %lld", (long long)lda,
                    (long long)ldw, (long long)hs::kLinearI8MaxStride);
  HS_TRY(check_rows(m, kMaxRows));
  HS_TRY(check_rows(n, kMaxRows));
  const size_t osz = type_size(out_type);
  const Span sa = rows_of("a", a, m, k, lda, 1), sw = rows_of("w", w, n, k, ldw, 1);
  const Span sas = rows_of("a_scale", a_scale, m, 1, 1, 4), sws = rows_of("w_scale", w_scale, n, 1, 1, 4);
  const Span sb = rows_of("bias", bias, n, 1, 1, 2), so = rows_of("out", out, n ? m : 0, n, ldo, osz);
  HS_TRY(check_matrix(sa, m, k, lda, 1));
  HS_TRY(check_matrix(sw, n, k, ldw, 1));
  HS_TRY(check_matrix(sas, m, 1, 1, 4));
  HS_TRY(check_matrix(sws, n, 1, 1, 4));
  if (bias) HS_TRY(check_matrix(sb, n, 1, 1, 2));
  HS_TRY(check_matrix(so, n ? m : 0, n, ldo, osz));
  for (const Span& in : {sa, sw, sas, sws, sb}) HS_TRY(check_disjoint(so, in));
  hs::LinearI8Args g{static_cast<const int8_t*>(a), lda, a_scale, static_cast<const int8_t*>(w), ldw, w_scale,
                     static_cast<const uint16_t*>(bias), out, out_type, ldo, m, n, k};
  return run(ctx, cu_budget, stream, m == 0 || n == 0, HS_KERNEL_LINEAR_I8,
             [&](hipStream_t s) { return hs::launch_linear_i8(g, cu_budget, s); });
}

// Which kernel hs_linear_i8 takes (see linear_i8_choice).  Internal to the library
// and its tests (not declared in horizon.h).
int32_t hs_linear_i8_kernel(int32_t m, int32_t n, int32_t k, int32_t cus, int32_t aligned) {
  return hs::linear_i8_choice(m, n, k, cus, aligned != 0);
}

// One 16-byte load of an aligned operand (see linear_i8_load): its vector and scalar
// byte offsets and the resource's bytes, as internal.
void hs_linear_i8_load(int32_t lane, int32_t l, int32_t stage, int32_t span, int64_t ld, int32_t k, uint32_t out[3]) {
  const hs::LinearI8Load at = hs::linear_i8_load(hs::linear_i8_offset(lane, ld), lane, l, stage, ld, k);
  out[0] = at.vector;
  out[1] = at.scalar;
  out[2] = hs::linear_i8_records(span, ld, k);
}

// The blocks a row is split over by hs_logprobs (see logprobs_shape), as internal.
int32_t hs_logprobs_splits(int32_t rows, int32_t vocab, int32_t elem_bytes, int32_t cus) {
  return hs::logprobs_shape(rows, vocab, elem_bytes, cus).splits;
}

hs_status hs_logprobs_workspace_size(int32_t max_rows, int32_t vocab, int32_t top_k, size_t* bytes) {
  hs::clear_error();
  if (!bytes) return hs::fail(HS_ERR_INVALID_ARG, "output pointer is null");
  if (max_rows < 0 || vocab < 1) return hs::fail(HS_ERR_INVALID_ARG, "shape [%d, %d]", max_rows, vocab);
  if (top_k < 0 || top_k > hs::kLogprobsMaxTop)
    return hs::fail(HS_ERR_UNSUPPORTED, "top_k %d outside [0, %d]", top_k, hs::kLogprobsMaxTop);
  HS_TRY(check_rows(max_rows, kLogprobsMaxRows));
  *bytes = hs::logprobs_workspace(max_rows, vocab, top_k);
  return HS_OK;
}

hs_status hs_logprobs(hs_context* ctx, const void* logits, int32_t type, int64_t ld, int32_t rows, int32_t vocab,
                      const int32_t* tokens, int32_t n_tokens, float* token_logprobs, float* entropy, int32_t top_k,
                      float* top_logprobs, int32_t* top_tokens, int32_t cu_budget, void* stream, void* workspace,
                      size_t ws_bytes) {
  size_t need = 0;
  HS_TRY(hs_logprobs_workspace_size(rows, vocab, top_k, &need));  // the shape's checks
  HS_TRY(check_type("logits", type));
  if (n_tokens < 0) return hs::fail(HS_ERR_INVALID_ARG, "n_tokens %d < 0", n_tokens);
  const int32_t token_rows = n_tokens ? rows : 0, top_rows = top_k ? rows : 0;
  const Span sz = rows_of("logits", logits, rows, vocab, ld, type_size(type));
  const Span st = rows_of("tokens", tokens, token_rows, n_tokens, n_tokens, 4);
  const Span sl = rows_of("token_logprobs", token_logprobs, token_rows, n_tokens, n_tokens, 4);
  const Span se = rows_of("entropy", entropy, rows, 1, 1, 4);
  const Span sv = rows_of("top_logprobs", top_logprobs, top_rows, top_k, top_k, 4);
  const Span si = rows_of("top_tokens", top_tokens, top_rows, top_k, top_k, 4);
  const Span sws = {"workspace", workspace, need};
  HS_TRY(check_matrix(sz, rows, vocab, ld, type_size(type)));
  HS_TRY(check_matrix(st, token_rows, n_tokens, n_tokens, 4));
  HS_TRY(check_matrix(sl, token_rows, n_tokens, n_tokens, 4));
  if (entropy) HS_TRY(check_matrix(se, rows, 1, 1, 4));
  HS_TRY(check_matrix(sv, top_rows, top_k, top_k, 4));
  HS_TRY(check_matrix(si, top_rows, top_k, top_k, 4));
  const Span outs[] = {sl, se, sv, si, sws};
  for (const Span& out : outs)
    for (const Span& in : {sz, st}) HS_TRY(check_disjoint(out, in));
  for (const Span& out : outs)
    for (const Span& other : outs)
      if (&other > &out) HS_TRY(check_disjoint(out, other));
  if (need) {
    if (!workspace) return hs::fail(HS_ERR_WORKSPACE, "workspace is null");
    if (reinterpret_cast<uintptr_t>(workspace) % 16 != 0)
      return hs::fail(HS_ERR_INVALID_ARG, "workspace is not aligned to 16 bytes");
    if (ws_bytes < need) return hs::fail(HS_ERR_WORKSPACE, "workspace has %zu bytes, %zu needed", ws_bytes, need);
  }
  hs::LogprobsArgs a{logits,  type,  ld,           rows,       vocab, tokens, n_tokens, token_logprobs,
                     entropy, top_k, top_logprobs, top_tokens, workspace};
  return run(ctx, cu_budget, stream, rows == 0, HS_KERNEL_LOGPROBS,
             [&](hipStream_t s) { return hs::launch_logprobs(a, cu_budget, s); });
}

}  // extern "C"
