// Argument checks and the launch of the stand-alone operators' entry points
// (internal to the library).
#pragma once

#include <hip/hip_runtime.h>

#include "context_call.h"
#include "plan.h"

namespace hs {
namespace {

constexpr int64_t kMaxStride = int64_t(1) << 30;  // elements between rows: byte extents stay below 2^63
constexpr int32_t kMaxRows = 1 << 30;             // rows plus a grid's stride stay below 2^31

size_t type_size(int32_t type) { return type == HS_TYPE_F32 ? 4 : 2; }

hs_status check_type(const char* what, int32_t type) {
  if (type != HS_TYPE_F32 && type != HS_TYPE_BF16 && type != HS_TYPE_F16)
    return fail(HS_ERR_INVALID_ARG, "%s has type %d", what, type);
  return HS_OK;
}

// Bytes [p, p + bytes) of one argument.
struct Span {
  const char* name;
  const void* p;
  uint64_t bytes;
};

Span rows_of(const char* name, const void* p, int64_t rows, int64_t cols, int64_t ld, size_t size) {
  return {name, p, rows < 1 ? 0 : (uint64_t(rows - 1) * uint64_t(ld) + uint64_t(cols)) * size};
}

hs_status check_rows(int32_t rows, int32_t most) {
  if (rows > most) return fail(HS_ERR_UNSUPPORTED, "%d rows: at most %d", rows, most);
  return HS_OK;
}

hs_status check_matrix(const Span& s, int64_t rows, int64_t cols, int64_t ld, size_t size) {
  if (rows > 0 && !s.p) return fail(HS_ERR_INVALID_ARG, "%s is null", s.name);
  if (ld < cols || ld > kMaxStride)
    return fail(HS_ERR_INVALID_ARG, "%s: row stride %lld outside [%lld, %lld]", s.name, (long long)ld,
                    (long long)cols, (long long)kMaxStride);
  if (reinterpret_cast<uintptr_t>(s.p) % size != 0)
    return fail(HS_ERR_INVALID_ARG, "%s is not aligned to its %zu-byte elements", s.name, size);
  return HS_OK;
}

hs_status check_disjoint(const Span& out, const Span& other) {
  if (!out.p || !other.p || !out.bytes || !other.bytes) return HS_OK;
  const uintptr_t a = reinterpret_cast<uintptr_t>(out.p), b = reinterpret_cast<uintptr_t>(other.p);
  if (a < b + other.bytes && b < a + out.bytes)
    return fail(HS_ERR_INVALID_ARG, "%s and %s overlap", out.name, other.name);
  return HS_OK;
}

#define HS_TRY(expr)                    \
  do {                                  \
    const hs_status st_ = (expr);       \
    if (st_ != HS_OK) return st_;       \
  } while (0)

template <typename F>
hs_status run(hs_context* ctx, int32_t cu_budget, void* stream, bool empty, int kind, F launch) {
  if (!ctx) return fail(HS_ERR_INVALID_ARG, "context is null");
  ContextCall call;
  HS_TRY(call.open(ctx, cu_budget, stream));
  if (empty) return HS_OK;
  call.timed_begin();
  const hipError_t e = launch(call.stream());
  if (e != hipSuccess) return fail(HS_ERR_HIP, "launch failed: %s", hipGetErrorString(e));
  call.timed_end(kind);
  return HS_OK;
}

}  // namespace
}  // namespace hs
