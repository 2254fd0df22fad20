// Host rules of the answering kernels (plain C++).
#pragma once

#include <stddef.h>
#include <stdint.h>

namespace hs {

constexpr int kLogprobsMaxTop = 64;       // alternatives a row can list: one per lane of a wavefront
constexpr int kLinearI8MaxK = 131071;     // (-128)^2 k stays below 2^31

// Workspace bytes of hs_logprobs, on any budget.
inline size_t logprobs_workspace(int64_t rows, int64_t vocab, int top_k) {
  (void)rows;
  (void)vocab;
  (void)top_k;
  return 0;
}

}  // namespace hs
