// Launch interface of the kernels that answer from the residual stream: row
// quantisation, 8-bit products and log probabilities (internal to the library).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "answer_policy.h"

namespace hs {

struct QuantizeArgs {
  const void* x;          // [rows, d] of `type`, row stride ldx
  int type;               // HS_TYPE_*
  int64_t ldx;
  const uint16_t* gain;   // bf16 [d], or null: no RMSNorm
  float eps;
  int rows, d;
  int8_t* q;              // [rows, d], row stride ldq
  int64_t ldq;
  float* scale;           // [rows]
};
hipError_t launch_quantize(const QuantizeArgs& a, int cus, hipStream_t s);

struct LinearI8Args {
  const int8_t* a;        // [m, k], row stride lda
  int64_t lda;
  const float* a_scale;   // [m]
  const int8_t* w;        // [n, k], row stride ldw
  int64_t ldw;
  const float* w_scale;   // [n]
  const uint16_t* bias;   // bf16 [n] or null
  void* out;              // [m, n] of out_type, row stride ldo
  int out_type;           // HS_TYPE_*
  int64_t ldo;
  int m, n, k;
};
hipError_t launch_linear_i8(const LinearI8Args& a, int cus, hipStream_t s);

struct LogprobsArgs {
  const void* logits;     // [rows, vocab] of `type`, row stride ld
  int type;               // HS_TYPE_*
  int64_t ld;
  int rows, vocab;
  const int32_t* tokens;  // [rows, n_tokens] or null (n_tokens 0)
  int n_tokens;
  float* token_lp;        // [rows, n_tokens]
  float* entropy;         // [rows] or null
  int top_k;
  float* top_lp;          // [rows, top_k] (top_k > 0)
  int32_t* top_tokens;    // [rows, top_k]
  void* part;             // partial states, logprobs_workspace() bytes (null when that is 0)
};
hipError_t launch_logprobs(const LogprobsArgs& a, int cus, hipStream_t s);

}  // namespace hs
