// A compute call on a context's device and stream, for entry points outside
// runtime.cpp (internal to the library).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "horizon.h"

namespace hs {

class ContextCall {
 public:
  ContextCall() = default;
  ~ContextCall();  // the caller's current device again
  ContextCall(const ContextCall&) = delete;
  ContextCall& operator=(const ContextCall&) = delete;

  // Resolves the stream (null: the context's SHARED stream of the budget;
  // otherwise it must carry cu_budget CUs of the context's device) and makes
  // the context's device current.
  hs_status open(hs_context* ctx, int32_t cu_budget, void* stream);

  hipStream_t stream() const { return stream_; }

  // Brackets the launches of one kernel kind with the context's timing events.
  void timed_begin();
  void timed_end(int kind);

 private:
  hs_context* ctx_ = nullptr;
  hipStream_t stream_ = nullptr;
  hipEvent_t a_ = nullptr, b_ = nullptr;
  int device_ = -1;
};

}  // namespace hs
