// The host side of scored attention (scored8.h): its entry point is engine.hip's, which has the context's scratch.
#pragma once

#include "cache_ops.h"

namespace relaygr {

// An AttendCall with scores and masks of its own; weight_out null: tokens' weights are not asked for.
struct ScoredCall {
  AttendCall attend;
  const relaygr_scoring* scoring;
  const float* weight_in;
  float* weight_out;
};
int scored8(KvPool* pool, const ScoredCall& call, hipStream_t st);

}  // namespace relaygr
