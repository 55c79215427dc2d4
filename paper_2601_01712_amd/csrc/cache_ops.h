// The host side of the 8-bit cache's calls: entry points of cache_ops.hip, and what engine.hip needs of them.
#pragma once

#include <hip/hip_runtime.h>

#include "../../include/relaygr.h"
#include "kv_pool.h"

namespace relaygr {

// One relaygr_cache_attend on a stream: `scratch` holds the partial sums of rows that are cut along the keys (null: none are cut).
struct AttendCall {
  const relaygr_kv_rows* rows;
  int32_t layer, causal;
  const void* q;
  int64_t q_stride;
  void* out;
  int64_t out_stride;
  bool softmax;
  int n_cus;
  char* scratch;
  size_t scratch_bytes;
  uint32_t* arrived;      // kArrivals counters, zero; null: the call may not use them (its stream is under capture)
};
// Counters of pieces that have arrived (attend8.h), behind a context's packed weights.  A call leaves them as it found them, zero, and a context's calls
// follow one another on the GPU; replays of captured graphs are not the library's to order, so that captured calls join by a launch of their own.
constexpr int kArrivals = 4096;
// A user's K and V of one layer, as 16-bit tiles in scratch, on their way into its 8-bit entry.
struct TilesJob { int64_t page0; int32_t tiles; const void* src; };
int quantise_tiles(const KvPool* pool, int layer, const TilesJob* jobs, int n_jobs, hipStream_t st);
int attend8(KvPool* pool, const AttendCall& call, hipStream_t st);

}  // namespace relaygr
