// What the calls on rows of a batch share on the host: the checks of their arguments, and the kernels' storage type and head size.
#pragma once

#include <type_traits>
#include <vector>

#include "../../include/relaygr.h"
#include "errors.h"
#include "gemm.h"
#include "kv_pool.h"

namespace relaygr {

// Rows of a [rows, d] array must be 16-byte aligned runs of d elements.
inline int check_rows_array(const char* what, const char* name, const void* base, int64_t stride, int d, int bytes = 2) {
  if (!base) return fail(RELAYGR_EINVAL, "%s: %s is null", what, name);
  if (((uintptr_t)base & 15) || stride % (16 / bytes)) return fail(RELAYGR_EINVAL, "%s: rows of %s are not 16-byte aligned", what, name);
  if (stride < d) return fail(RELAYGR_EINVAL, "%s: %s has a row stride of %lld elements, below d_model", what, name, (long long)stride);
  return RELAYGR_OK;
}

// The batch's entries, after the checks that all calls on an 8-bit pool share.
inline int resolve_rows(const char* what, KvPool* pool, int32_t layer, const relaygr_kv_rows* r, std::vector<PoolEntry>* entries) {
  if (!pool || !r) return fail(RELAYGR_EINVAL, "%s: null argument", what);
  if (!pool->q8) return fail(RELAYGR_EINVAL, "%s: the pool does not hold 8-bit K/V", what);
  if (layer < 0 || layer >= pool->cfg.n_layers) return fail(RELAYGR_EINVAL, "%s: layer %d out of range", what, layer);
  if (r->n_users < 0) return fail(RELAYGR_EINVAL, "%s: n_users < 0", what);
  if (r->row_off && r->row_off[0] != 0) return fail(RELAYGR_EINVAL, "%s: row offsets must start at 0", what);
  if (r->n_users == 0) return RELAYGR_OK;
  if (!r->handles || !r->row_off) return fail(RELAYGR_EINVAL, "%s: null handles or row offsets", what);
  for (int u = 0; u < r->n_users; ++u)
    if (r->row_off[u + 1] < r->row_off[u]) return fail(RELAYGR_EINVAL, "%s: row offsets not monotone at user %d", what, u);
  entries->resize(r->n_users);
  const int found = pool->resolve_all(r->handles, r->n_users, entries->data());
  if (found < r->n_users) return fail(RELAYGR_ENOENT, "%s: user %d: stale or unknown handle", what, found);
  return RELAYGR_OK;
}

// launch(storage type, d_head)
template <class F>
void by_head(const relaygr_model_config& cfg, F launch) {
  auto by_dh = [&](auto h) {
    switch (cfg.d_model / cfg.n_heads) {
      case 32: launch(h, std::integral_constant<int, 32>()); break;
      case 64: launch(h, std::integral_constant<int, 64>()); break;
      default: launch(h, std::integral_constant<int, 128>()); break;
    }
  };
  if (cfg.dtype == RELAYGR_DTYPE_FP16) by_dh(F16());
  else by_dh(Bf16());
}

}  // namespace relaygr
