// C-ABI entry points of the 8-bit K/V cache (kv8.h, attend8.h): writing rows, reading them back, and the planning and launches of
// attention over them, whose entry point is engine.hip's (it takes a context's scratch).
#include "cache_ops.h"

#include <algorithm>
#include <cmath>
#include <vector>

#include "attend8.h"
#include "attend_rules.h"
#include "errors.h"
#include "kv8.h"

using namespace relaygr;

#define LAUNCH_CHECK(name)                                                                     \
  do {                                                                                         \
    hipError_t e_ = hipGetLastError();                                                         \
    if (e_ != hipSuccess) return fail(RELAYGR_EHIP, "launch %s: %s", name, hipGetErrorString(e_)); \
  } while (0)

namespace {

// Rows of a [rows, d] array must be 16-byte aligned runs of d elements.
int check_rows_array(const char* what, const char* name, const void* base, int64_t stride, int d) {
  if (!base) return fail(RELAYGR_EINVAL, "%s: %s is null", what, name);
  if (((uintptr_t)base & 15) || stride % 8) return fail(RELAYGR_EINVAL, "%s: rows of %s are not 16-byte aligned", what, name);
  if (stride < d) return fail(RELAYGR_EINVAL, "%s: %s has a row stride of %lld elements, below d_model", what, name, (long long)stride);
  return RELAYGR_OK;
}

// The batch's entries, after the checks that all three calls share.
int resolve_rows(const char* what, KvPool* pool, int32_t layer, const relaygr_kv_rows* r, std::vector<PoolEntry>* entries) {
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

// once: rows and codes are more than the caches hold.
template <bool WRITE, int USERS>
int launch_rows(const char* what, const KvPool* pool, int layer, const relaygr_kv_rows* r, const std::vector<PoolEntry>& entries, void* k, int64_t k_stride,
                void* v, int64_t v_stride, bool once, hipStream_t st) {
  const relaygr_model_config& cfg = pool->cfg;
  RowsParams<USERS> p = {};
  p.k = k; p.v = v; p.k_stride = k_stride; p.v_stride = v_stride;
  p.slab = (char*)pool->slab; p.page_bytes = (int64_t)pool->page_bytes; p.tile_stride = pool->tile_stride;
  p.codes_off = layer * pool->layer_stride;
  p.scales_off = q8_scales_off(cfg, layer);
  p.d = cfg.d_model;
  for (int u = 0; u < r->n_users;) {
    p.n_users = 0; p.n_tiles = 0;
    for (; u < r->n_users && p.n_users < USERS; ++u) {
      const int32_t first = r->first_token ? r->first_token[u] : 0, n = r->row_off[u + 1] - r->row_off[u];
      if (n == 0) continue;
      p.users[p.n_users++] = {(int32_t)entries[u].page0, first, n, r->row_off[u], p.n_tiles};
      p.n_tiles += (int)(((int64_t)first + n - 1) / kTile - first / kTile + 1);
    }
    if (p.n_users == 0) break;
    by_head(cfg, [&](auto h, auto dim) {
      using H = decltype(h);
      constexpr int DH = decltype(dim)::value, FW = DH < 64 ? 64 : DH;      // (runs of 128 bytes of a row at least)
      const dim3 grid((unsigned)(((int64_t)p.n_tiles * (cfg.d_model / FW) * 2 + 3) / 4));
      auto go = [&](auto once) {
        constexpr bool ONCE = decltype(once)::value;
        if (WRITE) hipLaunchKernelGGL((kv8_write_kernel<H, DH, FW, ONCE, USERS>), grid, dim3(256), 0, st, p);
        else hipLaunchKernelGGL((kv8_read_kernel<H, DH, FW, ONCE, USERS>), grid, dim3(256), 0, st, p);
      };
      if constexpr (USERS > kFewRowUsers) {
        if (once) { go(std::true_type()); return; }
      }
      go(std::false_type());
    });
    LAUNCH_CHECK(what);
  }
  return RELAYGR_OK;
}

template <bool WRITE>
int move_rows(const char* what, KvPool* pool, int32_t layer, const relaygr_kv_rows* r, void* k, int64_t k_stride, void* v, int64_t v_stride, hipStream_t st) {
  std::vector<PoolEntry> entries;
  int rc = resolve_rows(what, pool, layer, r, &entries);
  if (rc != RELAYGR_OK || r->n_users == 0) return rc;
  for (int u = 0; u < r->n_users; ++u) {
    const int64_t first = r->first_token ? r->first_token[u] : 0, n = r->row_off[u + 1] - r->row_off[u];
    if (first < 0 || first + n > entries[u].prefix_len)
      return fail(RELAYGR_EINVAL, "%s: user %d: tokens %lld to %lld of an entry of %d", what, u, (long long)first, (long long)(first + n), entries[u].prefix_len);
  }
  if (r->row_off[r->n_users] == 0) return RELAYGR_OK;
  const relaygr_model_config& cfg = pool->cfg;
  if ((rc = check_rows_array(what, "k", k, k_stride, cfg.d_model)) != RELAYGR_OK) return rc;
  if ((rc = check_rows_array(what, "v", v, v_stride, cfg.d_model)) != RELAYGR_OK) return rc;
  if (WRITE && r->n_users > 1) {   // two users writing one entry would race
    std::vector<relaygr_kv_handle> hs;
    hs.reserve(r->n_users);
    for (int u = 0; u < r->n_users; ++u) if (r->row_off[u + 1] > r->row_off[u]) hs.push_back(r->handles[u]);
    std::sort(hs.begin(), hs.end());
    if (std::adjacent_find(hs.begin(), hs.end()) != hs.end()) return fail(RELAYGR_EINVAL, "%s: two users of the batch carry the same handle", what);
  }
  (void)hipGetLastError();   // a failure the caller's own HIP calls left behind is not this call's
  // (us without / with the hint to leave nothing in the caches, write and read, d = 256, 64 users of 4096 tokens, 402 MB: 78.2 / 65.9, 76.8 / 72.6; d = 512, 64 of 3600,
  // 708 MB: 141 / 145, 142 / 133; d = 1024, 16 of 4096: 78.9 / 69.9, 82.3 / 74.3; 16 of 1000, 49 MB: 10.7 / 11.4, 10.4 / 9.9)
  const bool once = (int64_t)r->row_off[r->n_users] * cfg.d_model * 6 >= kOnceBytes;
  if (r->n_users <= kFewRowUsers && !once) return launch_rows<WRITE, kFewRowUsers>(what, pool, layer, r, entries, k, k_stride, v, v_stride, once, st);
  return launch_rows<WRITE, kRowUsers>(what, pool, layer, r, entries, k, k_stride, v, v_stride, once, st);
}

template <typename H, int DH, bool SM, int USERS>
void launch_attend(const AttendParams<USERS>& p, int blocks, bool once, hipStream_t st) {
  const dim3 grid((unsigned)attend_groups(p.n_items, p.n_heads)), block(kAttendWaves * 64);
  if constexpr (USERS > kFewAttendUsers) {
    if constexpr (DH == 64) {
      if (blocks == 2) { hipLaunchKernelGGL((attend8_kernel<H, DH, 2, SM, false, USERS>), grid, block, 0, st, p); return; }
    }
    if (once) { hipLaunchKernelGGL((attend8_kernel<H, DH, 1, SM, true, USERS>), grid, block, 0, st, p); return; }
  }
  hipLaunchKernelGGL((attend8_kernel<H, DH, 1, SM, false, USERS>), grid, block, 0, st, p);
}

}  // namespace

int relaygr::quantise_tiles(const KvPool* pool, int layer, const TilesJob* jobs, int n_jobs, hipStream_t st) {
  const relaygr_model_config& cfg = pool->cfg;
  const int d = cfg.d_model;
  TilesParams p = {};
  p.tile_stride = pool->tile_stride; p.src_stride = (int64_t)2 * kTile * d;
  p.codes_off = layer * pool->layer_stride; p.scales_off = q8_scales_off(cfg, layer); p.n_heads = cfg.n_heads;
  for (int j = 0; j < n_jobs;) {
    p.n_users = 0; p.n_tiles = 0;
    for (; j < n_jobs && p.n_users < kTilesUsers; ++j) {
      p.users[p.n_users++] = {(char*)pool->slab + (size_t)jobs[j].page0 * pool->page_bytes, (const uint16_t*)jobs[j].src, p.n_tiles, 0};
      p.n_tiles += jobs[j].tiles;
    }
    const dim3 grid((unsigned)(((int64_t)p.n_tiles * cfg.n_heads * 2 + 3) / 4));
    by_head(cfg, [&](auto h, auto dim) { hipLaunchKernelGGL((kv8_tiles_kernel<decltype(h), decltype(dim)::value>), grid, dim3(256), 0, st, p); });
    LAUNCH_CHECK("kv8_tiles");
  }
  return RELAYGR_OK;
}

int relaygr::attend8(KvPool* pool, const AttendCall& c, hipStream_t st) {
  static const char* what = "cache_attend";
  std::vector<PoolEntry> entries;
  const relaygr_kv_rows* r = c.rows;
  int rc = resolve_rows(what, pool, c.layer, r, &entries);
  if (rc != RELAYGR_OK || r->n_users == 0) return rc;
  const relaygr_model_config& cfg = pool->cfg;
  const int d = cfg.d_model, H = cfg.n_heads, dh = d / H;
  struct Work { int user, rows, keys, parts, per; };
  std::vector<Work> work;
  std::vector<AttendLen> lens;
  for (int u = 0; u < r->n_users; ++u) {
    const int keys = r->key_len ? r->key_len[u] : entries[u].prefix_len, n = r->row_off[u + 1] - r->row_off[u];
    if (keys < 0 || keys > entries[u].prefix_len) return fail(RELAYGR_EINVAL, "%s: user %d: %d keys of an entry of %d tokens", what, u, keys, entries[u].prefix_len);
    if (n == 0) continue;
    work.push_back({u, n, keys, 1, 0});
    lens.push_back({n, keys});
  }
  if (work.empty()) return RELAYGR_OK;
  if ((rc = check_rows_array(what, "q", c.q, c.q_stride, d)) != RELAYGR_OK) return rc;
  if ((rc = check_rows_array(what, "out", c.out, c.out_stride, d)) != RELAYGR_OK) return rc;

  AttendRule rule = attend_rule(lens, H, dh, c.n_cus);
  if (!c.scratch) rule.piece = 0;
  const int blocks = rule.blocks, item_rows = 32 * blocks;
  const bool once = rule.once;
  const size_t row_bytes = (size_t)d * 4 + (c.softmax ? (size_t)H * 8 : 0);
  const auto items_of = [&](const Work& w) { return ((int64_t)w.rows + item_rows - 1) / item_rows * w.parts; };
  int64_t partial_rows, most_items;
  int most_sums;      // rows of an item times its pieces
  for (;; rule.piece = rule.piece > 1 << 20 ? 0 : 2 * rule.piece) {      // (0: nothing is cut)
    partial_rows = most_items = 0;
    most_sums = 0;
    for (Work& w : work) {
      const int nk = (w.keys + kTile - 1) / kTile;
      w.parts = attend_parts(nk, rule.piece);
      w.per = std::max(1, (nk + w.parts - 1) / w.parts);
      if (w.parts > 1) partial_rows += (int64_t)w.parts * w.rows;
      most_sums = std::max(most_sums, std::min(w.rows, item_rows) * w.parts);
      most_items = std::max(most_items, items_of(w));
    }
    if (partial_rows == 0 || ((size_t)partial_rows * row_bytes <= c.scratch_bytes && partial_rows < (1ll << 31) && attend_fits(most_items, H))) break;
  }
  if (!attend_fits(most_items, H)) return fail(RELAYGR_EINVAL, "%s: %lld row tiles of one user are more than a launch takes", what, (long long)most_items);
  std::stable_sort(work.begin(), work.end(), [](const Work& a, const Work& b) { return a.per > b.per; });    // the longest pieces first

  (void)hipGetLastError();
  float *part = (float*)c.scratch, *ml = (float*)(c.scratch + (size_t)partial_rows * d * 4);
  int32_t part0 = 0;
  auto launch = [&](auto users) -> int {
    constexpr int USERS = decltype(users)::value;
    AttendParams<USERS> p = {};
    JoinParams<USERS> j = {};
    p.q = (const uint16_t*)c.q; p.out = (uint16_t*)c.out; p.q_stride = c.q_stride; p.out_stride = c.out_stride;
    p.slab = (const char*)pool->slab + c.layer * pool->layer_stride;
    p.page_bytes = (int64_t)pool->page_bytes; p.tile_stride = pool->tile_stride;
    p.scales_off = q8_scales_off(cfg, c.layer) - c.layer * pool->layer_stride;
    p.part = part; p.ml = ml;
    p.d = d; p.n_heads = H; p.causal = c.causal ? 1 : 0;
    p.score_mul = 1.4426950408889634f / sqrtf((float)dh);
    j.out = p.out; j.out_stride = p.out_stride; j.part = part; j.ml = ml; j.d = d; j.n_heads = H; j.causal = p.causal;
    for (size_t i = 0; i < work.size();) {
      p.n_users = 0; p.n_items = 0; j.n_users = 0; j.n_rows = 0;
      for (; i < work.size() && p.n_users < USERS; ++i) {
        const Work& w = work[i];
        if (!attend_fits(p.n_items + items_of(w), H)) break;      // (never a launch's first)
        const int32_t row0 = r->row_off[w.user];
        p.users[p.n_users++] = {(int32_t)entries[w.user].page0, row0, w.rows, w.keys, p.n_items, part0, (uint32_t)w.parts | (uint32_t)w.per << 7};
        p.n_items += (int32_t)items_of(w);
        if (w.parts == 1) continue;
        j.users[j.n_users++] = {row0, w.rows, w.keys, part0, w.parts, j.n_rows};
        j.n_rows += w.rows;
        part0 += w.parts * w.rows;
      }
      p.arrived = USERS == kFewAttendUsers && attend_joins_itself(most_sums, (int64_t)p.n_items * H, kArrivals) ? c.arrived : nullptr;
      by_head(cfg, [&](auto h, auto dim) {
        using HT = decltype(h);
        constexpr int DH = decltype(dim)::value;
        if (c.softmax) launch_attend<HT, DH, true>(p, blocks, once, st);
        else launch_attend<HT, DH, false>(p, blocks, once, st);
        if (j.n_users == 0 || p.arrived) return;
        const dim3 grid((unsigned)(((int64_t)j.n_rows * std::max(1, d / 256) + 3) / 4));
        if (c.softmax) hipLaunchKernelGGL((attend8_join_kernel<HT, DH, true, USERS>), grid, dim3(256), 0, st, j);
        else hipLaunchKernelGGL((attend8_join_kernel<HT, DH, false, USERS>), grid, dim3(256), 0, st, j);
      });
      LAUNCH_CHECK(what);
    }
    return RELAYGR_OK;
  };
  if ((int)work.size() <= kFewAttendUsers && blocks == 1 && !once) return launch(std::integral_constant<int, kFewAttendUsers>());
  return launch(std::integral_constant<int, kAttendUsers>());
}

// (the planning allocates host memory: running out of it is an error code of the call)
#define NO_THROW(expr)                                                                          \
  try {                                                                                         \
    return expr;                                                                                \
  } catch (...) {                                                                               \
    return fail(RELAYGR_EINVAL, "out of host memory");                                          \
  }

extern "C" int relaygr_kv_pool_write(relaygr_kv_pool* pool, int32_t layer, const relaygr_kv_rows* rows, const void* k, int64_t k_stride,
                                     const void* v, int64_t v_stride, void* hip_stream) {
  NO_THROW(move_rows<true>("kv_pool_write", reinterpret_cast<KvPool*>(pool), layer, rows, const_cast<void*>(k), k_stride, const_cast<void*>(v), v_stride,
                           (hipStream_t)hip_stream))
}

extern "C" int relaygr_kv_pool_read(relaygr_kv_pool* pool, int32_t layer, const relaygr_kv_rows* rows, void* k, int64_t k_stride, void* v,
                                    int64_t v_stride, void* hip_stream) {
  NO_THROW(move_rows<false>("kv_pool_read", reinterpret_cast<KvPool*>(pool), layer, rows, k, k_stride, v, v_stride, (hipStream_t)hip_stream))
}
