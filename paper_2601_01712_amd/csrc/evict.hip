// C-ABI entry point of eviction from the 8-bit K/V cache (evict8.h).
#include <algorithm>
#include <vector>

#include "cache_rows.h"
#include "evict8.h"

using namespace relaygr;

namespace {

const char* const what = "kv_pool_evict";

// A user's piece of an array.  Outputs may share memory with nothing but their user's own input, from its first element on.
struct Span { uintptr_t from, to; int user; bool out; };
bool apart(std::vector<Span>& x) {
  std::sort(x.begin(), x.end(), [](const Span& a, const Span& b) { return a.from < b.from; });
  Span in = {0, 0, -1, false}, out = in;      // of the spans so far, those that end last
  bool shared = false, reused = false;        // inputs that overlap; outputs over an input
  for (const Span& s : x) {
    if (s.from == s.to) continue;
    const bool in_it = s.from < in.to, out_of_it = s.from < out.to;
    if (s.out) {
      if (out_of_it || (in_it && (s.user != in.user || s.from != in.from))) return false;
      reused = reused || in_it;
      out = s;
    } else {
      if (out_of_it && (s.user != out.user || s.from != out.from)) return false;
      reused = reused || out_of_it;
      shared = shared || in_it;
      if (s.to > in.to) in = s;
    }
  }
  return !(shared && reused);
}

int evict(KvPool* pool, const relaygr_kv_rows* r, const relaygr_kv_eviction* e, hipStream_t st) {
  std::vector<PoolEntry> from, to;
  int rc = resolve_rows(what, pool, 0, r, &from);
  if (rc != RELAYGR_OK) return rc;
  if (!e) return fail(RELAYGR_EINVAL, "%s: null argument", what);
  if (e->first < 0 || e->recent < 0) return fail(RELAYGR_EINVAL, "%s: first or recent < 0", what);
  const struct { const char* name; const void* p; } arrays[] = {{"weight", e->weight}, {"kept", e->kept}, {"weight_out", e->weight_out}, {"position", e->position},
                                                                {"position_out", e->position_out}};
  for (const auto& x : arrays)
    if ((uintptr_t)x.p & 3) return fail(RELAYGR_EINVAL, "%s: %s is not 4-byte aligned", what, x.name);
  if (e->position_out && !e->position) return fail(RELAYGR_EINVAL, "%s: position_out without position", what);
  if (r->n_users == 0) return RELAYGR_OK;
  const relaygr_model_config& cfg = pool->cfg;
  to = from;
  if (e->to) {
    to.resize(r->n_users);
    const int found = pool->resolve_all(e->to, r->n_users, to.data());
    if (found < r->n_users) return fail(RELAYGR_ENOENT, "%s: user %d: stale or unknown handle to move to", what, found);
  }
  const int64_t of_group = (int64_t)cfg.n_layers * cfg.n_heads * 2, most = ((1ll << 32) - 1) / (kMoveWaves * 64) / of_group;     // groups of a launch
  if (most == 0) return fail(RELAYGR_EINVAL, "%s: %d layers are more than a launch takes", what, cfg.n_layers);
  int32_t too_many = 0;
  bool any = false, in_place = false;
  for (int u = 0; u < r->n_users; ++u) in_place = in_place || (from[u].page0 == to[u].page0 && r->row_off[u + 1] > r->row_off[u]);
  std::vector<int64_t> written, read;       // first pages
  std::vector<Span> spans[2];               // of weights and positions
  for (int u = 0; u < r->n_users; ++u) {
    const int32_t len = r->key_len ? r->key_len[u] : from[u].prefix_len, keep = r->row_off[u + 1] - r->row_off[u];
    if (len < 0 || len > from[u].prefix_len) return fail(RELAYGR_EINVAL, "%s: user %d: %d tokens of an entry of %d", what, u, len, from[u].prefix_len);
    if (keep > len) return fail(RELAYGR_EINVAL, "%s: user %d: %d of %d tokens cannot stay", what, u, keep, len);
    if (keep > to[u].prefix_len) return fail(RELAYGR_EINVAL, "%s: user %d: %d tokens into an entry of %d", what, u, keep, to[u].prefix_len);
    if (keep == 0) continue;
    if (keep < len && (int64_t)e->first + e->recent > keep)
      return fail(RELAYGR_EINVAL, "%s: user %d: the first %d and the last %d tokens are more than %d", what, u, e->first, e->recent, keep);
    if (e->token_off && e->token_off[u] < 0) return fail(RELAYGR_EINVAL, "%s: user %d: token offset %lld", what, u, (long long)e->token_off[u]);
    if (e->out_off && e->out_off[u] < 0) return fail(RELAYGR_EINVAL, "%s: user %d: output offset %lld", what, u, (long long)e->out_off[u]);
    any = true;
    written.push_back(to[u].page0);
    if (from[u].page0 != to[u].page0) read.push_back(from[u].page0);
    const int64_t in = e->token_off ? e->token_off[u] : 0, o = e->out_off ? e->out_off[u] : r->row_off[u];
    const uintptr_t ins[2] = {(uintptr_t)e->weight, (uintptr_t)e->position}, outs[2] = {(uintptr_t)e->weight_out, (uintptr_t)e->position_out};
    for (int i = 0; i < 2; ++i) {
      if (!outs[i]) continue;
      spans[i].push_back({ins[i] + 4 * in, ins[i] + 4 * (in + len), u, false});
      spans[i].push_back({outs[i] + 4 * o, outs[i] + 4 * (o + keep), u, true});
    }
    if (!in_place && ((int64_t)keep + kTile * kMoveWaves - 1) / (kTile * kMoveWaves) > most) too_many = keep;
  }
  if (!any) return RELAYGR_OK;
  if (!e->weight || !e->kept || !e->token_off) return fail(RELAYGR_EINVAL, "%s: null weight, kept or token_off", what);
  // an entry that two users write, or one writes and another reads, would be a race
  std::sort(written.begin(), written.end());
  if (std::adjacent_find(written.begin(), written.end()) != written.end()) return fail(RELAYGR_EINVAL, "%s: two users move into one entry", what);
  for (int64_t x : read)
    if (std::binary_search(written.begin(), written.end(), x)) return fail(RELAYGR_EINVAL, "%s: an entry is moved out of and into by different users", what);
  for (auto& x : spans)
    if (!apart(x)) return fail(RELAYGR_EINVAL, "%s: outputs overlap each other, or inputs elsewhere than from a user's own first token on", what);
  if (too_many) return fail(RELAYGR_EINVAL, "%s: %d tokens are more than a launch takes", what, too_many);

  (void)hipGetLastError();
  EvictParams p = {};
  p.weight = e->weight; p.position = e->position; p.weight_out = e->weight_out; p.position_out = e->position_out; p.kept = e->kept;
  p.slab = (char*)pool->slab; p.page_bytes = (int64_t)pool->page_bytes; p.tile_stride = pool->tile_stride; p.layer_stride = pool->layer_stride;
  p.scales_off = q8_scales_off(cfg, 0);
  p.n_layers = cfg.n_layers; p.n_heads = cfg.n_heads; p.first = e->first; p.recent = e->recent; p.in_place = in_place ? 1 : 0;
  for (int u = 0; u < r->n_users;) {
    p.n_users = 0; p.n_units = 0;
    for (; u < r->n_users && p.n_users < kEvictUsers; ++u) {
      const int32_t len = r->key_len ? r->key_len[u] : from[u].prefix_len, keep = r->row_off[u + 1] - r->row_off[u];
      if (keep == 0) continue;
      const int64_t groups = in_place ? 1 : ((int64_t)keep + kTile * kMoveWaves - 1) / (kTile * kMoveWaves);
      if (p.n_units + groups > most) break;
      p.users[p.n_users++] = {(int32_t)from[u].page0, (int32_t)to[u].page0, len, keep, r->row_off[u], p.n_units, e->token_off[u],
                              e->out_off ? e->out_off[u] : (int64_t)r->row_off[u]};
      p.n_units += (int32_t)groups;
    }
    if (p.n_users == 0) break;
    hipLaunchKernelGGL(evict_choose_kernel, dim3((unsigned)p.n_users), dim3(kChooseThreads), 0, st, p);
    by_head(cfg, [&](auto h, auto dim) {
      using HT = decltype(h);
      constexpr int DH = decltype(dim)::value, WIDE = kWideWaves<DH>;
      const dim3 grid((unsigned)(p.n_units * of_group));
      if (in_place && grid.x <= kWideGroups) hipLaunchKernelGGL((evict_move_kernel<HT, DH, WIDE>), grid, dim3(WIDE * 64), 0, st, p);
      else hipLaunchKernelGGL((evict_move_kernel<HT, DH, kMoveWaves>), grid, dim3(kMoveWaves * 64), 0, st, p);
    });
    hipError_t err = hipGetLastError();
    if (err != hipSuccess) return fail(RELAYGR_EHIP, "launch %s: %s", what, hipGetErrorString(err));
  }
  return RELAYGR_OK;
}

}  // namespace

extern "C" int relaygr_kv_pool_evict(relaygr_kv_pool* pool, const relaygr_kv_rows* rows, const relaygr_kv_eviction* eviction, void* hip_stream) {
  try {
    return evict(reinterpret_cast<KvPool*>(pool), rows, eviction, (hipStream_t)hip_stream);
  } catch (...) {
    return fail(RELAYGR_EINVAL, "%s: out of host memory", what);
  }
}
