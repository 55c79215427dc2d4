// Planning and launches of scored attention (scored8.h).
#include "scored_ops.h"

#include <algorithm>
#include <cmath>
#include <vector>

#include "attend_rules.h"
#include "cache_rows.h"
#include "errors.h"
#include "scored8.h"

using namespace relaygr;

#define LAUNCH_CHECK(name)                                                                     \
  do {                                                                                         \
    hipError_t e_ = hipGetLastError();                                                         \
    if (e_ != hipSuccess) return fail(RELAYGR_EHIP, "launch %s: %s", name, hipGetErrorString(e_)); \
  } while (0)

namespace {

const char* const what = "cache_attend_scored";

int check_words(const char* name, const void* p) {
  if ((uintptr_t)p & 3) return fail(RELAYGR_EINVAL, "%s: %s is not 4-byte aligned", what, name);
  return RELAYGR_OK;
}

int check_scoring(const relaygr_kv_rows* r, const relaygr_scoring& s, const float* weight_in, const float* weight_out) {
  // (beyond these, the factors of a capped score leave fp32's range)
  if (!(s.cap == 0 || (s.cap >= 0x1p-100f && s.cap <= 0x1p100f))) return fail(RELAYGR_EINVAL, "%s: a cap of %g is neither 0 nor between 2^-100 and 2^100", what, s.cap);
  if (s.window < 0) return fail(RELAYGR_EINVAL, "%s: window < 0", what);
  int rc;
  for (const auto& x : {std::pair<const char*, const void*>("slopes", s.slopes), {"row_first", s.row_first}, {"row_end", s.row_end}, {"row_position", s.row_position},
                        {"key_position", s.key_position}, {"weight_in", weight_in}, {"weight_out", weight_out}})
    if ((rc = check_words(x.first, x.second)) != RELAYGR_OK) return rc;
  if (weight_in && !weight_out) return fail(RELAYGR_EINVAL, "%s: weight_in without weight_out", what);
  if ((s.key_position || weight_out) && !s.token_off && r->n_users > 0) return fail(RELAYGR_EINVAL, "%s: token arrays without token_off", what);
  for (int u = 0; u < r->n_users; ++u) {
    if (s.prefix && s.prefix[u] < 0) return fail(RELAYGR_EINVAL, "%s: user %d: a prefix of %d tokens", what, u, s.prefix[u]);
    if (s.token_off && s.token_off[u] < 0) return fail(RELAYGR_EINVAL, "%s: user %d: token offset %lld", what, u, (long long)s.token_off[u]);
  }
  return RELAYGR_OK;
}

// item_rows: of the launch's items, 16 or 32.
template <typename H, int DH, bool SM, bool BIAS, int USERS>
void launch_scored(const ScoredParams<USERS>& p, int item_rows, bool once, hipStream_t st) {
  const dim3 grid((unsigned)attend_groups(p.n_items, p.n_heads)), block(kAttendWaves * 64);
  if (item_rows == 32) { hipLaunchKernelGGL((scored8_kernel<H, DH, SM, BIAS, USERS>), grid, block, 0, st, p); return; }
  if constexpr (USERS > kFewScoredUsers) {
    if (once) { hipLaunchKernelGGL((scored8_few_kernel<H, DH, SM, BIAS, true, USERS>), grid, block, 0, st, p); return; }
  }
  hipLaunchKernelGGL((scored8_few_kernel<H, DH, SM, BIAS, false, USERS>), grid, block, 0, st, p);
}

struct Work { int user, rows, keys, parts, prefix, tiles; };

}  // namespace

int relaygr::scored8(KvPool* pool, const ScoredCall& call, hipStream_t st) {
  const AttendCall& c = call.attend;
  std::vector<PoolEntry> entries;
  const relaygr_kv_rows* r = c.rows;
  if (!call.scoring) return fail(RELAYGR_EINVAL, "%s: null argument", what);
  const relaygr_scoring& s = *call.scoring;
  int rc = resolve_rows(what, pool, c.layer, r, &entries);
  if (rc != RELAYGR_OK) return rc;
  if ((rc = check_scoring(r, s, call.weight_in, call.weight_out)) != RELAYGR_OK || r->n_users == 0) return rc;
  const relaygr_model_config& cfg = pool->cfg;
  const int d = cfg.d_model, H = cfg.n_heads, dh = d / H;
  const bool weigh = call.weight_out != nullptr;
  std::vector<Work> work, idle;      // idle: users without rows, whose weights are passed on
  std::vector<AttendLen> lens;
  int most_rows = 0;
  int64_t row_items = 0, row_tiles = 0;      // of 32 rows, and those times their tiles of keys
  for (int u = 0; u < r->n_users; ++u) {
    const int keys = r->key_len ? r->key_len[u] : entries[u].prefix_len, n = r->row_off[u + 1] - r->row_off[u];
    if (keys < 0 || keys > entries[u].prefix_len) return fail(RELAYGR_EINVAL, "%s: user %d: %d keys of an entry of %d tokens", what, u, keys, entries[u].prefix_len);
    const int prefix = s.prefix ? std::min(s.prefix[u], keys) : 0;
    if (prefix >= 1 << 25) return fail(RELAYGR_EINVAL, "%s: user %d: a prefix of %d tokens is more than a launch takes", what, u, prefix);
    if (n == 0) { idle.push_back({u, 0, keys, 1, prefix, 0}); continue; }
    // what an item's rows see at most: a window and the 32 or 64 tokens that its rows are apart
    const int64_t most = s.window > 0 ? std::min<int64_t>(keys, (int64_t)prefix + s.window + kTile) : keys;
    work.push_back({u, n, keys, 1, prefix, (int)((most + kTile - 1) / kTile)});
    lens.push_back({n, (int)most});
    most_rows = std::max(most_rows, n);
    row_items += (n + 31) / 32;
    row_tiles += (int64_t)((n + 31) / 32) * work.back().tiles;
  }
  if (weigh) {
    // (two users adding to one token would race)
    std::vector<std::pair<int64_t, int64_t>> tokens;
    for (const auto* list : {&work, &idle})
      for (const Work& w : *list) if (w.keys > 0) tokens.push_back({s.token_off[w.user], s.token_off[w.user] + w.keys});
    std::sort(tokens.begin(), tokens.end());
    for (size_t i = 1; i < tokens.size(); ++i)
      if (tokens[i].first < tokens[i - 1].second) return fail(RELAYGR_EINVAL, "%s: two users' weights overlap", what);
    // (and so would a token that is written where another's weight is read)
    if (call.weight_in && call.weight_in != call.weight_out) {
      const auto at = [&](const float* x, int64_t j) { return (uintptr_t)x + 4 * (uintptr_t)j; };
      for (size_t i = 0, j = 0; i < tokens.size() && j < tokens.size();) {
        const uintptr_t in = at(call.weight_in, tokens[i].second), out = at(call.weight_out, tokens[j].second);
        if (at(call.weight_in, tokens[i].first) < out && at(call.weight_out, tokens[j].first) < in)
          return fail(RELAYGR_EINVAL, "%s: weight_out overlaps weight_in elsewhere than token by token", what);
        if (in < out) ++i; else ++j;
      }
    }
  }
  if (!work.empty()) {
    if ((rc = check_rows_array(what, "q", c.q, c.q_stride, d)) != RELAYGR_OK) return rc;
    if ((rc = check_rows_array(what, "out", c.out, c.out_stride, d)) != RELAYGR_OK) return rc;
  }
  if (work.empty() && (!weigh || call.weight_in == call.weight_out)) return RELAYGR_OK;

  // scratch: rows' sums of weights | partial sums | scores
  char* scratch = c.scratch;
  size_t left = c.scratch_bytes;
  const auto take = [&](size_t bytes) { char* at = scratch; bytes = (bytes + 255) / 256 * 256; scratch += bytes; left -= bytes; return at; };
  float* lse = nullptr;
  if (weigh && c.softmax) {
    const size_t need = ((size_t)r->row_off[r->n_users] * H * 4 + 255) / 256 * 256;
    if (need > left) return fail(RELAYGR_ENOSPC, "%s: the rows' sums need %zu bytes of scratch, the context has %zu", what, need, left);
    lse = (float*)take(need);
  }
  AttendRule rule = attend_rule(lens, H, dh, c.n_cus);
  // Items of 16 rows where there are no more, and where there is little to do, of which twice as many make a shorter chain: at most 16 tiles of 32 rows a CU, or, of rows that
  // see from row_first on and so less than is known here, two items a CU.  17, 64 and 200 rows of one user over 2048, 2048 and 4096 tokens (1, 2 and 14 tiles a CU) take 8.8, 9.8 and 20.6 us
  // with 16 rows to an item and 10.3, 11.5 and 20.9 with 32 at heads of 128, 8.3, 8.7 and 14.2 against 9.0, 9.5 and 15.1 at 64; 8 users' 200 rows with sessions 13.5 and 16.9; 8 users of
  // 64 rows over 4096 (32 a CU) 18.8 and 19.3 at 64, 26.6 and 25.0 at 128; 16 of 200 over 4096 (224 a CU) 106 and 92.
  const bool little = s.row_first ? row_items * H <= 2 * c.n_cus : row_tiles * H <= 16 * c.n_cus;
  const int item_rows = most_rows <= 16 || little ? 16 : 32;
  const size_t row_bytes = (size_t)d * 4 + (c.softmax ? (size_t)H * 16 : 0);
  const auto items_of = [&](const Work& w) { return ((int64_t)w.rows + item_rows - 1) / item_rows * w.parts; };
  int64_t partial_rows = 0, most_items = 0;
  int most_sums = 0;      // rows of an item times its pieces
  for (;; rule.piece = rule.piece > 1 << 20 ? 0 : 2 * rule.piece) {      // (0: nothing is cut)
    partial_rows = most_items = 0;
    most_sums = 0;
    for (Work& w : work) {
      w.parts = attend_parts(w.tiles, rule.piece);
      if (w.parts > 1) partial_rows += (int64_t)w.parts * w.rows;
      most_sums = std::max(most_sums, std::min(w.rows, item_rows) * w.parts);
      most_items = std::max(most_items, items_of(w));
    }
    if (partial_rows == 0 || ((size_t)partial_rows * row_bytes + 512 <= left && partial_rows < (1ll << 31) && attend_fits(most_items, H))) break;
  }
  if (!attend_fits(most_items, H)) return fail(RELAYGR_EINVAL, "%s: %lld row tiles of one user are more than a launch takes", what, (long long)most_items);
  float* part = partial_rows ? (float*)take((size_t)partial_rows * d * 4) : nullptr;
  float4* ml = partial_rows && c.softmax ? (float4*)take((size_t)partial_rows * H * 16) : nullptr;
  float* saved = nullptr;
  int64_t saved_stride = 0;
  if (weigh && most_rows <= kSavedRows && !work.empty()) {
    for (const Work& w : work) saved_stride = std::max<int64_t>(saved_stride, ((int64_t)w.keys + kTile - 1) / kTile * kTile);
    // (a row's place in it is a 32-bit offset from its user's first)
    if (saved_stride * H * kSavedRows * 4 < 1ll << 31 && (size_t)r->row_off[r->n_users] * H * saved_stride * 4 <= left) saved = (float*)scratch;
  }
  std::stable_sort(work.begin(), work.end(), [](const Work& a, const Work& b) { return (int64_t)a.tiles * b.parts > (int64_t)b.tiles * a.parts; });    // the longest pieces first

  (void)hipGetLastError();
  Scoring sc = {};
  sc.slopes = s.slopes; sc.row_position = s.row_position; sc.key_position = s.key_position; sc.row_first = s.row_first; sc.row_end = s.row_end;
  sc.causal = c.causal ? 1 : 0; sc.window = s.window;
  const double alpha = 1.0 / std::sqrt((double)dh), log2e = 1.4426950408889634;
  sc.mul = (float)(alpha * log2e);
  if (s.cap > 0) {
    sc.mul = (float)(-2.0 * s.cap * log2e); sc.add = (float)(s.cap * log2e); sc.cap_mul = (float)(2.0 * alpha * log2e / s.cap);
    sc.cap_series = s.cap > kCapSeries;
  }
  const char* slab = (const char*)pool->slab + c.layer * pool->layer_stride;
  const int64_t scales_off = q8_scales_off(cfg, c.layer) - c.layer * pool->layer_stride;
  const auto user_of_work = [&](const Work& w, int32_t item0, int32_t part0) -> ScoredUser {
    ScoredUser x = {};
    x.page0 = (int32_t)entries[w.user].page0; x.row0 = r->row_off[w.user]; x.rows = w.rows; x.keys = w.keys; x.item0 = item0; x.part0 = part0;
    x.cut = (uint32_t)w.parts | (uint32_t)w.prefix << 7; x.token0 = s.token_off ? s.token_off[w.user] : 0;
    return x;
  };

  const auto by_form = [&](auto go) {      // go(softmax form, bias)
    if (c.softmax) { if (s.slopes) go(std::true_type(), std::true_type()); else go(std::true_type(), std::false_type()); }
    else if (s.slopes) go(std::false_type(), std::true_type());
    else go(std::false_type(), std::false_type());
  };
  int32_t part0 = 0;
  auto launch = [&](auto users) -> int {
    constexpr int USERS = decltype(users)::value;
    ScoredParams<USERS> p = {};
    p.q = (const uint16_t*)c.q; p.out = (uint16_t*)c.out; p.q_stride = c.q_stride; p.out_stride = c.out_stride;
    p.slab = slab; p.page_bytes = (int64_t)pool->page_bytes; p.tile_stride = pool->tile_stride; p.scales_off = scales_off;
    p.part = part; p.ml = ml; p.lse = lse; p.saved = saved; p.saved_stride = saved_stride;
    p.d = d; p.n_heads = H; p.s = sc;
    ScoredParams<USERS> j = p;
    const int launches = ((int)work.size() + USERS - 1) / USERS, per = ((int)work.size() + launches - 1) / launches;      // (as many users in each)
    for (size_t i = 0; i < work.size();) {
      p.n_users = 0; p.n_items = 0; j.n_users = 0; j.n_items = 0;
      for (; i < work.size() && p.n_users < per; ++i) {
        const Work& w = work[i];
        if (!attend_fits(p.n_items + items_of(w), H)) break;      // (never a launch's first)
        p.users[p.n_users++] = user_of_work(w, p.n_items, part0);
        p.n_items += (int32_t)items_of(w);
        if (w.parts == 1) continue;
        j.users[j.n_users++] = user_of_work(w, j.n_items, part0);
        j.n_items += w.rows;
        part0 += w.parts * w.rows;
      }
      p.arrived = USERS == kFewScoredUsers && attend_joins_itself(most_sums, (int64_t)p.n_items * H, kArrivals) ? c.arrived : nullptr;
      by_head(cfg, [&](auto h, auto dim) {
        using HT = decltype(h);
        constexpr int DH = decltype(dim)::value;
        by_form([&](auto sm, auto bias) {
          if constexpr (USERS != kTokenUsers || decltype(bias)::value) launch_scored<HT, DH, decltype(sm)::value, decltype(bias)::value>(p, item_rows, rule.once, st);
        });
        if (j.n_users == 0 || p.arrived) return;
        const dim3 grid((unsigned)(((int64_t)j.n_items * std::max(1, d / 256) + 3) / 4));
        if (c.softmax) hipLaunchKernelGGL((scored8_join_kernel<HT, DH, true, USERS>), grid, dim3(256), 0, st, j);
        else hipLaunchKernelGGL((scored8_join_kernel<HT, DH, false, USERS>), grid, dim3(256), 0, st, j);
      });
      LAUNCH_CHECK(what);
    }
    return RELAYGR_OK;
  };
  if (!work.empty()) {
    const bool few = (int)work.size() <= kFewScoredUsers && !(rule.once && item_rows == 16);
    rc = few ? launch(std::integral_constant<int, kFewScoredUsers>())
             : s.slopes && s.key_position ? launch(std::integral_constant<int, kTokenUsers>()) : launch(std::integral_constant<int, kScoredUsers>());
    if (rc != RELAYGR_OK) return rc;
  }
  if (!weigh) return RELAYGR_OK;

  WeighParams<kTokenUsers> w = {};
  w.q = (const uint16_t*)c.q; w.q_stride = c.q_stride;
  w.slab = slab; w.page_bytes = (int64_t)pool->page_bytes; w.tile_stride = pool->tile_stride; w.scales_off = scales_off;
  w.lse = lse; w.saved = saved; w.saved_stride = saved_stride; w.weight_in = call.weight_in; w.weight_out = call.weight_out;
  w.d = d; w.n_heads = H; w.s = sc;
  std::stable_sort(work.begin(), work.end(), [](const Work& a, const Work& b) { return a.rows > b.rows; });      // (a tile's work is its user's rows: 32 users of 200 to 1000 278 us, in the pieces' order 334)
  if (call.weight_in != call.weight_out) work.insert(work.end(), idle.begin(), idle.end());
  const int per = saved ? 256 : kTile;
  for (size_t i = 0; i < work.size();) {
    w.n_users = 0; w.n_units = 0;
    for (; i < work.size() && w.n_users < kTokenUsers; ++i) {
      const int units = (int)(((int64_t)work[i].keys + per - 1) / per);
      if (units == 0) continue;
      if (w.n_units > 0 && (int64_t)w.n_units + units >= 1 << 23) break;
      if (units >= 1 << 23) return fail(RELAYGR_EINVAL, "%s: the weights of %d tokens are more than a launch takes", what, work[i].keys);
      w.users[w.n_users++] = user_of_work(work[i], w.n_units, 0);
      w.n_units += units;
    }
    if (w.n_users == 0) break;
    const dim3 grid((unsigned)w.n_units);
    if (saved) {
      if (c.softmax) hipLaunchKernelGGL((weigh8_saved_kernel<true, kTokenUsers>), grid, dim3(256), 0, st, w);
      else hipLaunchKernelGGL((weigh8_saved_kernel<false, kTokenUsers>), grid, dim3(256), 0, st, w);
    } else {
      by_head(cfg, [&](auto h, auto dim) {
        using HT = decltype(h);
        constexpr int DH = decltype(dim)::value;
        by_form([&](auto sm, auto bias) {
          hipLaunchKernelGGL((weigh8_kernel<HT, DH, decltype(sm)::value, decltype(bias)::value, kTokenUsers>), grid, dim3(kWeighWaves * 64), 0, st, w);
        });
      });
    }
    LAUNCH_CHECK(what);
  }
  return RELAYGR_OK;
}
