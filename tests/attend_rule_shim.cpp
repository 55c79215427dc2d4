// csrc/attend_rules.h behind a C interface, for the tests.
#include "../paper_2601_01712_amd/csrc/attend_rules.h"

// out: 32-row blocks of an item, 1 if the codes are loaded once, key tiles of a piece (0: uncut), most pieces of a user
extern "C" void attend_rule_of(int n, const int32_t* rows, const int32_t* keys, int heads, int dh, int n_cus, int32_t* out) {
  std::vector<relaygr::AttendLen> users;
  for (int u = 0; u < n; ++u) users.push_back({rows[u], keys[u]});
  const relaygr::AttendRule r = relaygr::attend_rule(users, heads, dh, n_cus);
  out[0] = r.blocks; out[1] = r.once; out[2] = r.piece; out[3] = 1;
  for (int u = 0; u < n; ++u) out[3] = std::max(out[3], (int32_t)relaygr::attend_parts((keys[u] + 63) / 64, r.piece));
}
extern "C" int attend_parts_of(int tiles, int piece) { return relaygr::attend_parts(tiles, piece); }
extern "C" int attend_joins(int most_sums, int64_t items, int counters) { return relaygr::attend_joins_itself(most_sums, items, counters); }
