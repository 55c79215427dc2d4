// Launch sizes of csrc/attend_rules.h behind a C interface, for the tests.
#include "../paper_2601_01712_amd/csrc/attend_rules.h"

extern "C" int64_t attend_groups_of(int64_t items, int heads) { return relaygr::attend_groups(items, heads); }
extern "C" int attend_fits_in(int64_t items, int heads) { return relaygr::attend_fits(items, heads); }
