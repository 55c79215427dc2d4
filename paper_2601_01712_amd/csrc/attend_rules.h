// Which kernel a launch of attention over the 8-bit cache takes and how its key sequences are cut, by the batch's sizes.  No HIP in this file: the
// tests compile it with the host compiler, so that a test of a kernel can say that its launches take that kernel.
#pragma once

#include <stdint.h>

#include <algorithm>
#include <vector>

#include "plan.h"

namespace relaygr {

struct AttendLen { int rows, keys; };      // of a user: query rows, tokens that take part
struct AttendRule {
  int blocks = 1;        // 32-row blocks of an item
  bool once = false;     // the kernel whose loads are not kept in the caches
  int piece = 0;         // key tiles of a piece, about (0: nothing is cut)
};

// Pieces of a key sequence of nk tiles: as many as it has of `piece` tiles, to nearest, none of them empty.
constexpr int kAttendParts = 64;
inline int attend_parts(int nk, int piece) {
  if (piece <= 0 || nk == 0) return 1;
  const int parts = std::max(1, std::min((nk + piece / 2) / piece, kAttendParts)), per = (nk + parts - 1) / parts;
  return (nk + per - 1) / per;
}

// Whether a launch of few users joins the pieces of its rows itself, the last workgroup of an item's to arrive, or leaves that to a second launch, which takes 3.3 us of
// the host and 2 of the GPU but has all of the chip for it.  most_sums: rows of an item times its pieces, at most.
// (us among calls, itself / a second launch: one row over 2048 keys 8.2 / 11.0; in launches of many users, whose kernels do without it, the wait for the sums to reach
// the other XCDs costs more than the launch: 32 users of 8 to 60 rows over about 4096 keys 41.7 / 38.9.)
inline bool attend_joins_itself(int most_sums, int64_t items, int counters) { return most_sums <= 256 && items <= counters; }

// Workgroups of a launch of `items` items for each head, heads dealt to eight XCDs; and whether a launch takes them: it counts its threads, 256 a workgroup,
// in 32 bits.
inline int64_t attend_groups(int64_t items, int heads) { return heads >= 8 ? items * heads : (items + 8 / heads - 1) / (8 / heads) * 8; }
inline bool attend_fits(int64_t items, int heads) { return attend_groups(items, heads) < 1ll << 24; }

// A workgroup is four wavefronts that share an item's key tiles, and two or three of them a compute unit are full speed.
//
// Two blocks of 32 rows an item (one conversion of the codes for twice the rows) where the launch still has four items a compute unit and users have
// so many rows that few blocks are empty; at d_head 64, where the registers hold them.  us, one block / two, d = 512: 16 users of 512 rows over 4096
// keys 94.4 / 88.1, 32 of 200 to 1000 over about 4096 249 / 238, softmax 87.8 / 83.2 and 228 / 215; 64 of 200 over 2048, whose fourth block of 64 is nearly empty,
// 95.9 / 103, softmax 85.8 / 91.8, 40 of 200 to 700, causal, over about 1500 76.7 / 77.7; fewer items: one of 512 over 4096 13.4 / 15.4; few rows: 64 of 50 to 100 103 / 120; d_head 32, 16
// of 500 to 1000 over 8000 211 / 218.
//
// Sequences are cut where the launch has fewer items than the chip has compute units (at d = 512 one user of 4096 keys: 512 rows, 128 items, uncut 16.1, 256
// pieces 13.4, 512 14.8; one row of 16 384 keys, 8 items, uncut 50, 128 pieces 10.4, 256 11.2, 512 14.4), and where items are of unequal length
// those that would be left running behind the others (32 users of 8 to 60 rows over about 4096 keys, 48 key tiles a piece 40.6, uncut 55.6): each cut
// is a partial sum to write and read and the first one a launch.  Unequal items: as many pieces as the chip has room for at once, so that no compute unit is left with the
// last; three a unit (d_head 128 and two blocks: the registers hold two), unless these are short.  us, pieces for two a unit / for three: the 32 users above 35.6 / 32.9, 24
// of 1 to 8 rows over about 6000 40.3 / 35.0, 50 of 30 to 64, causal, 71 / 65, 8 of 100 to 300 over 3000 42.5 / 38.4; fewer keys: 100 of 1 to 4 rows over about
// 1000 (16 784 key tiles) 29.5 / 30.7, 6 of 4 to 40 over about 10 000 (10 096) 18.9 / 20.0; d_head 128 in 12 of 20 to 90 over about 5000 47.9 / 50.0.  Around the
// switch single lists decide more than their size: 22 lists at d_head 64 and 22 at 32, of 38 to 145 key tiles a unit (12 to 48 users of 1 to 90 rows), three over two 0.88 to 1.12; mean of those with 80
// and more 0.98 at either d_head, of those with 53 to 80 0.97 too, of those with 38 1.03.  448 equal items of 33 tiles: uncut 12.3, in halves 14.5.
//
// Codes that one item alone reads, more of them than the caches could keep until they are read again: 128 users of 8192 keys, one row each (1.07 GB) 180 / 162
// without keeping, of 2048 and four rows (268 MB) 51.3 / 44.8; 64 of 4096 and 20 at d = 1024 93.7 / 83.4.
constexpr int kLeastPiece = 4;
constexpr int64_t kOnceBytes = (int64_t)128 << 20;      // half of the last-level cache
inline AttendRule attend_rule(const std::vector<AttendLen>& users, int heads, int dh, int n_cus) {
  AttendRule r;
  int64_t rows = 0, keys = 0, items1 = 0, items2 = 0, key_tiles = 0, most = 0;
  int most_rows = 0;
  for (const AttendLen& u : users) {
    const int64_t nk = (u.keys + kTile - 1) / kTile;
    rows += u.rows; keys += u.keys;
    items1 += (u.rows + 31) / 32; items2 += (u.rows + 63) / 64;
    most_rows = std::max(most_rows, u.rows);
    most = std::max(most, nk);
  }
  if (dh == 64 && items2 * heads >= 4 * n_cus && rows >= 192 * (int64_t)users.size()) r.blocks = 2;
  r.once = most_rows <= 32 && 2 * keys * heads * dh >= kOnceBytes;
  const int64_t items = (r.blocks == 2 ? items2 : items1) * heads;
  for (const AttendLen& u : users) key_tiles += (u.rows + 32 * r.blocks - 1) / (32 * r.blocks) * (int64_t)((u.keys + kTile - 1) / kTile) * heads;
  const bool equal = 3 * most * items <= 4 * key_tiles;                   // the longest is at most a third over the mean
  if (equal && items >= n_cus) return r;
  const int64_t slots = equal ? n_cus : dh < 128 && r.blocks == 1 && key_tiles >= 80 * (int64_t)n_cus ? 3 * n_cus : 2 * n_cus;
  r.piece = (int)std::max<int64_t>(kLeastPiece, std::min<int64_t>((key_tiles + slots - 1) / slots, 1 << 20));
  return r;
}

}  // namespace relaygr
