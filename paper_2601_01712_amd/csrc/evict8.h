// Eviction from the 8-bit K/V cache (kv8.h): of a user's n tokens m stay, the first ones, the last ones and between them those with the largest weight, in their
// order, in every layer.  One kernel chooses them, another moves them.
//
// Choosing: weights as unsigned numbers of the same order; the smallest that stays is found by digits of 11, 11 and 10 bits, ties go to the lowest
// token.  Moving: tile t of what stays takes its 64 tokens from tiles t and on, and is quantised anew from the values their codes stand for.  What bounds it is HBM: the
// codes of all n tokens in, of m out.
#pragma once

#include "kv8.h"

namespace relaygr {

constexpr int kEvictUsers = 64;
struct EvictUser {
  int32_t from, to;    // first pages of the entry that is read and of the one that is written
  int32_t len, keep;   // tokens now, and afterwards
  int32_t kept0;       // where in `kept` its tokens' places go
  int32_t unit0;       // groups of tiles of the launch's users before it
  int64_t token0;      // where its tokens stand in `weight` and `position`
  int64_t out0;        // where those that stay go in weight_out and position_out
};
struct EvictParams {
  const float* weight;
  const int32_t* position;           // or null
  float* weight_out;                 // or null
  int32_t* position_out;             // or null
  int32_t* kept;
  char* slab;
  int64_t page_bytes, tile_stride, layer_stride, scales_off;      // of a page; between tiles, layers; of layer 0's scales
  int32_t n_users, n_units, n_layers, n_heads;
  int32_t first, recent;
  int32_t in_place;
  EvictUser users[kEvictUsers];
};

// A weight as a number of the same order: NaN below all, -0 as 0.
__device__ __forceinline__ uint32_t weight_order(float w) {
  const uint32_t b = __float_as_uint(w == 0.0f ? 0.0f : w);
  return w != w ? 0u : b & 0x80000000u ? ~b : b | 0x80000000u;
}

// Running sums over a wavefront's lanes, each with its own.
__device__ __forceinline__ uint32_t lanes_upto(uint32_t x) {
  x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x111, 0xF, 0xF, true);      // rows of 16 lanes: from 1, 2, 4 and 8 lanes below
  x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x112, 0xF, 0xF, true);
  x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x114, 0xF, 0xF, true);
  x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x118, 0xF, 0xF, true);
  x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x142, 0xA, 0xF, true);      // the last lane of rows 0 and 2 to rows 1 and 3
  x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x143, 0xC, 0xF, true);      // and lane 31 to rows 2 and 3
  return x;
}

// One workgroup a user.  What bounds it is the chain of its steps, so that there are few: digits of 11 bits (and the exponents of a few orders of magnitude do not meet in a
// few counters), a histogram of its own for each of the three, in each of which one wavefront finds first the 32 digits and then the digit.  The
// orders of 4096 tokens are in registers, those of 32 768 in LDS; the weights of longer entries are read again for each step.
// 4095 tokens 7.4 us, 32 users of up to 16 384 24.7 us (four digits of 8 bits and the weights read again for each: 11.3 and 43.5; 16 orders a thread in registers: 10.5 and
// 30.6, most of it code that is fetched once).
constexpr int kChooseThreads = 1024, kChooseStaged = 32768;
__global__ __launch_bounds__(kChooseThreads) void evict_choose_kernel(EvictParams p) {
  constexpr int EACH = 4, SPAN = kChooseThreads * EACH, WAVES = kChooseThreads / 64, BINS = 2048, PAD = BINS + BINS / 32 * 4;      // (32 bins to a lane: 16 bytes more to each)
  __shared__ __attribute__((aligned(16))) uint32_t counts[3 * PAD];
  __shared__ __attribute__((aligned(16))) uint32_t totals[2][EACH * WAVES];
  __shared__ uint32_t found[3][3];
  __shared__ uint32_t staged[kChooseStaged];
  const EvictUser u = p.users[blockIdx.x];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const float* weight = p.weight + u.token0;
  const bool all = u.keep == u.len;
  const int a = all ? u.len : p.first, b = all ? u.len : u.len - p.recent;      // the tokens [a, b) are those to choose from
  uint32_t want = all ? 0 : (uint32_t)(u.keep - p.first - p.recent);             // and so many of them stay
  const bool once = u.len <= SPAN, in_lds = u.len <= kChooseStaged;
  uint32_t order[EACH], choice = 0;      // bit i: token i of the thread is one of [a, b)
  int each = 0;
  auto load = [&](int j0) {
    each = min((u.len - j0 + kChooseThreads - 1) / kChooseThreads, EACH);
    choice = 0;
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
      if (i >= each) continue;      // (the same for all)
      const int j = j0 + i * kChooseThreads + tid;
      order[i] = in_lds && !once ? staged[j] : weight_order(weight[min(j, u.len - 1)]);
      choice |= (uint32_t)(j >= a && j < b) << i;
    }
  };
  for (int i = tid; i < 3 * PAD; i += kChooseThreads) counts[i] = 0;
  if (once) {
    load(0);
  } else if (in_lds) {
#pragma unroll 8
    for (int j = tid; j < (u.len + SPAN - 1) / SPAN * SPAN; j += kChooseThreads) staged[j] = weight_order(weight[min(j, u.len - 1)]);
  }
  __syncthreads();
  // the order of the want-th largest, and how many of those equal to it stay, of how many
  uint32_t prefix = 0, equal = 0;
  if (want > 0) {
    int shift = 32;
#pragma unroll 1
    for (int pass = 0; pass < 3; ++pass) {
      const int above_shift = shift, bits = pass < 2 ? 11 : 10;
      shift -= bits;
      for (int j0 = 0; j0 < u.len; j0 += SPAN) {
        if (!once) load(j0);
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
          if (i >= each) continue;
          const uint32_t o = order[i], digit = (o >> shift) & ((1u << bits) - 1), bin = digit + (digit >> 5) * 4;
          const bool counted = ((choice >> i) & 1) && (pass == 0 || (o >> above_shift) == (prefix >> above_shift));
          const uint64_t mine = __builtin_amdgcn_ballot_w64(counted);
          if (mine == 0) continue;
          // (equal weights, like the zeros of tokens that were never looked at: one count for all of them)
          const uint32_t one = (uint32_t)__builtin_amdgcn_readlane((int)bin, __builtin_ctzll(mine));
          if (__builtin_amdgcn_ballot_w64(counted & (bin != one)) == 0) {
            if (lane == 0) atomicAdd(&counts[pass * PAD + one], (uint32_t)__builtin_popcountll(mine));
          } else if (counted) {
            atomicAdd(&counts[pass * PAD + bin], 1u);
          }
        }
      }
      __syncthreads();
      if (wave == 0) {
        // lane i: the 32 digits from BINS - 32 (i + 1) on, and how many are above them; then lane i: the i-th largest of the 32
        const uint32_t* mine = &counts[pass * PAD + (63 - lane) * 36];
        uint32_t sum = 0;
#pragma unroll
        for (int i = 0; i < 32; i += 4) {
          const u32x4_t x = *reinterpret_cast<const u32x4_t*>(mine + i);
          sum += x[0] + x[1] + x[2] + x[3];
        }
        uint32_t upto = lanes_upto(sum);
        const int at = __builtin_ctzll(__builtin_amdgcn_ballot_w64(upto >= want));
        const uint32_t above = (uint32_t)__builtin_amdgcn_readlane((int)(upto - sum), at);
        sum = counts[pass * PAD + (63 - at) * 36 + 31 - (lane & 31)];
        upto = above + lanes_upto(lane < 32 ? sum : 0);
        if (lane == __builtin_ctzll(__builtin_amdgcn_ballot_w64(upto >= want))) {
          found[pass][0] = (uint32_t)((63 - at) * 32 + 31 - lane);
          found[pass][1] = want - (upto - sum);
          found[pass][2] = sum;
        }
      }
      __syncthreads();
      prefix |= found[pass][0] << shift;
      want = found[pass][1];
      equal = found[pass][2];
    }
  }
  // their places.  before(flags): how many of the flags of a span's tokens are set before the thread's own, for each of them; how many in all
  const uint64_t below = (1ull << lane) - 1;
  auto before = [&](uint32_t flags, uint32_t* sums, uint32_t (&at)[EACH]) -> uint32_t {
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
      const uint64_t set = i < each ? __builtin_amdgcn_ballot_w64((flags >> i) & 1) : 0;
      at[i] = __builtin_popcountll(set & below);
      if (lane == 0) sums[i * WAVES + wave] = __builtin_popcountll(set);
    }
    __syncthreads();
    static_assert(EACH * WAVES == 64);
    const uint32_t sum = sums[lane], upto = lanes_upto(sum);
#pragma unroll
    for (int i = 0; i < EACH; ++i) at[i] += (uint32_t)__builtin_amdgcn_readlane((int)(upto - sum), i * WAVES + wave);
    return (uint32_t)__builtin_amdgcn_readlane((int)upto, 63);
  };
  uint32_t out = 0, ties = 0;
  float w_next[EACH];
  int32_t pos_next[EACH];
  auto fetch = [&](int j0) {
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
      const int j = min(j0 + i * kChooseThreads + tid, u.len - 1);
      w_next[i] = p.weight_out ? weight[j] : 0.0f;
      pos_next[i] = p.position_out ? p.position[u.token0 + j] : 0;
    }
  };
  fetch(0);
  for (int j0 = 0; j0 < u.len; j0 += SPAN) {
    if (!once) load(j0);
    float w[EACH];
    int32_t pos[EACH];
#pragma unroll
    for (int i = 0; i < EACH; ++i) { w[i] = w_next[i]; pos[i] = pos_next[i]; }
    if (j0 + SPAN < u.len) fetch(j0 + SPAN);
    uint32_t tied = 0, stay = 0;
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
      if (i >= each) continue;
      const int j = j0 + i * kChooseThreads + tid;
      const bool chosen = (choice >> i) & 1;
      tied |= (uint32_t)(chosen && want > 0 && order[i] == prefix) << i;
      stay |= (uint32_t)(j < u.len && (!chosen || (want > 0 && order[i] > prefix))) << i;
    }
    uint32_t at[EACH];
    if (want == equal) {
      stay |= tied;
    } else {
      const uint32_t of_all = before(tied, totals[0], at);
#pragma unroll
      for (int i = 0; i < EACH; ++i) stay |= (uint32_t)(((tied >> i) & 1) && ties + at[i] < want) << i;
      ties += of_all;
    }
    const uint32_t more = before(stay, totals[1], at);      // (behind its barrier all weights and positions of the span have been read)
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
      if (i >= each || !((stay >> i) & 1)) continue;
      const uint32_t to = out + at[i];
      if (to >= (uint32_t)u.keep) continue;      // (never, unless the weights change meanwhile)
      p.kept[u.kept0 + (int)to] = j0 + i * kChooseThreads + tid;
      if (p.weight_out) p.weight_out[u.out0 + to] = w[i];
      if (p.position_out) p.position_out[u.out0 + to] = pos[i];
    }
    out += more;
    if (!once) __syncthreads();      // (the counts are read)
  }
}

// The largest magnitude of codes, a word at a time as 16-bit pairs, and 0x7F for a NaN among them.
__device__ __forceinline__ uint32_t code_max(uint32_t top, uint32_t w) { return max_u16x2(max_u16x2(top, w & 0x007F007Fu), (w >> 8) & 0x007F007Fu); }

// A 4 x 4 transposition of bytes within four neighbouring lanes: lane i's byte j becomes lane j's byte i.
__device__ __forceinline__ uint32_t quad_transpose(uint32_t w, uint32_t sel1, uint32_t sel2) {
  const uint32_t x = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)w, 0xB1, 0xF, 0xF, true);      // of lane ^ 1
  w = __builtin_amdgcn_perm(w, x, sel1);
  const uint32_t y = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)w, 0x4E, 0xF, 0xF, true);      // of lane ^ 2
  return __builtin_amdgcn_perm(w, y, sel2);
}

// Moving: a wavefront to a tile of one head of K or of V, a workgroup to WAVES of them, one behind the other, and a lane to a token: K's features of one are 16-byte pieces, V's are
// bytes of tiles that go to LDS, two at a time, and the tile that is written goes by way of it too, after words have changed from four features of a token to four tokens of a feature.
// In place a workgroup takes all the tiles of its head one group after the other: what a group reads are tiles from its first on, which the groups before it have left
// alone, and its wavefronts write only when all of them have read.  32 users of 151 316 tokens, three quarters of which stay, of a width of 512 in two layers elsewhere: 107 us,
// 5.1 TB/s (a byte at a time from V's tiles where they lie in memory, with the words in scratch: 242); one user's 4095 tokens of a width of 256 6.2 us.
// In place, and in few workgroups (of a user's heads, K and V, and layers), those are as wide as the registers and LDS allow: us, four wavefronts / 16 (eight at heads of 128), three quarters stay in two
// layers: one user of 16 384 tokens, d = 512 186 / 112 (elsewhere 40), 8 of 4096 54.5 / 39.8 (34), 16 (512 workgroups) 65.6 / 62.6, 32 103 / 112 (106); d = 1024, 8 84 / 68, 16 (512) 113 / 120; d = 256,
// 32 users of 1000 and four heads (512) 23.4 / 24.1, 64 32 / 40.
constexpr int kMoveWaves = 4, kWideGroups = 512;
template <int DH> constexpr int kWideWaves = DH == 128 ? 8 : 16;
template <typename H, int DH, int WAVES>
__global__ __launch_bounds__(WAVES * 64) void evict_move_kernel(EvictParams p) {
  constexpr int BLOCK = kTile * DH, CHUNKS = DH / 16, KP = DH / 32, WORDS = DH / 4, SLOTS = 2;
  __shared__ __attribute__((aligned(16))) uint8_t turn[WAVES][SLOTS * BLOCK];
  const int lane = threadIdx.x & 63, l32 = lane & 31, g = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  const int of_group = p.n_layers * p.n_heads * 2;
  const int group = (int)(blockIdx.x / of_group), in_group = (int)(blockIdx.x - (unsigned)group * of_group);
  const int layer = in_group / (p.n_heads * 2), head = (in_group >> 1) % p.n_heads, is_v = in_group & 1;
  const EvictUser u = user_of(p.users, p.n_users, group, lane, [](const EvictUser& x) { return x.unit0; });
  const int tiles = (u.keep + kTile - 1) / kTile;
  const int32_t* kept = p.kept + u.kept0;
  const int64_t codes_off = layer * p.layer_stride + (int64_t)head * (2 * BLOCK) + is_v * BLOCK;
  const int64_t scale_off = p.scales_off + ((int64_t)layer * p.n_heads + head) * 8 + is_v * 4;
  const char* from = p.slab + u.from * p.page_bytes;
  char* to = p.slab + u.to * p.page_bytes;
  uint8_t* lds = turn[wave];
  for (int t0 = (group - u.unit0) * WAVES;; t0 += WAVES) {
    const int t = t0 + wave;
    const bool mine = t < tiles;
    u32x4_t x[CHUNKS];
    float scale = 1.0f;
    if (mine) {
      const int r = t * kTile + lane;
      const bool there = r < u.keep;
      const int s = min(max(kept[min(r, u.keep - 1)], 0), u.len - 1);       // where the lane's token is
      const int s_tile = s / kTile, s_in = s & (kTile - 1);
      const float s_scale = *reinterpret_cast<const float*>(from + s_tile * p.tile_stride + scale_off);
      uint32_t w[WORDS];      // its codes, four features to a word
      if (!is_v) {
        const char* at = from + s_tile * p.tile_stride + codes_off + (s_in >> 5) * (KP * 1024) + (s_in & 31) * 16;
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {      // (words in the chunks' order)
          const u32x4_t v = *reinterpret_cast<const u32x4_t*>(at + (c >> 1) * 1024 + (c & 1) * 512);
          w[4 * c] = v[0]; w[4 * c + 1] = v[1]; w[4 * c + 2] = v[2]; w[4 * c + 3] = v[3];
        }
      } else {
#pragma unroll
        for (int i = 0; i < WORDS; ++i) w[i] = 0;
        const int first = __builtin_amdgcn_readfirstlane(s_tile), last = __builtin_amdgcn_readlane(s_tile, 63);
        const int in_tile = ((s_in >> 5) * 64 + ((s_in >> 2) & 1) * 32) * 16 + ((s_in >> 4) & 1) * 8 + ((s_in >> 3) & 1) * 4 + (s_in & 3);
        for (int ts = first; ts <= last; ts += SLOTS) {
          u32x4_t y[SLOTS][CHUNKS];
#pragma unroll
          for (int k = 0; k < SLOTS; ++k) {
            const char* tile = from + min(ts + k, last) * p.tile_stride + codes_off;
#pragma unroll
            for (int c = 0; c < CHUNKS; ++c) y[k][c] = *reinterpret_cast<const u32x4_t*>(tile + c * 1024 + lane * 16);
          }
          wave_lds_done();
#pragma unroll
          for (int k = 0; k < SLOTS; ++k)
#pragma unroll
            for (int c = 0; c < CHUNKS; ++c) *reinterpret_cast<u32x4_t*>(lds + k * BLOCK + c * 1024 + lane * 16) = y[k][c];
          wave_lds_done();
          if (s_tile >= ts && s_tile < ts + SLOTS) {
            const uint8_t* at = lds + (s_tile - ts) * BLOCK + in_tile;
#pragma unroll
            for (int i = 0; i < WORDS; ++i) {
              const int f = 4 * i;
              const uint8_t* b = at + (f >> 5) * 2048 + (f & 31) * 16;
              w[i] = (uint32_t)b[0] | (uint32_t)b[16] << 8 | (uint32_t)b[32] << 16 | (uint32_t)b[48] << 24;
            }
          }
        }
      }
      uint32_t top2 = 0;
#pragma unroll
      for (int i = 0; i < WORDS; ++i) {
        w[i] = there ? w[i] : 0;
        top2 = code_max(top2, w[i]);
      }
      uint32_t top = max(top2 & 0xFFFFu, top2 >> 16);
      if (__builtin_amdgcn_ballot_w64(top == 0x7Fu) != 0) {      // NaN among them: left out
        top = 0;
#pragma unroll
        for (int i = 0; i < WORDS; ++i)
#pragma unroll
          for (int b = 0; b < 4; ++b) { const uint32_t code = (w[i] >> (8 * b)) & 0x7Fu; top = max(top, code == 0x7Fu ? 0u : code); }
      }
      const f32x2_t mag = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(top, s_scale, false);
      scale = pow2f(fp8_exponent(__uint_as_float(wave_max_u32(__float_as_uint(there ? mag[0] : 0.0f)))));
      const bool other = there && s_scale != scale;
      if (__builtin_amdgcn_ballot_w64(other) != 0) {
#pragma unroll
        for (int i = 0; i < WORDS; ++i) w[i] = other ? fp8_rescale4(w[i], s_scale, scale) : w[i];
      }
      if (!is_v) {
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) x[c] = u32x4_t{w[4 * c], w[4 * c + 1], w[4 * c + 2], w[4 * c + 3]};
      } else {
        const uint32_t sel1 = lane & 1 ? 0x07030501u : 0x02060004u, sel2 = lane & 2 ? 0x07060302u : 0x01000504u;
        wave_lds_done();
        // the word of feature 4 i + lane % 4 and of the tile's tokens 4 (lane / 4) + {0..3}
        uint8_t* at = lds + ((g * 64 + ((lane >> 2) & 1) * 32) + (lane & 3)) * 16 + ((lane >> 4) & 1) * 8 + ((lane >> 3) & 1) * 4;
#pragma unroll
        for (int i = 0; i < WORDS; ++i) *reinterpret_cast<uint32_t*>(at + (i >> 3) * 2048 + (i & 7) * 64) = quad_transpose(w[i], sel1, sel2);
        wave_lds_done();
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) x[c] = *reinterpret_cast<const u32x4_t*>(lds + c * 1024 + lane * 16);
      }
    }
    if (p.in_place) __syncthreads();
    if (mine) {
      char* tile = to + t * p.tile_stride;
      char* at = tile + codes_off;
#pragma unroll
      for (int c = 0; c < CHUNKS; ++c) *reinterpret_cast<u32x4_t*>(at + (is_v ? c * 1024 + lane * 16 : g * (KP * 1024) + (c >> 1) * 1024 + (c & 1) * 512 + l32 * 16)) = x[c];
      if (lane == 0) *reinterpret_cast<float*>(tile + scale_off) = scale;
    }
    if (!p.in_place || t0 + WAVES >= tiles) break;
  }
}

}  // namespace relaygr
