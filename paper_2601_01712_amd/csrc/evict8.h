// Eviction from the 8-bit K/V cache (kv8.h): of a user's n tokens m stay, the first ones, the last ones and between them those with the largest weight, in their
// order, in every layer.  One kernel chooses them, another moves them.
//
// Choosing: weights as unsigned numbers of the same order; the smallest that stays is found digit by digit (four histograms of 256 counts), ties go to the lowest
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

// One workgroup a user.
constexpr int kChooseThreads = 1024;
__global__ __launch_bounds__(kChooseThreads) void evict_choose_kernel(EvictParams p) {
  constexpr int WAVES = kChooseThreads / 64;
  __shared__ uint32_t counts[256];
  __shared__ uint32_t found[2];
  __shared__ int totals[2][WAVES];
  const EvictUser u = p.users[blockIdx.x];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const float* weight = p.weight + u.token0;
  const bool all = u.keep == u.len;
  const int a = all ? u.len : p.first, b = all ? u.len : u.len - p.recent;      // the tokens [a, b) are those to choose from
  uint32_t want = all ? 0 : (uint32_t)(u.keep - p.first - p.recent);             // and so many of them stay
  // the order of the want-th largest, and how many of those equal to it stay
  uint32_t prefix = 0;
  if (want > 0) {
    for (int shift = 24; shift >= 0; shift -= 8) {
      if (tid < 256) counts[tid] = 0;
      __syncthreads();
      for (int j = a + tid; j < b; j += kChooseThreads) {
        const uint32_t o = weight_order(weight[j]);
        if (shift == 24 || (o >> (shift + 8)) == (prefix >> (shift + 8))) atomicAdd(&counts[(o >> shift) & 255u], 1u);
      }
      __syncthreads();
      if (wave == 0) {      // lane i: digits 255 - 4i and the three below
        uint32_t mine[4], sum = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) { mine[i] = counts[255 - 4 * lane - i]; sum += mine[i]; }
        uint32_t above = sum;
#pragma unroll
        for (int by = 1; by < 64; by *= 2) {
          const uint32_t x = __shfl_up(above, by, 64);
          above += lane >= by ? x : 0;
        }
        above -= sum;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (above < want && above + mine[i] >= want) { found[0] = 255 - 4 * lane - i; found[1] = want - above; }
          above += mine[i];
        }
      }
      __syncthreads();
      prefix |= found[0] << shift;
      want = found[1];
    }
  }
  // their places, 1024 tokens at a time
  int out = 0;
  uint32_t ties = 0;
  for (int j0 = 0; j0 < u.len; j0 += kChooseThreads) {
    const int j = j0 + tid;
    const bool there = j < u.len, choice = there && j >= a && j < b;
    const float w = there ? weight[j] : 0.0f;
    const int32_t pos = there && p.position ? p.position[u.token0 + j] : 0;
    const uint32_t o = weight_order(w);
    const bool tie = choice && want > 0 && o == prefix;
    const uint64_t below = (1ull << lane) - 1;
    const uint64_t tied = __builtin_amdgcn_ballot_w64(tie);
    if (lane == 0) totals[0][wave] = __builtin_popcountll(tied);
    __syncthreads();
    uint32_t before = ties, of_all = 0;
#pragma unroll
    for (int i = 0; i < WAVES; ++i) { before += i < wave ? totals[0][i] : 0; of_all += totals[0][i]; }
    ties += of_all;
    const bool stays = there && (!choice || (want > 0 && (o > prefix || (tie && before + __builtin_popcountll(tied & below) < want))));
    const uint64_t staying = __builtin_amdgcn_ballot_w64(stays);
    if (lane == 0) totals[1][wave] = __builtin_popcountll(staying);
    __syncthreads();       // (and all weights and positions of the 1024 have been read)
    int at = out, more = 0;
#pragma unroll
    for (int i = 0; i < WAVES; ++i) { at += i < wave ? totals[1][i] : 0; more += totals[1][i]; }
    out += more;
    if (stays) {
      at += __builtin_popcountll(staying & below);
      p.kept[u.kept0 + at] = j;
      if (p.weight_out) p.weight_out[u.out0 + at] = w;
      if (p.position_out) p.position_out[u.out0 + at] = pos;
    }
  }
}

// Moving: a wavefront to a tile of one head of K or of V, a workgroup to kMoveWaves of them, one behind the other.  In place a workgroup takes all the tiles of its head one
// group after the other: what a group reads are tiles from its first on, which the groups before it have left alone, and its wavefronts write only
// when all of them have read.
constexpr int kMoveWaves = 4;
template <typename H, int DH>
__global__ __launch_bounds__(kMoveWaves * 64) void evict_move_kernel(EvictParams p) {
  constexpr int BLOCK = kTile * DH, CHUNKS = DH / 16, KP = DH / 32;
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
  for (int t0 = (group - u.unit0) * kMoveWaves;; t0 += kMoveWaves) {
    const int t = t0 + wave;
    const bool mine = t < tiles;
    uint4 x[CHUNKS];
    float scale = 1.0f;
    if (mine) {
      const int r = t * kTile + lane;
      const bool there = r < u.keep;
      const int s = there ? min(max(kept[r], 0), u.len - 1) : 0;       // (the place of a token of this tile, to each lane)
      const int64_t s_tile = (int64_t)(s / kTile) * p.tile_stride;
      const float s_scale = there ? *reinterpret_cast<const float*>(from + s_tile + scale_off) : 0.0f;
      if (!is_v) {
        // a lane moves a token
        const char* at = from + s_tile + codes_off + ((s >> 5) & 1) * (KP * 1024) + (s & 31) * 16;
        uint32_t w[CHUNKS][4];
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
          const uint4 v = *reinterpret_cast<const uint4*>(at + (c >> 1) * 1024 + (c & 1) * 512);
          w[c][0] = there ? v.x : 0; w[c][1] = there ? v.y : 0; w[c][2] = there ? v.z : 0; w[c][3] = there ? v.w : 0;
        }
        uint32_t top = 0;
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
          for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int b = 0; b < 4; ++b) { const uint32_t code = (w[c][i] >> (8 * b)) & 0x7Fu; top = max(top, code == 0x7Fu ? 0u : code); }
        const f32x2_t mag = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(top, s_scale, false);
        const float amax = __uint_as_float(wave_max_u32(__float_as_uint(there ? mag[0] : 0.0f)));
        scale = pow2f(fp8_exponent(amax));
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
          uint32_t o[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) o[i] = !there || s_scale == scale ? w[c][i] : fp8_rescale4(w[c][i], s_scale, scale);
          x[c] = make_uint4(o[0], o[1], o[2], o[3]);
        }
      } else {
        // a lane takes a feature of 32 of the tile's tokens, four to a word (kv8.h)
        const char* at = from + codes_off + l32 * 16;
        uint32_t w[2][8][DH / 32];       // [token half][word][feature block]
        float ws[2][8][4];
        float amax = 0.0f;
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
          for (int m2 = 0; m2 < 4; ++m2) {
#pragma unroll
            for (int db = 0; db < DH / 32; ++db) w[kb][m2][db] = 0;
#pragma unroll
            for (int b = 0; b < 4; ++b) {
              const int r4 = kb * 32 + (m2 >> 1) * 16 + (m2 & 1) * 8 + 4 * g + b;
              const int q = __shfl(s, r4, 64);
              ws[kb][m2][b] = __shfl(s_scale, r4, 64);
              const bool is = t * kTile + r4 < u.keep;
              const int qr = q & 63, qw = qr & 15;
              const char* src = at + (int64_t)(q / kTile) * p.tile_stride + (((qr >> 5) * 64) + ((qw >> 2) & 1) * 32) * 16 + ((qr >> 4) & 1) * 8 + ((qw >> 3) << 2) + (qw & 3);
#pragma unroll
              for (int db = 0; db < DH / 32; ++db) {
                const uint32_t code = is ? (uint32_t)*reinterpret_cast<const uint8_t*>(src + db * 2048) : 0u;
                w[kb][m2][db] |= code << (8 * b);
                const uint32_t mag = code & 0x7Fu;
                const f32x2_t v = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(mag == 0x7Fu ? 0u : mag, ws[kb][m2][b], false);
                amax = fmaxf(amax, is ? v[0] : 0.0f);
              }
            }
          }
        scale = pow2f(fp8_exponent(__uint_as_float(wave_max_u32(__float_as_uint(amax)))));
#pragma unroll
        for (int db = 0; db < DH / 32; ++db)
#pragma unroll
          for (int kb = 0; kb < 2; ++kb) {
            uint32_t o[4];
#pragma unroll
            for (int m2 = 0; m2 < 4; ++m2) {
              const uint32_t c = w[kb][m2][db];
              float y[4];
#pragma unroll
              for (int b = 0; b < 4; ++b) {
                const f32x2_t v = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8((c >> (8 * b)) & 0xFFu, ws[kb][m2][b], false);
                y[b] = ws[kb][m2][b] == 0.0f ? 0.0f : v[0];
              }
              o[m2] = fp8_down4_f32(y[0], y[1], y[2], y[3], scale);
            }
            x[db * 2 + kb] = make_uint4(o[0], o[1], o[2], o[3]);
          }
      }
    }
    if (p.in_place) __syncthreads();
    if (mine) {
      char* tile = to + t * p.tile_stride;
      char* at = tile + codes_off;
      if (!is_v) {
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) *reinterpret_cast<uint4*>(at + g * (KP * 1024) + (c >> 1) * 1024 + (c & 1) * 512 + l32 * 16) = x[c];
      } else {
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) *reinterpret_cast<uint4*>(at + c * 1024 + lane * 16) = x[c];
      }
      if (lane == 0) *reinterpret_cast<float*>(tile + scale_off) = scale;
    }
    if (!p.in_place || t0 + kMoveWaves >= tiles) break;
  }
}

}  // namespace relaygr
