// Attention of query rows over the 8-bit K/V cache (kv8.h) with scores that are capped or biased, masks that are ranges of tokens, and the weight that each
// token received.  Row i of user u, at position p_i, sees the first `prefix` tokens of the user's entry and those in [first_i, end_i):
//     t_ij = alpha <q_i, k_j>,   t <- cap tanh(t / cap),   t <- t - slope_h |p_i - p_j|
//     softmax form  w_ij = exp(t_ij) / sum_j exp(t_ij)        SiLU form  w_ij = SiLU(t_ij) / n_i, n_i the tokens that the row sees
//     o_i = sum_j w_ij v_j        (0 where n_i = 0)           W_j <- W_j + sum over heads and rows of |w_ij|
// Products, operand layouts and roundings are those of attend8.h; scores are in units of ln 2.  cap tanh(t / cap) = cap - 2 cap / (1 + e), e = exp(2 t / cap): an exp2 and a
// reciprocal, right also where e is beyond fp32.  In units of 2^-23, with exp2 and the reciprocal an ulp off: exp2 and its argument |2 t / cap| + 1 of e, the sum 1/2 and the reciprocal 1 of
// themselves, in all at most 1.64 of 1 / (1 + e), which is twice as much of the cap; the factors and the last sum 1/2 each: 4.3, 2^-20.8 of the cap (2.2 with both rounded right, 3.2 with both an ulp off,
// over a million scores).  Up to a cap of kCapSeries that is 7e-5 of a weight, a seventh of its rounding to fp16; above, where it would be felt in small scores, the
// power series of tanh is taken up to 0.3 as well.
//
// Tokens' weights need the sums that a row ends with, so that a second kernel adds them up: from the scores, where the first left them in scratch (few rows: 4 bytes
// a score instead of d_head codes of K), or from K and q again.  It adds in one order, one workgroup to a token: no atomics.
#pragma once

#include "attend8.h"

namespace relaygr {

// Users of a launch: many without arrays of their tokens, fewer with them, few.
constexpr int kScoredUsers = 128, kTokenUsers = 64, kFewScoredUsers = 16;
constexpr float kCapSeries = 128.0f;
// Rows of a user up to which the scores are kept for the tokens' weights.  us of a call, kept / from K again: d = 512, 64 users over 4096 keys, one row 55.7 / 94.5, four 68.1 / 94.8, eight 78.8 /
// 95.3; one user 14.8 / 18.4, 18.2 / 19.5 and 21.9 / 20.3; 16 over 2048, SiLU form, 20.4 / 28.6, 24.4 / 30.0 and 29.2 / 31.3; d = 256, 32 over 4096, eight 33.2 / 42.5.
constexpr int kSavedRows = 8;
struct ScoredUserShort {
  int32_t page0;       // the entry's first page in the slab
  int32_t row0, rows;  // the user's rows in q and out
  int32_t keys;        // tokens that take part
  int32_t item0;       // items of the launch's users before it, for one head
  int32_t part0;       // first of its rows in the table of partial sums
  uint32_t cut;        // pieces that the tiles of each item are cut into (7 bits), tokens that all of its rows see (at most keys)
  __host__ __device__ __forceinline__ int parts() const { return (int)(cut & 127); }
  __host__ __device__ __forceinline__ int prefix() const { return (int)(cut >> 7); }
};
static_assert(sizeof(ScoredUserShort) == 28, "ScoredUserShort layout");
struct ScoredUser : ScoredUserShort {
  int64_t token0;      // where its tokens stand in key_position and the weights
};
__device__ __forceinline__ ScoredUser whole_user(const ScoredUser& u) { return u; }
__device__ __forceinline__ ScoredUser whole_user(const ScoredUserShort& u) { ScoredUser w; static_cast<ScoredUserShort&>(w) = u; w.token0 = 0; return w; }
// What scores and masks go by, the same for all kernels of a call.
struct Scoring {
  const float* slopes;               // [heads], or null
  const int32_t *row_position, *key_position, *row_first, *row_end;     // or null
  int32_t causal, window;
  float mul, add;                    // score = mul * x + add, x the product (mul = alpha log2(e)), or with a cap 1 / (1 + exp2(cap_mul * product)) (mul = -2 cap log2(e))
  float cap_mul;                     // 2 alpha log2(e) / cap; 0: no cap
  int32_t cap_series;
};
template <int USERS> struct ScoredParams {
  const uint16_t* q;
  uint16_t* out;
  int64_t q_stride, out_stride;      // elements between rows
  const char* slab;                  // of the pool, at the call's layer
  int64_t page_bytes, tile_stride, scales_off;   // bytes: of a page, between tiles, from a tile's codes to its layer's scales
  float* part;                       // [partial rows][d] sums of rows that are cut along the keys
  float4* ml;                        // [partial rows][heads]: reference score, sum of rounded weights, sum of weights
  float* lse;                        // [rows][heads]: log2 of a row's sum of weights (softmax form), or null
  float* saved;                      // scores [rows][heads][saved_stride], or null
  int64_t saved_stride;
  uint32_t* arrived;                 // as AttendParams'
  int32_t n_users, n_items, d, n_heads;
  Scoring s;
  std::conditional_t<USERS == kScoredUsers, ScoredUserShort, ScoredUser> users[USERS];
};

// The tokens that a row sees: the first `pre`, and [lo, hi) behind them.
struct RowRange {
  int pre, lo, hi;
  __device__ __forceinline__ int count() const { return pre + hi - lo; }
  __device__ __forceinline__ int from() const { return lo == pre ? 0 : lo; }      // of the range that ends at hi
};
__device__ __forceinline__ RowRange row_range(const Scoring& s, const ScoredUser& u, int i) {
  int end = s.causal ? max(u.keys - u.rows + 1 + i, 0) : u.keys, first = 0;
  if (s.row_end) end = min(end, max(s.row_end[u.row0 + i], 0));
  if (s.row_first) first = max(s.row_first[u.row0 + i], 0);
  if (s.window > 0) first = max(first, end - s.window);
  RowRange r;
  r.pre = u.prefix();
  r.lo = max(first, r.pre);
  r.hi = max(end, r.lo);
  return r;
}
__device__ __forceinline__ int row_place(const Scoring& s, const ScoredUser& u, int i) {
  return s.row_position ? s.row_position[u.row0 + i] : s.causal ? u.keys - u.rows + i : u.keys;
}
__device__ __forceinline__ int wave_max_i32(int v) { return (int)(wave_max_u32((uint32_t)v ^ 0x80000000u) ^ 0x80000000u); }
__device__ __forceinline__ int wave_min_i32(int v) { return ~wave_max_i32(~v); }

// Which tiles the rows of a wavefront see, and of a tile whether all of them see all of it.
struct TileRange {
  int pre_tiles, t0, n;              // the prefix's tiles, and behind them the tiles from t0 on: n together
  int pre, all_from, all_hi;
  __device__ __forceinline__ int tile(int v) const { return v < pre_tiles ? v : t0 + v - pre_tiles; }
  __device__ __forceinline__ bool whole(int t) const {
    const int a = t * kTile, b = a + kTile;
    return b <= pre || (b <= all_hi && a >= all_from);
  }
};
__device__ __forceinline__ TileRange tile_range(const Scoring& s, const ScoredUser& u, int row0, int rows, const RowRange& r, bool is_row) {
  TileRange t;
  t.pre = u.prefix();
  t.pre_tiles = (t.pre + kTile - 1) / kTile;
  int lo, hi;
  if (!s.row_first && !s.row_end) {      // ranges climb with the rows: scalar work, of the first and the last
    const RowRange a = row_range(s, u, row0), b = row_range(s, u, row0 + rows - 1);
    lo = a.lo;
    hi = b.hi > b.lo ? b.hi : 0;
    t.all_from = b.from();
    t.all_hi = a.hi;
  } else {
    const bool any = is_row && r.hi > r.lo;
    hi = wave_max_i32(any ? r.hi : 0);
    lo = wave_min_i32(any ? r.lo : 0x7FFFFFFF);
    t.all_from = wave_max_i32(is_row ? r.from() : 0);
    t.all_hi = wave_min_i32(is_row ? r.hi : 0x7FFFFFFF);
  }
  t.t0 = max(lo / kTile, t.pre_tiles);
  t.n = t.pre_tiles + max((hi + kTile - 1) / kTile - t.t0, 0);
  return t;
}

// The bias by distance, of one wavefront's rows and head.  The positions of a tile's tokens are in LDS, one word each.  Where the rows are close together (kTight) a word is
// slope * (position - base), base the least of the rows' positions, so that the bias is a sum for tokens behind every row, and is turned where one is not: its rounding is
// that of a product with the distance from base.  Otherwise words are the positions, and distances whole numbers before they are rounded.
constexpr int kTight = 64;
struct Bias {
  const int32_t* at;      // positions of the user's tokens, or null: their places in the entry
  float slope;            // in units of ln 2
  int base, last;
  bool tight;
  __device__ __forceinline__ int load(int t, int lane) const { return at ? at[min(t * kTile + lane, last)] : t * kTile + lane; }
  __device__ __forceinline__ uint32_t word(int k) const { return tight ? __float_as_uint(slope * (float)(k - base)) : (uint32_t)k; }
  __device__ __forceinline__ bool behind(int k) const { return __builtin_amdgcn_ballot_w64(k > base) == 0; }
};
// row0, rows: the wavefront's rows, place_of a lane's position among them.
__device__ __forceinline__ Bias bias_of(const Scoring& s, const ScoredUser& u, int head, int row0, int rows, int place_of) {
  int lo = s.causal ? u.keys - u.rows + row0 : u.keys, hi = s.causal ? lo + rows - 1 : lo;
  if (s.row_position) { lo = wave_min_i32(place_of); hi = wave_max_i32(place_of); }
  Bias b;
  b.at = s.key_position ? s.key_position + u.token0 : nullptr;
  b.slope = s.slopes[head] * 1.4426950408889634f;
  b.base = __builtin_amdgcn_readfirstlane(lo);
  b.last = u.keys - 1;
  b.tight = __builtin_amdgcn_readfirstlane((int64_t)hi - lo < kTight) != 0;
  return b;
}
enum ScoreKind { kPlain, kTightBias, kAnyBias };

// Scores of a row less `off` from the products of 16 tokens; words: of their positions, element e's at 8 * (e / 4) + e % 4.  A score is one product and one sum behind its cap; what
// is taken off it is in the sum, and the tight bias one instruction more.
__device__ __forceinline__ float tanh_series(float x) {
  const float y = x * x;
  return x * fmaf(y, fmaf(y, fmaf(y, fmaf(y, 2.1869488e-2f, -5.3968254e-2f), 1.3333333e-1f), -3.3333333e-1f), 1.0f);
}
template <ScoreKind KIND>
__device__ __forceinline__ void scores_of(const Scoring& c, const Bias& bias, int place_of, float off, bool behind, const uint32_t* words, f32x16_t& s) {
  float mul = c.mul, add = c.add;
  if (c.cap_mul != 0.0f) {
    if (!c.cap_series) {
#pragma unroll
      for (int e = 0; e < 16; ++e) s[e] = __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(s[e] * c.cap_mul));
    } else {
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const float x2 = s[e] * c.cap_mul, x = x2 * 0.34657359027997264f;       // 2 x log2(e), x = score / cap
        const float far = fmaf(c.mul, __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(x2)), c.add);
        s[e] = fabsf(x) < 0.3f ? c.add * tanh_series(x) : far;
        if (e % 2) __builtin_amdgcn_sched_barrier(0);      // (few of them at once: registers)
      }
      mul = 1.0f;
      add = 0.0f;
    }
  }
  const float k = add - off;
  if constexpr (KIND == kPlain) {
#pragma unroll
    for (int e = 0; e < 16; ++e) s[e] = fmaf(mul, s[e], k);
  } else {
    const float from = bias.slope * (float)(place_of - bias.base), kb = k - from, turn = bias.slope < 0.0f ? 1.0f : -1.0f;
#pragma unroll
    for (int h = 0; h < 16; h += 8) {      // (eight at a time: registers)
      const u32x4_t w[2] = {*reinterpret_cast<const u32x4_t*>(words + 2 * h), *reinterpret_cast<const u32x4_t*>(words + 2 * h + 8)};
      if constexpr (KIND == kTightBias) {      // slope (p_j - p_i), or where a token is not behind every row its magnitude, less or more
        float a[8];
        if (behind) {
#pragma unroll
          for (int e = 0; e < 8; ++e) a[e] = kb + __uint_as_float(w[e >> 2][e & 3]);
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e) a[e] = fmaf(turn, fabsf(__uint_as_float(w[e >> 2][e & 3]) - from), k);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) s[h + e] = fmaf(mul, s[h + e], a[e]);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) s[h + e] = fmaf(-bias.slope, fabsf((float)(place_of - (int)w[e >> 2][e & 3])), fmaf(mul, s[h + e], k));
      }
    }
  }
}
// Which of a lane's 16 tokens its row sees: bit 8 * (e / 4) + e % 4 for element e.  from: the first of the 32 tokens that they are of; add: place - from.
__device__ __forceinline__ uint32_t bits_below(int n) { return (uint32_t)((1ull << min(max(n, 0), 32)) - 1); }
__device__ __forceinline__ uint32_t seen_bits(const RowRange& r, int from, int add) {
  return (bits_below(r.pre - from) | (bits_below(r.hi - from) & ~bits_below(r.lo - from))) >> add;
}
// All ones or none, for element e.
__device__ __forceinline__ uint32_t seen_mask(uint32_t bits, int e) { return (uint32_t)__builtin_amdgcn_sbfe((int)bits, 8 * (e >> 2) + (e & 3), 1); }
__device__ __forceinline__ float seen_or(uint32_t bits, int e, float x, float otherwise) {
  const uint32_t m = seen_mask(bits, e);
  return __uint_as_float((m & __float_as_uint(x)) | (~m & __float_as_uint(otherwise)));      // (one instruction, no condition registers)
}

// attend8_nans for tokens that rows see or not one by one.  add(a, b) adds the product of a and b to the sums of the chunk's features.
template <class Add>
__device__ __forceinline__ void scored8_nans(uint4& chunk, uint32_t bits, Add add) {
  const uint32_t big = 0x7180;          // 2^100 in bf16
#pragma unroll
  for (int m = 0; m < 2; ++m) {
    uint32_t &w0 = m == 0 ? chunk.x : chunk.z, &w1 = m == 0 ? chunk.y : chunk.w;
    asm volatile("" : "+v"(w0), "+v"(w1), "+v"(bits));      // (what is worked out here is not kept in registers from before)
    const uint32_t n0 = fp8_nans(w0), n1 = fp8_nans(w1);
    w0 &= ~(n0 * 0xFFu);
    w1 &= ~(n1 * 0xFFu);
    const u32x4_t pos = fp8_frag<Bf16>(n0 * 0x38u, n1 * 0x38u, 0x1p100f), neg = fp8_frag<Bf16>(n0 * 0xB8u, n1 * 0xB8u, 0x1p100f);   // codes of 1 and -1
    uint32_t see[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) see[j] = (seen_mask(bits, 8 * m + 2 * j) & big) | (seen_mask(bits, 8 * m + 2 * j + 1) & (big << 16));
    const uint4 seen = make_uint4(see[0], see[1], see[2], see[3]);
    add(pos, seen);
    add(neg, seen);
    __builtin_amdgcn_sched_barrier(0);
  }
}

// A tile's codes of K and V of one head.  Loads of a tile that is not there (no bytes) are made all the same, as zeros and without memory: a wavefront always has as many on their way,
// so that it waits for those it needs and not for all.
struct TileCodes {
  __amdgpu_buffer_rsrc_t rsrc;
  __device__ __forceinline__ TileCodes(const char* at, int bytes) : rsrc(__builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(at), 0, bytes, 0x00020000)) {}
  template <bool ONCE> __device__ __forceinline__ uint4 load(int lane_off, int off) const {
    return __builtin_bit_cast(uint4, __builtin_amdgcn_raw_buffer_load_b128(rsrc, lane_off, off, ONCE ? 2 : 0));      // (2: not temporal)
  }
  template <bool ONCE> __device__ __forceinline__ uint2 load8(int lane_off, int off) const {
    return __builtin_bit_cast(uint2, __builtin_amdgcn_raw_buffer_load_b64(rsrc, lane_off, off, ONCE ? 2 : 0));
  }
};

// An item of the launch: rows of one user, one head, one piece of the tiles that they see.
struct ScoredItem {
  ScoredUser u;
  int head, piece, first_row, n_rows;
};
template <int ROWS, int USERS>
__device__ __forceinline__ bool scored8_item(const ScoredParams<USERS>& p, int lane, ScoredItem* it) {
  const int xcd = blockIdx.x & 7, turn = blockIdx.x >> 3, heads_sh = __builtin_ctz(p.n_heads);
  int item;
  if (p.n_heads >= 8) {
    const int sh = heads_sh - 3;
    it->head = (xcd << sh) + (turn & ((1 << sh) - 1));
    item = turn >> sh;
  } else {
    it->head = xcd & (p.n_heads - 1);
    item = (turn << (3 - heads_sh)) + (xcd >> heads_sh);
  }
  if (item >= p.n_items) return false;
  it->u = whole_user(user_of(p.users, p.n_users, item, lane, [](const ScoredUserShort& x) { return x.item0; }));
  const int row_tiles = (it->u.rows + ROWS - 1) / ROWS;
  it->piece = (item - it->u.item0) / row_tiles;
  it->first_row = (item - it->u.item0 - it->piece * row_tiles) * ROWS;
  it->n_rows = min(ROWS, it->u.rows - it->first_row);
  return true;
}

// The sums of a row's pieces, as PieceSum, with the sum of the weights before they were rounded beside them.
template <bool SOFTMAX> struct ScoredSum {
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
  float M = -INFINITY, l = 0.f, lx = 0.f;
  __device__ __forceinline__ void add(const float4& x, float m, float w, float wx) {
    if constexpr (SOFTMAX) {
      const float mn = fmaxf(M, m), c0 = M == mn ? 1.0f : __builtin_amdgcn_exp2f(M - mn), c1 = m == mn ? 1.0f : __builtin_amdgcn_exp2f(m - mn);
      o = make_float4(fmaf(x.x, c1, o.x * c0), fmaf(x.y, c1, o.y * c0), fmaf(x.z, c1, o.z * c0), fmaf(x.w, c1, o.w * c0));
      l = fmaf(w, c1, l * c0);
      lx = fmaf(wx, c1, lx * c0);
      M = mn;
    } else {
      o = make_float4(o.x + x.x, o.y + x.y, o.z + x.z, o.w + x.w);
    }
  }
  template <typename H> __device__ __forceinline__ uint2 out(int seen) const {
    const float mul = SOFTMAX ? 1.0f / l : 0.69314718055994531f / (float)seen;
    return seen == 0 ? make_uint2(0, 0) : make_uint2(H::pack2(o.x * mul, o.y * mul), H::pack2(o.z * mul, o.w * mul));
  }
  __device__ __forceinline__ float lse() const { return M + __builtin_amdgcn_logf(lx); }
};

// Joins the pieces of an item's rows in the workgroup that is the last of them to arrive, as attend8_join_last.
template <typename H, int DH, bool SOFTMAX, int ROWS, int USERS>
__device__ __forceinline__ void scored8_join_last(const ScoredParams<USERS>& p, const ScoredItem& it, int wave, int lane) {
  constexpr int LANES = DH / 4, GROUPS = 64 / LANES;
  __shared__ int last;
  if (wave == 0) {
    uint32_t* count = p.arrived + (it.u.item0 + it.first_row / ROWS) * p.n_heads + it.head;
    if (lane == 0) {      // (the release is of all the wavefront's stores)
      const uint32_t before = __hip_atomic_fetch_add(count, 1u, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT);
      last = before + 1 == (uint32_t)it.u.parts();
      if (last) *count = 0;
    }
  }
  __syncthreads();
  if (!last) return;
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "agent");
  const int group = lane / LANES, f = it.head * DH + (lane % LANES) * 4, parts = it.u.parts();
  const int64_t step = (int64_t)it.u.rows;
  for (int r0 = wave; r0 < it.n_rows; r0 += 16) {
    ScoredSum<SOFTMAX> sum[4];
    for (int k = group; k < parts + group; k += GROUPS) {      // (as many turns for every lane)
      float4 x[4], ml[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int64_t pr = it.u.part0 + min(k, parts - 1) * step + it.first_row + min(r0 + 4 * i, it.n_rows - 1);
        x[i] = *reinterpret_cast<const float4*>(p.part + pr * p.d + f);
        ml[i] = SOFTMAX ? p.ml[pr * p.n_heads + it.head] : make_float4(0.f, 0.f, 0.f, 0.f);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (k < parts) sum[i].add(x[i], ml[i].x, ml[i].y, ml[i].z);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (r0 + 4 * i >= it.n_rows) break;      // (the same for all lanes)
      ScoredSum<SOFTMAX>& a = sum[i];
#pragma unroll
      for (int by = LANES; by < 64; by *= 2) {
        const float4 x = make_float4(__shfl_xor(a.o.x, by, 64), __shfl_xor(a.o.y, by, 64), __shfl_xor(a.o.z, by, 64), __shfl_xor(a.o.w, by, 64));
        a.add(x, SOFTMAX ? __shfl_xor(a.M, by, 64) : 0.f, SOFTMAX ? __shfl_xor(a.l, by, 64) : 0.f, SOFTMAX ? __shfl_xor(a.lx, by, 64) : 0.f);
      }
      const int r = r0 + 4 * i;
      if (group == 0 && r < it.n_rows) {
        const int64_t row = it.u.row0 + it.first_row + r;
        *reinterpret_cast<uint2*>(p.out + row * p.out_stride + f) = a.template out<H>(row_range(p.s, it.u, it.first_row + r).count());
        if constexpr (SOFTMAX) {
          if (p.lse && lane == 0) p.lse[row * p.n_heads + it.head] = a.lse();
        }
      }
    }
  }
}

// Of a row's reference score (or its sum's logarithm) up to which scores_of takes it off as it makes the scores: those are rounded as sums with it are, 2^-24 of
// it (of 64: 4e-6).  Beyond, where a bias has put the first tokens' scores far below the last ones', scores are made whole and the reference is taken off them.
constexpr float kFoldOff = 64.0f;
// A row's running sums over its tokens: a softmax's reference score (mref, -inf before the first token), the sum of the rounded weights, and of the weights as they are
// (where tokens' weights are asked for).
struct RowSums {
  float mref, lsum, lexact;
  __device__ __forceinline__ void clear() { mref = -INFINITY; lsum = 0.f; lexact = 0.f; }
  // What scores_of may take off the scores, and whether that is all of the reference.
  __device__ __forceinline__ bool offset(float* off) const {
    *off = mref == -INFINITY ? 0.f : mref;
    const bool folded = __builtin_amdgcn_ballot_w64(fabsf(*off) > kFoldOff) == 0;
    *off = folded ? *off : 0.f;
    return folded;
  }
};
// Weights of 16 tokens, as packed pairs, from their scores less off, all of their reference if `folded`.  In the softmax form the row's reference score follows the largest seen
// score at a distance of at most kSlack, in which exp2 still fits either type; rescale(c) multiplies its output sums, and a row is the lanes that differ in the bits
// from ROW_LANES on of their number.
template <typename H, bool SOFTMAX, int ROW_LANES, class Rescale>
__device__ __forceinline__ void weights_of(f32x16_t& s, float off, bool folded, RowSums& sums, bool exact, uint32_t (&pk)[8], Rescale rescale) {
  if constexpr (SOFTMAX) {
    constexpr float kSlack = 8.0f;
    float mx = -INFINITY;
#pragma unroll
    for (int e = 0; e < 16; ++e) mx = fmaxf(mx, s[e]);
    const bool moves = __builtin_amdgcn_ballot_w64(mx > sums.mref - off + kSlack) != 0;
    if (moves) {
#pragma unroll
      for (int by = ROW_LANES; by < 64; by *= 2) mx = fmaxf(mx, __shfl_xor(mx, by, 64));
      const float mn = fmaxf(sums.mref, off + mx);
      const float c = mn == sums.mref ? 1.0f : __builtin_amdgcn_exp2f(sums.mref - mn);     // from -inf: 0
      sums.mref = mn;
      sums.lsum *= c;
      sums.lexact *= c;
      rescale(c);
    }
    if (moves || !folded) {
      const float more = sums.mref == -INFINITY ? 0.f : sums.mref - off;      // (a row that has seen nothing: weights exp2(-inf) = 0)
#pragma unroll
      for (int e = 0; e < 16; ++e) s[e] -= more;
    }
#pragma unroll
    for (int e = 0; e < 16; e += 2) {
      s[e] = __builtin_amdgcn_exp2f(s[e]);
      s[e + 1] = __builtin_amdgcn_exp2f(s[e + 1]);
      pk[e >> 1] = H::pack2(s[e], s[e + 1]);
      sums.lsum = H::dot2(pk[e >> 1], H::kOnes, sums.lsum);       // of the weights that the second product takes
    }
    if (exact) {
#pragma unroll
      for (int e = 0; e < 16; ++e) sums.lexact += s[e];
    }
  } else {
#pragma unroll
    for (int e = 0; e < 16; e += 2) {     // SiLU(t) / ln 2
      const float ta = s[e], tb = s[e + 1];
      pk[e >> 1] = H::pack2(ta * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-ta)), tb * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-tb)));
    }
  }
}
// Adds the sums of the workgroup's wavefronts, upper half to lower half, twice (a fixed order): wavefront 0 ends with all of them.  N: a lane's output sums, each(i).
template <bool SOFTMAX, int N, class Each>
__device__ __forceinline__ void join_waves(float (*join)[(N + (SOFTMAX ? 3 : 0)) * 64], int wave, int lane, RowSums& sums, Each each) {
#pragma unroll
  for (int half = kAttendWaves / 2; half >= 1; half >>= 1) {
    if (wave >= half && wave < 2 * half) {
      float* x = join[wave - half] + lane;
#pragma unroll
      for (int i = 0; i < N; ++i) x[i * 64] = each(i);
      if constexpr (SOFTMAX) { x[N * 64] = sums.mref; x[(N + 1) * 64] = sums.lsum; x[(N + 2) * 64] = sums.lexact; }
    }
    __syncthreads();
    if (wave < half) {
      const float* x = join[wave] + lane;
      float c0 = 1.0f, c1 = 1.0f;
      if constexpr (SOFTMAX) {
        const float m1 = x[N * 64], M = fmaxf(sums.mref, m1);
        c0 = sums.mref == M ? 1.0f : __builtin_amdgcn_exp2f(sums.mref - M);
        c1 = m1 == M ? 1.0f : __builtin_amdgcn_exp2f(m1 - M);
        sums.lsum = sums.lsum * c0 + x[(N + 1) * 64] * c1;
        sums.lexact = sums.lexact * c0 + x[(N + 2) * 64] * c1;
        sums.mref = M;
      }
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const float y = x[i * 64];
        float& o = each(i);
        if constexpr (SOFTMAX) o = o * c0 + y * c1;
        else o += y;
      }
    }
    __syncthreads();
  }
}
// Writes a lane's sums of one row, fours of features each at f(i): over all of its tokens as outputs, over one piece as partial sums.  The row is the lanes that differ in
// ROW_LANES; `first` is one of them.
template <typename H, bool SOFTMAX, int FOURS, int ROW_LANES, int USERS, class Feature, class Sum>
__device__ __forceinline__ void scored8_store(const ScoredParams<USERS>& p, const ScoredItem& it, int r, bool first, int seen, const RowSums& sums, Feature f, Sum sum) {
  float lsum = sums.lsum, exact = sums.lexact;
  if constexpr (SOFTMAX) {
#pragma unroll
    for (int by = ROW_LANES; by < 64; by *= 2) { lsum += __shfl_xor(lsum, by, 64); exact += __shfl_xor(exact, by, 64); }
  }
  if (r >= it.n_rows) return;
  const int64_t row = it.u.row0 + it.first_row + r;
  if (it.u.parts() == 1) {
    const float mul = SOFTMAX ? 1.0f / lsum : 0.69314718055994531f / (float)seen;
    uint16_t* dst = p.out + row * p.out_stride;
#pragma unroll
    for (int i = 0; i < FOURS; ++i) {
      const float4 o = sum(i);
      *reinterpret_cast<uint2*>(dst + f(i)) = seen == 0 ? make_uint2(0, 0) : make_uint2(H::pack2(o.x * mul, o.y * mul), H::pack2(o.z * mul, o.w * mul));
    }
    if constexpr (SOFTMAX) {
      if (p.lse && first) p.lse[row * p.n_heads + it.head] = sums.mref + __builtin_amdgcn_logf(exact);
    }
  } else {
    const int64_t pr = (int64_t)it.u.part0 + (int64_t)it.piece * it.u.rows + it.first_row + r;
    float* dst = p.part + pr * p.d;
#pragma unroll
    for (int i = 0; i < FOURS; ++i) *reinterpret_cast<float4*>(dst + f(i)) = sum(i);
    if constexpr (SOFTMAX) {
      if (first) p.ml[pr * p.n_heads + it.head] = make_float4(sums.mref, lsum, exact, 0.f);
    }
  }
}

// One item of up to 32 rows, as attend8_kernel: the workgroup's wavefronts take its tiles in turn, each straight from memory to its registers.  What bounds it is the vector ALU: 14
// instructions a score with a cap and a bias, of which two exp and a reciprocal.  16 users of 512 rows over 4096 keys, d = 512, SiLU form, bias by positions 106 us (0.65 PFLOP/s,
// the ALU issuing in 85 % of the units' cycles; relaygr_cache_attend's kernel 94); 32 of 200 to 1000 over about 4096, softmax, cap and bias 277 (95 %); 16 of 200 that see 2016 of 8192, d = 1024,
// cap 56 (63 %, MFMAs 27 %).  Three wavefronts a SIMD at d_head 64 and two at 128 are what the registers hold; 64 rows an item spill (the second 395 us where 32 took 357).
template <typename H, int DH, bool SOFTMAX, bool BIAS, int USERS>
__global__ __launch_bounds__(kAttendWaves * 64, DH == 128 ? 2 : 3) void scored8_kernel(ScoredParams<USERS> p) {
  constexpr int KS = DH / 16, KP = DH / 32, DB = DH / 32;
  constexpr int BLOCK = kTile * DH;            // bytes of codes of K, and of V
  __shared__ float join[kAttendWaves / 2][(DB * 16 + (SOFTMAX ? 3 : 0)) * 64];
  __shared__ __attribute__((aligned(16))) uint32_t words[kAttendWaves][kTile];
  const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, g = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  ScoredItem it;
  if (!scored8_item<32>(p, lane, &it)) return;
  const ScoredUser& u = it.u;
  const int head = it.head;

  const bool is_row = l32 < it.n_rows;
  const int i_row = it.first_row + (is_row ? l32 : 0);
  const RowRange range = row_range(p.s, u, i_row);
  uint4 qf[KS];
  const uint16_t* qr = p.q + (int64_t)(u.row0 + i_row) * p.q_stride + head * DH + g * 8;
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) qf[ks] = *reinterpret_cast<const uint4*>(qr + ks * 16);
  const int place_of = BIAS ? row_place(p.s, u, i_row) : 0;
  Bias bias = {};
  if constexpr (BIAS) bias = bias_of(p.s, u, head, it.first_row, it.n_rows, place_of);
  const TileRange tiles = tile_range(p.s, u, it.first_row, it.n_rows, range, is_row);
  const int v0 = (int)((int64_t)it.piece * tiles.n / u.parts()), v1 = (int)((int64_t)(it.piece + 1) * tiles.n / u.parts());

  f32x16_t oacc[DB];
  RowSums sums;
  sums.clear();
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int e = 0; e < 16; ++e) oacc[db][e] = 0.f;

  const char* kv = p.slab + (int64_t)u.page0 * p.page_bytes;
  const char* base = kv + (int64_t)head * (2 * BLOCK);
  const char* scales = kv + p.scales_off + head * 8;
  uint4 kr[2][KP], vr[2][DB];                   // codes of the tile's two halves
  float2 sc;
  int key_place = 0;
  auto load_k = [&](const TileCodes& tile, int kb) {
#pragma unroll
    for (int kp = 0; kp < KP; ++kp) kr[kb][kp] = tile.load<false>(lane * 16, (kb * KP + kp) * 1024);
  };
  auto load_v = [&](const TileCodes& tile, int kb) {
#pragma unroll
    for (int db = 0; db < DB; ++db) vr[kb][db] = tile.load<false>(lane * 16, BLOCK + (db * 2 + kb) * 1024);
  };
  auto load_scales = [&](int t) { return *reinterpret_cast<const float2*>(scales + (int64_t)t * p.tile_stride); };

  // one tile, half by half; each piece of codes makes room for the wavefront's next tile (tn, if there are more) as soon as it has been converted
  auto tile = [&](auto kind_tag, bool more, int t, int tn) {
    constexpr ScoreKind KIND = decltype(kind_tag)::value;
    const float2 sn = load_scales(tn);
    const TileCodes next(base + (int64_t)tn * p.tile_stride, more ? 2 * BLOCK : 0);
    bool behind = true;
    if constexpr (BIAS) {
      words[wave][lane] = bias.word(key_place);      // (a wavefront's own: its reads come behind its writes)
      behind = bias.behind(key_place);
      __builtin_amdgcn_wave_barrier();
      key_place = bias.load(tn, lane);
    }
    const bool whole = tiles.whole(t);
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
      f32x16_t s;
#pragma unroll
      for (int e = 0; e < 16; ++e) s[e] = 0.f;
#pragma unroll
      for (int kp = 0; kp < KP; ++kp) {
        s = H::mfma(fp8_frag<H>(kr[kb][kp].x, kr[kb][kp].y, sc.x), qf[2 * kp], s);
        s = H::mfma(fp8_frag<H>(kr[kb][kp].z, kr[kb][kp].w, sc.x), qf[2 * kp + 1], s);
      }
      __builtin_amdgcn_sched_barrier(0);      // (the next tile's codes take these ones' registers)
      load_k(next, kb);
      __builtin_amdgcn_sched_barrier(0);
      float off;
      const bool folded = sums.offset(&off);      // (the SiLU form has none)
      scores_of<KIND>(p.s, bias, place_of, off, behind, words[wave] + kb * 32 + 4 * g, s);
      if (!whole) {
        uint32_t any = 0;
        const uint32_t bits = seen_bits(range, t * kTile + kb * 32, 4 * g);
#pragma unroll
        for (int e = 0; e < 16; ++e) s[e] = seen_or(bits, e, s[e], SOFTMAX ? -INFINITY : 0.f);   // (SiLU(0) = 0)
#pragma unroll
        for (int db = 0; db < DB; ++db) any |= fp8_nans(vr[kb][db].x) | fp8_nans(vr[kb][db].y) | fp8_nans(vr[kb][db].z) | fp8_nans(vr[kb][db].w);
        if (__builtin_amdgcn_ballot_w64(any != 0) != 0) {
#pragma unroll
          for (int db = 0; db < DB; ++db)
            scored8_nans(vr[kb][db], bits, [&](const u32x4_t& a, const uint4& b) { oacc[db] = Bf16::mfma(a, b, oacc[db]); });
        }
      }
      uint32_t pk[8];
      weights_of<H, SOFTMAX, 32>(s, off, folded, sums, p.lse != nullptr, pk, [&](float c) {
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
          for (int e = 0; e < 16; ++e) oacc[db][e] *= c;
      });
#pragma unroll
      for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int db = 0; db < DB; ++db)
          oacc[db] = H::mfma(m == 0 ? fp8_frag<H>(vr[kb][db].x, vr[kb][db].y, sc.y) : fp8_frag<H>(vr[kb][db].z, vr[kb][db].w, sc.y),
                             make_uint4(pk[4 * m], pk[4 * m + 1], pk[4 * m + 2], pk[4 * m + 3]), oacc[db]);
      __builtin_amdgcn_sched_barrier(0);
      load_v(next, kb);
      __builtin_amdgcn_sched_barrier(0);
    }
    sc = sn;
  };
  // from the last tile to the first: where a bias falls with the distance the largest scores come first, and the reference scores stay where they are
  auto all_tiles = [&](auto kind) {
    int v = v1 - 1 - wave;
    if (v < v0) return;
    int t = tiles.tile(v);
    sc = load_scales(t);
    if constexpr (BIAS) key_place = bias.load(t, lane);
    const TileCodes first(base + (int64_t)t * p.tile_stride, 2 * BLOCK);
    load_k(first, 0);
    load_v(first, 0);
    load_k(first, 1);
    load_v(first, 1);
    for (; v >= v0; v -= kAttendWaves) {      // (one copy of a tile's code: with another for the last one it takes 40 registers more)
      const bool more = v - kAttendWaves >= v0;
      const int tn = more ? tiles.tile(v - kAttendWaves) : t;
      tile(kind, more, t, tn);
      t = tn;
    }
  };
  if constexpr (!BIAS) all_tiles(std::integral_constant<ScoreKind, kPlain>());
  else if (bias.tight) all_tiles(std::integral_constant<ScoreKind, kTightBias>());
  else all_tiles(std::integral_constant<ScoreKind, kAnyBias>());
  join_waves<SOFTMAX, DB * 16>(join, wave, lane, sums, [&](int i) -> float& { return reinterpret_cast<float*>(&oacc[i >> 4])[i & 15]; });
  if (wave == 0)
    scored8_store<H, SOFTMAX, DB * 4, 32>(p, it, l32, g == 0, range.count(), sums, [&](int i) { return head * DH + (i >> 2) * 32 + (i & 3) * 8 + 4 * g; },
                                          [&](int i) {
                                            const f32x16_t& o = oacc[i >> 2];
                                            return make_float4(o[4 * (i & 3)], o[4 * (i & 3) + 1], o[4 * (i & 3) + 2], o[4 * (i & 3) + 3]);
                                          });
  if constexpr (USERS <= kFewScoredUsers) {
    if (p.arrived != nullptr && u.parts() > 1) scored8_join_last<H, DH, SOFTMAX, 32>(p, it, wave, lane);
  }
}

// Items of up to 16 rows, by the 16x16x32 MFMA: half the work on the vector ALU for each tile, and so few registers that twice the wavefronts wait for memory.  The codes are in the
// order of the 32x32x16 product, and are taken from it so that a lane still loads 16 bytes at once.  Lane (quad, l16), kb = quad / 2, g = quad % 2:
//   K, T = 0..3 (16 tokens each): row i of the operand is token (i / 8) * 32 + 8 T + 4 (i / 4 % 2) + i % 4 of the tile, so that the product leaves a lane the tokens
//     kb * 32 + 4 g + 8 T + {0..3} of row l16, which is the order that scores_of and weights_of take; features as the chunk has them, q's in the same order
//     (d_head 32: a chunk's halves are lanes' 8 bytes)
//   V: the chunk of feature l16 of 16, token half kb, lane half g holds these very tokens, the first eight bytes those of T = 0, 1
// What bounds it is HBM, or for single rows the chain of loads: 128 users of one row over 8192 keys, d = 512, bias, 162 us (1.07 GB, 6.7 TB/s), 201 with the scores
// kept, whose 33.5 MB cost the same in whatever pieces they are stored; one row over 2048, d = 256, 8.2.  All arrays are in registers but two words (12 bytes of scratch) of the
// softmax form with a bias at d_head 64 for few users.
template <typename H, int DH, bool SOFTMAX, bool BIAS, bool ONCE, int USERS>
__global__ __launch_bounds__(kAttendWaves * 64, DH == 128 ? 2 : 4) void scored8_few_kernel(ScoredParams<USERS> p) {
  constexpr int KP = DH / 32, FB = DH / 16, KL = DH < 64 ? 1 : KP / 2;      // feature blocks; a lane's loads of K for 16 tokens
  constexpr int BLOCK = kTile * DH;
  __shared__ float join[kAttendWaves / 2][(FB * 4 + (SOFTMAX ? 3 : 0)) * 64];
  __shared__ __attribute__((aligned(16))) float turn[kAttendWaves][kSavedRows][kTile + 4];
  __shared__ __attribute__((aligned(16))) uint32_t words[kAttendWaves][kTile];
  const int tid = threadIdx.x, lane = tid & 63, l16 = lane & 15, quad = lane >> 4, kb = quad >> 1, g = quad & 1;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  ScoredItem it;
  if (!scored8_item<16>(p, lane, &it)) return;
  const ScoredUser& u = it.u;
  const int head = it.head;

  const bool is_row = l16 < it.n_rows;
  const int i_row = it.first_row + (is_row ? l16 : 0);
  const RowRange range = row_range(p.s, u, i_row);
  // q: operand h of load c holds features (kp * 2 + h) * 16 + 8 g, kp = kb + 2 c (d_head 32: kb * 16 + 8 g)
  uint4 qf[KL][2];
  const uint16_t* qr = p.q + (int64_t)(u.row0 + i_row) * p.q_stride + head * DH + g * 8;
#pragma unroll
  for (int c = 0; c < KL; ++c)
#pragma unroll
    for (int h = 0; h < (DH < 64 ? 1 : 2); ++h) qf[c][h] = *reinterpret_cast<const uint4*>(qr + (DH < 64 ? kb * 16 : (kb + 2 * c) * 32 + h * 16));
  const int place_of = BIAS ? row_place(p.s, u, i_row) : 0;
  Bias bias = {};
  if constexpr (BIAS) bias = bias_of(p.s, u, head, it.first_row, it.n_rows, place_of);
  const TileRange tiles = tile_range(p.s, u, it.first_row, it.n_rows, range, is_row);
  const int v0 = (int)((int64_t)it.piece * tiles.n / u.parts()), v1 = (int)((int64_t)(it.piece + 1) * tiles.n / u.parts());

  f32x4_t oacc[FB];
  RowSums sums;
  sums.clear();
#pragma unroll
  for (int fb = 0; fb < FB; ++fb)
#pragma unroll
    for (int e = 0; e < 4; ++e) oacc[fb][e] = 0.f;

  const char* kv = p.slab + (int64_t)u.page0 * p.page_bytes;
  const char* base = kv + (int64_t)head * (2 * BLOCK);
  const char* scales = kv + p.scales_off + head * 8;
  // where the lane's codes are in a tile
  const int token0 = (l16 >> 3) * 32 + ((l16 >> 2) & 1) * 4 + (l16 & 3);      // of T = 0
  const int k_off = DH < 64 ? ((token0 >> 5) * 64 + g * 32 + (token0 & 31)) * 16 + kb * 8 : (((token0 >> 5) * KP + kb) * 64 + g * 32 + (token0 & 31)) * 16;
  const int v_off = BLOCK + (kb * 64 + g * 32 + l16) * 16;
  uint4 kr[4][KL], vr[FB];
  float2 sc;
  int key_place = 0;
  auto load_k = [&](const TileCodes& tile) {
#pragma unroll
    for (int T = 0; T < 4; ++T) {
      if constexpr (DH < 64) {
        const uint2 w = tile.load8<ONCE>(k_off, T * 128);
        kr[T][0] = make_uint4(w.x, w.y, 0, 0);
      } else {
#pragma unroll
        for (int c = 0; c < KL; ++c) kr[T][c] = tile.load<ONCE>(k_off, T * 128 + c * 2048);
      }
    }
  };
  auto load_v = [&](const TileCodes& tile) {
#pragma unroll
    for (int fb = 0; fb < FB; ++fb) vr[fb] = tile.load<ONCE>(v_off, (fb >> 1) * 2048 + (fb & 1) * 256);
  };
  auto load_scales = [&](int t) { return *reinterpret_cast<const float2*>(scales + (int64_t)t * p.tile_stride); };

  // where the lane's scores of rows quad and 4 + quad go (beyond every bound: nowhere)
  float* saved = p.saved + ((int64_t)(u.row0 + it.first_row) * p.n_heads + head) * p.saved_stride;
  int saved_off[kSavedRows / 4];
#pragma unroll
  for (int i = 0; i < kSavedRows / 4; ++i) saved_off[i] = 4 * i + quad < it.n_rows ? (int)((4 * i + quad) * p.n_heads * p.saved_stride + l16 * 4) * 4 : (int)0x80000000u;

  auto tile = [&](auto kind_tag, bool more, int t, int tn) {
    constexpr ScoreKind KIND = decltype(kind_tag)::value;
    const float2 sn = load_scales(tn);
    const TileCodes next(base + (int64_t)tn * p.tile_stride, more ? 2 * BLOCK : 0);
    bool behind = true;
    if constexpr (BIAS) {
      words[wave][lane] = bias.word(key_place);
      behind = bias.behind(key_place);
      __builtin_amdgcn_wave_barrier();
      key_place = bias.load(tn, lane);
    }
    f32x16_t s;
#pragma unroll
    for (int T = 0; T < 4; ++T) {
      f32x4_t x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int c = 0; c < KL; ++c) {
        x = H::mfma16(fp8_frag<H>(kr[T][c].x, kr[T][c].y, sc.x), qf[c][0], x);
        if constexpr (DH >= 64) x = H::mfma16(fp8_frag<H>(kr[T][c].z, kr[T][c].w, sc.x), qf[c][1], x);
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) s[4 * T + j] = x[j];
    }
    __builtin_amdgcn_sched_barrier(0);      // (the next tile's codes take these ones' registers)
    load_k(next);
    __builtin_amdgcn_sched_barrier(0);
    float off;
    const bool folded = sums.offset(&off);
    scores_of<KIND>(p.s, bias, place_of, off, behind, words[wave] + kb * 32 + 4 * g, s);
    if (p.saved && l16 < kSavedRows) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *reinterpret_cast<float4*>(&turn[wave][l16][kb * 32 + 4 * g + 8 * i]) = make_float4(s[4 * i] + off, s[4 * i + 1] + off, s[4 * i + 2] + off, s[4 * i + 3] + off);
    }
    if (!tiles.whole(t)) {
      uint32_t any = 0;
      const uint32_t bits = seen_bits(range, t * kTile + kb * 32, 4 * g);
#pragma unroll
      for (int e = 0; e < 16; ++e) s[e] = seen_or(bits, e, s[e], SOFTMAX ? -INFINITY : 0.f);   // (SiLU(0) = 0)
#pragma unroll
      for (int fb = 0; fb < FB; ++fb) any |= fp8_nans(vr[fb].x) | fp8_nans(vr[fb].y) | fp8_nans(vr[fb].z) | fp8_nans(vr[fb].w);
      if (__builtin_amdgcn_ballot_w64(any != 0) != 0) {
#pragma unroll
        for (int fb = 0; fb < FB; ++fb) scored8_nans(vr[fb], bits, [&](const u32x4_t& a, const uint4& b) { oacc[fb] = Bf16::mfma16(a, b, oacc[fb]); });
      }
    }
    uint32_t pk[8];
    weights_of<H, SOFTMAX, 16>(s, off, folded, sums, p.lse != nullptr, pk, [&](float c) {
#pragma unroll
      for (int fb = 0; fb < FB; ++fb)
#pragma unroll
        for (int e = 0; e < 4; ++e) oacc[fb][e] *= c;
    });
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
      for (int fb = 0; fb < FB; ++fb)
        oacc[fb] = H::mfma16(m == 0 ? fp8_frag<H>(vr[fb].x, vr[fb].y, sc.y) : fp8_frag<H>(vr[fb].z, vr[fb].w, sc.y),
                             make_uint4(pk[4 * m], pk[4 * m + 1], pk[4 * m + 2], pk[4 * m + 3]), oacc[fb]);
    __builtin_amdgcn_sched_barrier(0);
    load_v(next);
    __builtin_amdgcn_sched_barrier(0);
    // the scores of four rows at a time, behind the loads, and as many stores in every tile, into nowhere where there is nothing to keep, so that a wait for loads counts past them
    const __amdgpu_buffer_rsrc_t to = __builtin_amdgcn_make_buffer_rsrc(saved + t * kTile, 0, p.saved ? 0x7FFFFFFF : 0, 0x00020000);
#pragma unroll
    for (int i = 0; i < kSavedRows / 4; ++i)
      __builtin_amdgcn_raw_buffer_store_b128(*reinterpret_cast<const u32x4_t*>(&turn[wave][4 * i + quad][l16 * 4]), to, saved_off[i], 0, 0);
    __builtin_amdgcn_wave_barrier();
    sc = sn;
  };
  auto all_tiles = [&](auto kind) {      // (from the last tile to the first, as above)
    int v = v1 - 1 - wave;
    if (v < v0) return;
    int t = tiles.tile(v);
    sc = load_scales(t);
    if constexpr (BIAS) key_place = bias.load(t, lane);
    const TileCodes first(base + (int64_t)t * p.tile_stride, 2 * BLOCK);
    load_k(first);
    load_v(first);
    for (; v >= v0; v -= kAttendWaves) {      // (one copy of a tile's code: with another for the last one it takes 40 registers more)
      const bool more = v - kAttendWaves >= v0;
      const int tn = more ? tiles.tile(v - kAttendWaves) : t;
      tile(kind, more, t, tn);
      t = tn;
    }
  };
  if constexpr (!BIAS) all_tiles(std::integral_constant<ScoreKind, kPlain>());
  else if (bias.tight) all_tiles(std::integral_constant<ScoreKind, kTightBias>());
  else all_tiles(std::integral_constant<ScoreKind, kAnyBias>());
  join_waves<SOFTMAX, FB * 4>(join, wave, lane, sums, [&](int i) -> float& { return reinterpret_cast<float*>(&oacc[i >> 2])[i & 3]; });
  if (wave == 0)
    scored8_store<H, SOFTMAX, FB, 16>(p, it, l16, quad == 0, range.count(), sums, [&](int i) { return head * DH + i * 16 + quad * 4; },
                                      [&](int i) { return make_float4(oacc[i][0], oacc[i][1], oacc[i][2], oacc[i][3]); });
  if constexpr (USERS <= kFewScoredUsers) {
    if (p.arrived != nullptr && u.parts() > 1) scored8_join_last<H, DH, SOFTMAX, 16>(p, it, wave, lane);
  }
}

// The same as a launch of its own: one wavefront for 256 features of a row, pieces loaded eight at a time.
template <typename H, int DH, bool SOFTMAX, int USERS>
__global__ __launch_bounds__(256) void scored8_join_kernel(ScoredParams<USERS> p) {
  constexpr int GROUPS = 256 / DH;
  const int lane = threadIdx.x & 63, segs_sh = max(__builtin_ctz(p.d) - 8, 0);
  const int unit = __builtin_amdgcn_readfirstlane((int)(blockIdx.x * 4 + (threadIdx.x >> 6)));
  const int row = unit >> segs_sh, f = (unit - (row << segs_sh)) * 256 + lane * 4;
  if (row >= p.n_items) return;        // (rows of the launch's users that are cut; item0: those of the users before)
  const ScoredUser u = whole_user(user_of(p.users, p.n_users, row, lane, [](const ScoredUserShort& x) { return x.item0; }));
  const int r = row - u.item0;
  const bool mine = f < p.d;           // (d = 128: half of the lanes)
  const int head = (mine ? f : 0) / DH;
  const float* x = p.part + ((int64_t)u.part0 + r) * p.d + (mine ? f : 0);
  const int64_t step = (int64_t)u.rows * p.d;      // between a row's pieces
  ScoredSum<SOFTMAX> sum[GROUPS];
  for (int k0 = 0; k0 < u.parts(); k0 += 8) {
    float4 v[8], ml[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const int kk = min(k0 + k, u.parts() - 1);
      v[k] = *reinterpret_cast<const float4*>(x + kk * step);
      ml[k] = SOFTMAX ? p.ml[((int64_t)u.part0 + (int64_t)kk * u.rows + r) * p.n_heads + head] : make_float4(0.f, 0.f, 0.f, 0.f);
    }
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (k0 + k < u.parts()) sum[k % GROUPS].add(v[k], ml[k].x, ml[k].y, ml[k].z);
  }
#pragma unroll
  for (int by = 1; by < GROUPS; by *= 2)
#pragma unroll
    for (int i = 0; i < GROUPS; i += 2 * by) sum[i].add(sum[i + by].o, sum[i + by].M, sum[i + by].l, sum[i + by].lx);
  if (!mine) return;
  const int64_t at = u.row0 + r;
  *reinterpret_cast<uint2*>(p.out + at * p.out_stride + f) = sum[0].template out<H>(row_range(p.s, u, r).count());
  if constexpr (SOFTMAX) {
    if (p.lse && f % DH == 0) p.lse[at * p.n_heads + head] = sum[0].lse();
  }
}

// ---- what each token was worth ----------------------------------------------------------------------------------------------------------
template <int USERS> struct WeighParams {
  const uint16_t* q;
  int64_t q_stride;
  const char* slab;
  int64_t page_bytes, tile_stride, scales_off;
  const float *lse, *saved;
  int64_t saved_stride;
  const float* weight_in;            // or null: zero
  float* weight_out;
  int32_t n_users, n_units, d, n_heads;
  Scoring s;
  ScoredUser users[USERS];           // item0: units of the launch's users before it
};
// |w| of a score, in the softmax form less the row's sum.  inv: SiLU form, ln 2 / n.
template <bool SOFTMAX>
__device__ __forceinline__ float weight_of(float t, float inv) {
  return SOFTMAX ? __builtin_amdgcn_exp2f(t) : fabsf(t * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-t))) * inv;
}

// From the scores that the attention kernel left, a token to a lane: units of 256 tokens.  64 users of one row over 8192 keys and 8 heads 5.9 us (16.8 MB of scores); from K again
// the same read 268 MB.
template <bool SOFTMAX, int USERS>
__global__ __launch_bounds__(256) void weigh8_saved_kernel(WeighParams<USERS> p) {
  const int lane = threadIdx.x & 63, unit = (int)blockIdx.x;
  const ScoredUser u = whole_user(user_of(p.users, p.n_users, unit, lane, [](const ScoredUserShort& x) { return x.item0; }));
  const int j = (unit - u.item0) * 256 + (int)threadIdx.x;
  if (j >= u.keys) return;
  const float* at = p.saved + (int64_t)u.row0 * p.n_heads * p.saved_stride + j;
  const int eights = (p.n_heads + 7) / 8, n = u.rows * eights;
  float sum = 0.f, x[2][8];
  auto load = [&](int i, float (&to)[8]) {      // eight heads of a row, the next eight on their way
    const int r = i / eights, h0 = (i - r * eights) * 8;
#pragma unroll
    for (int k = 0; k < 8; ++k) to[k] = at[((int64_t)r * p.n_heads + min(h0 + k, p.n_heads - 1)) * p.saved_stride];
  };
  auto add = [&](int i, const float (&of)[8]) {
    const int r = i / eights, h0 = (i - r * eights) * 8;
    const RowRange range = row_range(p.s, u, r);
    if (j >= range.pre && (j < range.lo || j >= range.hi)) return;
    const float inv = 0.69314718055994531f / (float)range.count();
    const float* lse = p.lse + (int64_t)(u.row0 + r) * p.n_heads + h0;
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (h0 + k < p.n_heads) sum += weight_of<SOFTMAX>(of[k] - (SOFTMAX ? lse[k] : 0.f), inv);
  };
  if (n > 0) load(0, x[0]);      // (users without rows have no scores)
  for (int i = 0; i < n; i += 2) {
    if (i + 1 < n) load(i + 1, x[1]);
    add(i, x[0]);
    if (i + 1 >= n) break;
    if (i + 2 < n) load(i + 2, x[0]);
    add(i + 1, x[1]);
  }
  p.weight_out[u.token0 + j] = (p.weight_in ? p.weight_in[u.token0 + j] : 0.f) + sum;
}

// From K and q again: a workgroup to a tile, whose wavefronts share the user's (head, row block) pairs and add up over them in registers; the next pair's rows are on their
// way while one is worked on.  What bounds it is the vector ALU, 14 instructions a score: 32 users of 200 to 1000 rows over about 4096 keys, d = 512, cap and bias (561 M scores) 278 us, the users
// of most rows first (334 in another order, the ALU issuing in 87 % of the units' cycles); eight wavefronts a workgroup took 456 where four took 394.  With a bias at d_head 64 the 168 registers of
// three wavefronts a SIMD do not hold everything: 13 words (SiLU form) or 16 are in scratch.  Rows are asked for their ranges after their products, so that masks save the scores and not the
// products: 16 users of 200 rows over 8192 keys, d = 512, 73 us (of a call's 162) if all see all, 75 with a window of 2000 or 81 with sessions of 400, where the attention itself falls from 89 to 29 and 16.
constexpr int kWeighWaves = 4;
template <typename H, int DH, bool SOFTMAX, bool BIAS, int USERS>
__global__ __launch_bounds__(kWeighWaves * 64, DH == 128 ? 2 : 3) void weigh8_kernel(WeighParams<USERS> p) {
  constexpr int KS = DH / 16, KP = DH / 32, BLOCK = kTile * DH;
  __shared__ float join[kWeighWaves][kTile];
  __shared__ __attribute__((aligned(16))) uint32_t words[kWeighWaves][kTile];
  const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, g = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), unit = (int)blockIdx.x;
  const ScoredUser u = whole_user(user_of(p.users, p.n_users, unit, lane, [](const ScoredUserShort& x) { return x.item0; }));
  const int t = unit - u.item0, first = t * kTile, end = first + kTile;
  const char* tile = p.slab + (int64_t)u.page0 * p.page_bytes + (int64_t)t * p.tile_stride;
  const int blocks = (u.rows + 31) / 32;
  const int64_t pairs = (int64_t)blocks * p.n_heads;
  const int64_t at0 = pairs * wave / kWeighWaves, at1 = pairs * (wave + 1) / kWeighWaves;
  float sum[2][16];
#pragma unroll
  for (int kb = 0; kb < 2; ++kb)
#pragma unroll
    for (int e = 0; e < 16; ++e) sum[kb][e] = 0.f;
  if (at0 < at1) {
    int head = (int)(at0 / blocks), block = (int)(at0 - (int64_t)head * blocks);
    u32x4_t kf[2][KS];
    uint4 q[KS];
    float lse = 0.f;
    auto load_rows = [&](int h, int b) {
      const int64_t row = u.row0 + min(b * 32 + l32, u.rows - 1);
      const uint16_t* qr = p.q + row * p.q_stride + h * DH + g * 8;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) q[ks] = *reinterpret_cast<const uint4*>(qr + ks * 16);
      if constexpr (SOFTMAX) lse = p.lse[row * p.n_heads + h];
    };
    load_rows(head, block);
    const int key_place = BIAS && p.s.key_position ? p.s.key_position[u.token0 + min(first + lane, u.keys - 1)] : first + lane;
    bool fresh = true;
    for (int64_t at = at0; at < at1; ++at) {
      if (fresh) {
        const char* codes = tile + (int64_t)head * (2 * BLOCK);
        const float scale = *reinterpret_cast<const float*>(tile + p.scales_off + head * 8);
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
          for (int kp = 0; kp < KP; ++kp) {
            const uint4 c = load16<false>(codes + (kb * KP + kp) * 1024 + lane * 16);
            kf[kb][2 * kp] = fp8_frag<H>(c.x, c.y, scale);
            kf[kb][2 * kp + 1] = fp8_frag<H>(c.z, c.w, scale);
          }
        fresh = false;
      }
      const bool is_row = block * 32 + l32 < u.rows;
      const int i = min(block * 32 + l32, u.rows - 1);
      f32x16_t s[2];
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
#pragma unroll
        for (int e = 0; e < 16; ++e) s[kb][e] = 0.f;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) s[kb] = H::mfma(kf[kb][ks], q[ks], s[kb]);
      }
      const float of_row = lse;
      const bool folded = __builtin_amdgcn_ballot_w64(fabsf(of_row) > kFoldOff) == 0;
      const int head_now = head, block_now = block;
      if (++block == blocks) { block = 0; ++head; fresh = true; }
      __builtin_amdgcn_sched_barrier(0);      // (the next rows take these ones' registers)
      if (at + 1 < at1) load_rows(head, block);
      const RowRange range = row_range(p.s, u, i);
      // (of the lane's row: whether it sees all tokens of the tile, or any)
      const bool all = end <= range.pre || (end <= range.hi && first >= range.from());
      const bool any = first < range.pre || (first < range.hi && end > range.lo);
      if (__builtin_amdgcn_ballot_w64(is_row && any) != 0) {
        const bool masked = __builtin_amdgcn_ballot_w64(!all || !is_row) != 0;
        const float inv = 0.69314718055994531f / (float)range.count();
        const int place_of = BIAS ? row_place(p.s, u, i) : 0;
        Bias bias = {};
        bool behind = true;
        if constexpr (BIAS) {
          bias = bias_of(p.s, u, head_now, block_now * 32, 32, place_of);
          words[wave][lane] = bias.word(key_place);
          behind = bias.behind(key_place);
          __builtin_amdgcn_wave_barrier();
        }
        auto halves = [&](auto kind) {
#pragma unroll
          for (int kb = 0; kb < 2; ++kb) {
            scores_of<decltype(kind)::value>(p.s, bias, place_of, folded ? of_row : 0.f, behind, words[wave] + kb * 32 + 4 * g, s[kb]);
            if (!folded) {
#pragma unroll
              for (int e = 0; e < 16; ++e) s[kb][e] -= of_row;
            }
#pragma unroll
            for (int e = 0; e < 16; ++e) s[kb][e] = weight_of<SOFTMAX>(s[kb][e], inv);
            if (masked) {
              const uint32_t bits = is_row ? seen_bits(range, first + kb * 32, 4 * g) : 0;
#pragma unroll
              for (int e = 0; e < 16; ++e) s[kb][e] = seen_or(bits, e, s[kb][e], 0.f);
            }
#pragma unroll
            for (int e = 0; e < 16; ++e) sum[kb][e] += s[kb][e];
            __builtin_amdgcn_sched_barrier(0);
          }
        };
        if constexpr (!BIAS) halves(std::integral_constant<ScoreKind, kPlain>());
        else if (bias.tight) halves(std::integral_constant<ScoreKind, kTightBias>());
        else halves(std::integral_constant<ScoreKind, kAnyBias>());
      }
    }
  }
#pragma unroll
  for (int kb = 0; kb < 2; ++kb)
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const float x = lanes32_sum(sum[kb][e]);
      if (l32 == 0) join[wave][kb * 32 + 8 * (e >> 2) + 4 * g + (e & 3)] = x;
    }
  __syncthreads();
  if (tid < kTile && first + tid < u.keys) {
    float x = 0.f;
#pragma unroll
    for (int w = 0; w < kWeighWaves; ++w) x += join[w][tid];
    const int64_t j = u.token0 + first + tid;
    p.weight_out[j] = (p.weight_in ? p.weight_in[j] : 0.f) + x;
  }
}

}  // namespace relaygr
