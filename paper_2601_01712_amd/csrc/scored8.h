// Attention of query rows over the 8-bit K/V cache (kv8.h) with scores that are capped or biased, masks that are ranges of tokens, and the weight that each
// token received.  Row i of user u, at position p_i, sees the first `prefix` tokens of the user's entry and those in [first_i, end_i):
//     t_ij = alpha <q_i, k_j>,   t <- cap tanh(t / cap),   t <- t - slope_h |p_i - p_j|
//     softmax form  w_ij = exp(t_ij) / sum_j exp(t_ij)        SiLU form  w_ij = SiLU(t_ij) / n_i, n_i the tokens that the row sees
//     o_i = sum_j w_ij v_j        (0 where n_i = 0)           W_j <- W_j + sum over heads and rows of |w_ij|
// Products, operand layouts and roundings are those of attend8.h; scores are in units of ln 2.  cap tanh(t / cap) = cap - 2 cap / (1 + exp(2 t / cap)): an exp2 and a
// reciprocal, off by 2^-23 of the cap at most, and nothing where the score is beyond fp32.  Caps above kCapSeries, where that would be felt in small scores, take the
// power series of tanh up to 0.3 as well.
//
// Tokens' weights need the sums that a row ends with, so that a second kernel adds them up: from the scores, where the first left them in scratch (few rows: 4 bytes
// a score instead of d_head codes of K), or from K and q again.  It adds in one order, one workgroup to a token: no atomics.
#pragma once

#include "attend8.h"

namespace relaygr {

constexpr int kScoredUsers = 64, kFewScoredUsers = 16;
constexpr float kCapSeries = 128.0f;
struct ScoredUser {
  int32_t page0;       // the entry's first page in the slab
  int32_t row0, rows;  // the user's rows in q and out
  int32_t keys;        // tokens that take part
  int32_t item0;       // items of the launch's users before it, for one head
  int32_t part0;       // first of its rows in the table of partial sums
  int32_t parts;       // pieces that the tiles of each item are cut into
  int32_t prefix;      // tokens that all of its rows see (at most keys)
  int64_t token0;      // where its tokens stand in key_position and the weights
  int64_t saved0;      // where its scores stand in `saved`, [head][row][saved_keys]
  __host__ __device__ __forceinline__ int64_t saved_keys() const { return ((int64_t)keys + kTile - 1) / kTile * kTile; }
};
// What scores and masks go by, the same for all kernels of a call.
struct Scoring {
  const float* slopes;               // [heads], or null
  const int32_t *row_position, *key_position, *row_first, *row_end;     // or null
  int32_t causal, window;
  float score_mul;                   // alpha * log2(e)
  float cap, cap_mul;                // cap * log2(e), 2 alpha log2(e) / cap; cap = 0: none
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
  float* saved;                      // scores, or null
  uint32_t* arrived;                 // as AttendParams'
  int32_t n_users, n_items, d, n_heads;
  Scoring s;
  ScoredUser users[USERS];
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
  r.pre = u.prefix;
  r.lo = max(first, r.pre);
  r.hi = max(end, r.lo);
  return r;
}
__device__ __forceinline__ int row_place(const Scoring& s, const ScoredUser& u, int i) {
  return s.row_position ? s.row_position[u.row0 + i] : s.causal ? u.keys - u.rows + i : u.keys;
}
__device__ __forceinline__ int wave_max_i32(int v) { return (int)(wave_max_u32((uint32_t)v ^ 0x80000000u) ^ 0x80000000u); }
__device__ __forceinline__ int wave_min_i32(int v) { return ~wave_max_i32(~v); }

// Which tiles the rows of a wavefront see (32 * NQ rows, a lane's in range[]; those that are none sees[] = false), and of a tile whether all of them see all of it.
struct TileRange {
  int pre_tiles, t0, n;              // the prefix's tiles, and behind them the tiles from t0 on: n together
  int pre, all_from, all_hi;
  __device__ __forceinline__ int tile(int v) const { return v < pre_tiles ? v : t0 + v - pre_tiles; }
  __device__ __forceinline__ bool whole(int t) const {
    const int a = t * kTile, b = a + kTile;
    return b <= pre || (b <= all_hi && a >= all_from);
  }
};
template <int NQ>
__device__ __forceinline__ TileRange tile_range(const RowRange (&r)[NQ], const bool (&is_row)[NQ], int pre) {
  int lo = 0x7FFFFFFF, hi = 0, from = 0, all_hi = 0x7FFFFFFF;
#pragma unroll
  for (int q = 0; q < NQ; ++q)
    if (is_row[q]) {
      if (r[q].hi > r[q].lo) { lo = min(lo, r[q].lo); hi = max(hi, r[q].hi); }
      from = max(from, r[q].from());
      all_hi = min(all_hi, r[q].hi);
    }
  TileRange t;
  t.pre = pre;
  t.pre_tiles = (pre + kTile - 1) / kTile;
  hi = wave_max_i32(hi);
  t.t0 = max(wave_min_i32(lo) / kTile, t.pre_tiles);
  t.n = t.pre_tiles + max((hi + kTile - 1) / kTile - t.t0, 0);
  t.all_from = wave_max_i32(from);
  t.all_hi = wave_min_i32(all_hi);
  return t;
}

// Scores of a half tile from the products: element e is token place + 8 * (e / 4) + e % 4 of the entry (place includes the lane's 4g).
__device__ __forceinline__ float tanh_series(float x) {
  const float y = x * x;
  return x * fmaf(y, fmaf(y, fmaf(y, fmaf(y, 2.1869488e-2f, -5.3968254e-2f), 1.3333333e-1f), -3.3333333e-1f), 1.0f);
}
template <int NQ>
__device__ __forceinline__ void scores_of(const Scoring& c, f32x16_t (&s)[NQ]) {
  if (c.cap == 0.0f) {
#pragma unroll
    for (int q = 0; q < NQ; ++q)
#pragma unroll
      for (int e = 0; e < 16; ++e) s[q][e] *= c.score_mul;
  } else if (!c.cap_series) {
#pragma unroll
    for (int q = 0; q < NQ; ++q)
#pragma unroll
      for (int e = 0; e < 16; ++e)
        s[q][e] = fmaf(-2.0f * c.cap, __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(s[q][e] * c.cap_mul)), c.cap);
  } else {
#pragma unroll
    for (int q = 0; q < NQ; ++q)
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const float x2 = s[q][e] * c.cap_mul, x = x2 * 0.34657359027997264f;       // 2 x log2(e), x = score / cap
        const float far = fmaf(-2.0f * c.cap, __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(x2)), c.cap);
        s[q][e] = fabsf(x) < 0.3f ? c.cap * tanh_series(x) : far;
      }
  }
}
typedef int i32x4_any_t __attribute__((ext_vector_type(4), aligned(4)));
// The bias by distance.  slope: in units of ln 2; place_of[]: the rows' positions.
template <int NQ>
__device__ __forceinline__ void bias_of(const Scoring& c, const ScoredUser& u, float slope, const int (&place_of)[NQ], int place, bool inside, f32x16_t (&s)[NQ]) {
  if (c.key_position) {
    const int32_t* at = c.key_position + u.token0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      i32x4_any_t k;
      if (inside) {
        k = *reinterpret_cast<const i32x4_any_t*>(at + place + 8 * i);
      } else {      // (the last tile: no reads behind the last token)
#pragma unroll
        for (int j = 0; j < 4; ++j) k[j] = at[min(place + 8 * i + j, u.keys - 1)];
      }
#pragma unroll
      for (int q = 0; q < NQ; ++q)
#pragma unroll
        for (int j = 0; j < 4; ++j) s[q][4 * i + j] = fmaf(-slope, fabsf((float)(place_of[q] - k[j])), s[q][4 * i + j]);
    }
  } else {
#pragma unroll
    for (int q = 0; q < NQ; ++q) {
      const float apart = (float)(place_of[q] - place);
#pragma unroll
      for (int e = 0; e < 16; ++e) s[q][e] = fmaf(-slope, fabsf(apart - (float)(8 * (e >> 2) + (e & 3))), s[q][e]);
    }
  }
}
// Whether a row sees element e of a half tile whose element 0 is token `place`.
__device__ __forceinline__ bool sees(const RowRange& r, int place, int e) {
  const int j = place + 8 * (e >> 2) + (e & 3);
  return j < r.pre || (j >= r.lo && j < r.hi);
}

// attend8_nans for tokens that rows see or not one by one.
template <int NQ>
__device__ __forceinline__ void scored8_nans(uint4& chunk, f32x16_t (&o)[NQ], const RowRange (&r)[NQ], int place) {
  const uint32_t big = 0x7180;          // 2^100 in bf16
#pragma unroll
  for (int m = 0; m < 2; ++m) {
    uint32_t &w0 = m == 0 ? chunk.x : chunk.z, &w1 = m == 0 ? chunk.y : chunk.w;
    const uint32_t n0 = fp8_nans(w0), n1 = fp8_nans(w1);
    w0 &= ~(n0 * 0xFFu);
    w1 &= ~(n1 * 0xFFu);
    const u32x4_t pos = fp8_frag<Bf16>(n0 * 0x38u, n1 * 0x38u, 0x1p100f), neg = fp8_frag<Bf16>(n0 * 0xB8u, n1 * 0xB8u, 0x1p100f);   // codes of 1 and -1
#pragma unroll
    for (int qb = 0; qb < NQ; ++qb) {
      uint32_t see[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) see[j] = (sees(r[qb], place, 8 * m + 2 * j) ? big : 0u) | (sees(r[qb], place, 8 * m + 2 * j + 1) ? big << 16 : 0u);
      const uint4 seen = make_uint4(see[0], see[1], see[2], see[3]);
      o[qb] = Bf16::mfma(neg, seen, Bf16::mfma(pos, seen, o[qb]));
    }
    __builtin_amdgcn_sched_barrier(0);
  }
}

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
  it->u = user_of(p.users, p.n_users, item, lane, [](const ScoredUser& x) { return x.item0; });
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

// Writes a wavefront's 32 * NQ rows, as attend8_store.
template <typename H, int DH, int NQ, bool SOFTMAX, int USERS>
__device__ __forceinline__ void scored8_store(const ScoredParams<USERS>& p, const ScoredItem& it, int lane, const RowRange (&range)[NQ], f32x16_t (&o)[DH / 32][NQ],
                                              const float (&mref)[NQ], const float (&lane_sum)[NQ], const float (&lane_exact)[NQ]) {
  constexpr int DB = DH / 32;
  const int l32 = lane & 31, g = lane >> 5;
#pragma unroll
  for (int qb = 0; qb < NQ; ++qb) {
    const int r = qb * 32 + l32;
    const float lsum = SOFTMAX ? lane_sum[qb] + __shfl_xor(lane_sum[qb], 32, 64) : 0.f;
    const float exact = SOFTMAX ? lane_exact[qb] + __shfl_xor(lane_exact[qb], 32, 64) : 0.f;
    if (r >= it.n_rows) continue;
    const int seen = range[qb].count();
    const int64_t row = it.u.row0 + it.first_row + r;
    if (it.u.parts == 1) {
      const float mul = SOFTMAX ? 1.0f / lsum : 0.69314718055994531f / (float)seen;
      uint16_t* dst = p.out + row * p.out_stride + it.head * DH + 4 * g;
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int e4 = 0; e4 < 4; ++e4) {
          uint2 w = make_uint2(H::pack2(o[db][qb][4 * e4] * mul, o[db][qb][4 * e4 + 1] * mul), H::pack2(o[db][qb][4 * e4 + 2] * mul, o[db][qb][4 * e4 + 3] * mul));
          if (seen == 0) w = make_uint2(0, 0);
          *reinterpret_cast<uint2*>(dst + db * 32 + 8 * e4) = w;
        }
      if constexpr (SOFTMAX) {
        if (p.lse && g == 0) p.lse[row * p.n_heads + it.head] = mref[qb] + __builtin_amdgcn_logf(exact);
      }
    } else {
      const int64_t pr = (int64_t)it.u.part0 + (int64_t)it.piece * it.u.rows + it.first_row + r;
      float* dst = p.part + pr * p.d + it.head * DH + 4 * g;
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int e4 = 0; e4 < 4; ++e4)
          *reinterpret_cast<float4*>(dst + db * 32 + 8 * e4) = make_float4(o[db][qb][4 * e4], o[db][qb][4 * e4 + 1], o[db][qb][4 * e4 + 2], o[db][qb][4 * e4 + 3]);
      if constexpr (SOFTMAX) {
        if (g == 0) p.ml[pr * p.n_heads + it.head] = make_float4(mref[qb], lsum, exact, 0.f);
      }
    }
  }
}

// Joins the pieces of an item's rows in the workgroup that is the last of them to arrive, as attend8_join_last.
template <typename H, int DH, bool SOFTMAX, int USERS>
__device__ __forceinline__ void scored8_join_last(const ScoredParams<USERS>& p, const ScoredItem& it, int wave, int lane) {
  constexpr int LANES = DH / 4, GROUPS = 64 / LANES;
  __shared__ int last;
  if (wave == 0) {
    uint32_t* count = p.arrived + (it.u.item0 + it.first_row / 32) * p.n_heads + it.head;
    if (lane == 0) {      // (the release is of all the wavefront's stores)
      const uint32_t before = __hip_atomic_fetch_add(count, 1u, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT);
      last = before + 1 == (uint32_t)it.u.parts;
      if (last) *count = 0;
    }
  }
  __syncthreads();
  if (!last) return;
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "agent");
  const int group = lane / LANES, f = it.head * DH + (lane % LANES) * 4, parts = it.u.parts;
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

// One item, as attend8_kernel: the workgroup's wavefronts take its tiles in turn, each straight from memory to its registers.
template <typename H, int DH, int NQ, bool SOFTMAX, bool ONCE, int USERS>
__global__ __launch_bounds__(kAttendWaves * 64, 2) void scored8_kernel(ScoredParams<USERS> p) {
  constexpr int KS = DH / 16, KP = DH / 32, DB = DH / 32;
  constexpr int BLOCK = kTile * DH;            // bytes of codes of K, and of V
  constexpr int SUMS = SOFTMAX ? 3 * NQ : 0;
  __shared__ float join[kAttendWaves / 2][(DB * NQ * 16 + SUMS) * 64];
  const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, g = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  ScoredItem it;
  if (!scored8_item<32 * NQ>(p, lane, &it)) return;
  const ScoredUser& u = it.u;
  const int head = it.head, first_row = it.first_row, n_rows = it.n_rows;

  RowRange range[NQ];
  bool is_row[NQ];
  int place_of[NQ];
  uint4 qf[NQ][KS];
#pragma unroll
  for (int qb = 0; qb < NQ; ++qb) {
    const int r = qb * 32 + l32;
    is_row[qb] = r < n_rows;
    const int i = first_row + (is_row[qb] ? r : 0);
    range[qb] = row_range(p.s, u, i);
    place_of[qb] = p.s.slopes ? row_place(p.s, u, i) : 0;
    const uint16_t* qr = p.q + (int64_t)(u.row0 + i) * p.q_stride + head * DH + g * 8;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) qf[qb][ks] = *reinterpret_cast<const uint4*>(qr + ks * 16);
  }
  const float slope = p.s.slopes ? p.s.slopes[head] * 1.4426950408889634f : 0.f;
  const TileRange tiles = tile_range(range, is_row, u.prefix);
  const int v0 = (int)((int64_t)it.piece * tiles.n / u.parts), v1 = (int)((int64_t)(it.piece + 1) * tiles.n / u.parts);

  f32x16_t oacc[DB][NQ];
  float mref[NQ], lsum[NQ], lexact[NQ];
#pragma unroll
  for (int qb = 0; qb < NQ; ++qb) {
    mref[qb] = -INFINITY; lsum[qb] = 0.f; lexact[qb] = 0.f;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int e = 0; e < 16; ++e) oacc[db][qb][e] = 0.f;
  }

  const char* kv = p.slab + (int64_t)u.page0 * p.page_bytes;
  const char* base = kv + (int64_t)head * (2 * BLOCK);
  const char* scales = kv + p.scales_off + head * 8;
  uint4 kr[2][KP], vr[2][DB];                   // codes of the tile's two halves
  float2 sc;
  auto load_k = [&](int t, int kb) {
    const char* tile = base + (int64_t)t * p.tile_stride;
#pragma unroll
    for (int kp = 0; kp < KP; ++kp) kr[kb][kp] = load16<ONCE>(tile + (kb * KP + kp) * 1024 + lane * 16);
  };
  auto load_v = [&](int t, int kb) {
    const char* tile = base + (int64_t)t * p.tile_stride + BLOCK;
#pragma unroll
    for (int db = 0; db < DB; ++db) vr[kb][db] = load16<ONCE>(tile + (db * 2 + kb) * 1024 + lane * 16);
  };
  auto load_scales = [&](int t) { return *reinterpret_cast<const float2*>(scales + (int64_t)t * p.tile_stride); };

  // one tile, half by half; each piece of codes makes room for the wavefront's next tile (tn) as soon as it has been converted
  auto tile = [&](auto more_tag, int t, int tn) {
    constexpr bool MORE = decltype(more_tag)::value;
    float2 sn = sc;
    if constexpr (MORE) sn = load_scales(tn);
    const bool whole = tiles.whole(t), inside = (t + 1) * kTile <= u.keys;
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
      const int place = t * kTile + kb * 32 + 4 * g;
      f32x16_t s[NQ];
#pragma unroll
      for (int qb = 0; qb < NQ; ++qb)
#pragma unroll
        for (int e = 0; e < 16; ++e) s[qb][e] = 0.f;
#pragma unroll
      for (int kp = 0; kp < KP; ++kp) {
        const u32x4_t lo = fp8_frag<H>(kr[kb][kp].x, kr[kb][kp].y, sc.x), hi = fp8_frag<H>(kr[kb][kp].z, kr[kb][kp].w, sc.x);
#pragma unroll
        for (int qb = 0; qb < NQ; ++qb) s[qb] = H::mfma(lo, qf[qb][2 * kp], s[qb]);
#pragma unroll
        for (int qb = 0; qb < NQ; ++qb) s[qb] = H::mfma(hi, qf[qb][2 * kp + 1], s[qb]);
      }
      if constexpr (MORE) load_k(tn, kb);
      __builtin_amdgcn_sched_barrier(0);
      scores_of<NQ>(p.s, s);
      if (p.s.slopes) bias_of<NQ>(p.s, u, slope, place_of, place, inside, s);
      if (p.saved) {
#pragma unroll
        for (int qb = 0; qb < NQ; ++qb) {
          const int r = qb * 32 + l32;
          if (r < n_rows) {
            float* to = p.saved + u.saved0 + ((int64_t)head * u.rows + first_row + r) * u.saved_keys() + place;
#pragma unroll
            for (int i = 0; i < 4; ++i) *reinterpret_cast<float4*>(to + 8 * i) = make_float4(s[qb][4 * i], s[qb][4 * i + 1], s[qb][4 * i + 2], s[qb][4 * i + 3]);
          }
        }
      }
      if (!whole) {
        uint32_t any = 0;
#pragma unroll
        for (int qb = 0; qb < NQ; ++qb)
#pragma unroll
          for (int e = 0; e < 16; ++e) s[qb][e] = sees(range[qb], place, e) ? s[qb][e] : (SOFTMAX ? -INFINITY : 0.f);   // (SiLU(0) = 0)
#pragma unroll
        for (int db = 0; db < DB; ++db) any |= fp8_nans(vr[kb][db].x) | fp8_nans(vr[kb][db].y) | fp8_nans(vr[kb][db].z) | fp8_nans(vr[kb][db].w);
        if (__builtin_amdgcn_ballot_w64(any != 0) != 0) {
          int at = place;
          asm volatile("" : "+v"(at));      // (its compares are made here, not kept in registers from the ones above)
#pragma unroll
          for (int db = 0; db < DB; ++db) scored8_nans<NQ>(vr[kb][db], oacc[db], range, at);
        }
      }
      uint32_t pk[NQ][8];
      if constexpr (SOFTMAX) {
        // the rows' reference scores follow the largest seen score at a distance of at most kSlack, in which exp2 still fits either type
        constexpr float kSlack = 8.0f;
        float mx[NQ];
        bool need = false;
#pragma unroll
        for (int qb = 0; qb < NQ; ++qb) {
          mx[qb] = -INFINITY;
#pragma unroll
          for (int e = 0; e < 16; ++e) mx[qb] = fmaxf(mx[qb], s[qb][e]);
          need |= mx[qb] > mref[qb] + kSlack;
        }
        if (__builtin_amdgcn_ballot_w64(need) != 0) {
#pragma unroll
          for (int qb = 0; qb < NQ; ++qb) {
            const float mn = fmaxf(mref[qb], fmaxf(mx[qb], __shfl_xor(mx[qb], 32, 64)));
            const float c = mn == mref[qb] ? 1.0f : __builtin_amdgcn_exp2f(mref[qb] - mn);     // from -inf: 0
            mref[qb] = mn;
            lsum[qb] *= c;
            lexact[qb] *= c;
#pragma unroll
            for (int db = 0; db < DB; ++db)
#pragma unroll
              for (int e = 0; e < 16; ++e) oacc[db][qb][e] *= c;
          }
        }
#pragma unroll
        for (int qb = 0; qb < NQ; ++qb) {
          const float m = mref[qb] == -INFINITY ? 0.f : mref[qb];      // (a row that has seen nothing: weights exp2(-inf) = 0)
#pragma unroll
          for (int e = 0; e < 16; e += 2) {
            const float a = __builtin_amdgcn_exp2f(s[qb][e] - m), b = __builtin_amdgcn_exp2f(s[qb][e + 1] - m);
            pk[qb][e >> 1] = H::pack2(a, b);
            lsum[qb] = H::dot2(pk[qb][e >> 1], H::kOnes, lsum[qb]);       // of the weights that the second product takes
            lexact[qb] += a + b;
          }
        }
      } else {
#pragma unroll
        for (int qb = 0; qb < NQ; ++qb)
#pragma unroll
          for (int e = 0; e < 16; e += 2) {     // SiLU(t) / ln 2
            const float ta = s[qb][e], tb = s[qb][e + 1];
            pk[qb][e >> 1] = H::pack2(ta * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-ta)), tb * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-tb)));
          }
      }
#pragma unroll
      for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int db = 0; db < DB; ++db) {
          const u32x4_t vf = m == 0 ? fp8_frag<H>(vr[kb][db].x, vr[kb][db].y, sc.y) : fp8_frag<H>(vr[kb][db].z, vr[kb][db].w, sc.y);
#pragma unroll
          for (int qb = 0; qb < NQ; ++qb)
            oacc[db][qb] = H::mfma(vf, make_uint4(pk[qb][4 * m], pk[qb][4 * m + 1], pk[qb][4 * m + 2], pk[qb][4 * m + 3]), oacc[db][qb]);
        }
      if constexpr (MORE) load_v(tn, kb);
      __builtin_amdgcn_sched_barrier(0);
    }
    sc = sn;
  };
  int v = v0 + wave;
  if (v < v1) {
    int t = tiles.tile(v);
    sc = load_scales(t);
    load_k(t, 0);
    load_v(t, 0);
    load_k(t, 1);
    load_v(t, 1);
    for (; v + kAttendWaves < v1; v += kAttendWaves) {
      const int tn = tiles.tile(v + kAttendWaves);
      tile(std::true_type(), t, tn);
      t = tn;
    }
    tile(std::false_type(), t, t);
  }

  // the wavefronts' sums: upper half to lower half, twice (a fixed order)
#pragma unroll
  for (int half = kAttendWaves / 2; half >= 1; half >>= 1) {
    if (wave >= half && wave < 2 * half) {
      float* x = join[wave - half];
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int qb = 0; qb < NQ; ++qb)
#pragma unroll
          for (int e = 0; e < 16; ++e) x[((db * NQ + qb) * 16 + e) * 64 + lane] = oacc[db][qb][e];
      if constexpr (SOFTMAX) {
#pragma unroll
        for (int qb = 0; qb < NQ; ++qb) {
          x[(DB * NQ * 16 + 3 * qb) * 64 + lane] = mref[qb];
          x[(DB * NQ * 16 + 3 * qb + 1) * 64 + lane] = lsum[qb];
          x[(DB * NQ * 16 + 3 * qb + 2) * 64 + lane] = lexact[qb];
        }
      }
    }
    __syncthreads();
    if (wave < half) {
      const float* x = join[wave];
#pragma unroll
      for (int qb = 0; qb < NQ; ++qb) {
        float c0 = 1.0f, c1 = 1.0f;
        if constexpr (SOFTMAX) {
          const float m1 = x[(DB * NQ * 16 + 3 * qb) * 64 + lane], M = fmaxf(mref[qb], m1);
          c0 = mref[qb] == M ? 1.0f : __builtin_amdgcn_exp2f(mref[qb] - M);
          c1 = m1 == M ? 1.0f : __builtin_amdgcn_exp2f(m1 - M);
          lsum[qb] = lsum[qb] * c0 + x[(DB * NQ * 16 + 3 * qb + 1) * 64 + lane] * c1;
          lexact[qb] = lexact[qb] * c0 + x[(DB * NQ * 16 + 3 * qb + 2) * 64 + lane] * c1;
          mref[qb] = M;
        }
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const float y = x[((db * NQ + qb) * 16 + e) * 64 + lane];
            if constexpr (SOFTMAX) oacc[db][qb][e] = oacc[db][qb][e] * c0 + y * c1;
            else oacc[db][qb][e] += y;
          }
      }
    }
    __syncthreads();
  }
  if (wave == 0) scored8_store<H, DH, NQ, SOFTMAX>(p, it, lane, range, oacc, mref, lsum, lexact);
  if constexpr (USERS <= kFewScoredUsers) {
    if (p.arrived != nullptr && u.parts > 1) scored8_join_last<H, DH, SOFTMAX>(p, it, wave, lane);
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
  const ScoredUser u = user_of(p.users, p.n_users, row, lane, [](const ScoredUser& x) { return x.item0; });
  const int r = row - u.item0;
  const bool mine = f < p.d;           // (d = 128: half of the lanes)
  const int head = (mine ? f : 0) / DH;
  const float* x = p.part + ((int64_t)u.part0 + r) * p.d + (mine ? f : 0);
  const int64_t step = (int64_t)u.rows * p.d;      // between a row's pieces
  ScoredSum<SOFTMAX> sum[GROUPS];
  for (int k0 = 0; k0 < u.parts; k0 += 8) {
    float4 v[8], ml[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const int kk = min(k0 + k, u.parts - 1);
      v[k] = *reinterpret_cast<const float4*>(x + kk * step);
      ml[k] = SOFTMAX ? p.ml[((int64_t)u.part0 + (int64_t)kk * u.rows + r) * p.n_heads + head] : make_float4(0.f, 0.f, 0.f, 0.f);
    }
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (k0 + k < u.parts) sum[k % GROUPS].add(v[k], ml[k].x, ml[k].y, ml[k].z);
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
  const float* weight_in;            // or null: zero
  float* weight_out;
  int32_t n_users, n_units, d, n_heads;
  Scoring s;
  ScoredUser users[USERS];           // item0: units of the launch's users before it
};
// |w| of a score.  lse: softmax form, of the row; inv: SiLU form, ln 2 / n.
template <bool SOFTMAX>
__device__ __forceinline__ float weight_of(float t, float lse, float inv) {
  return SOFTMAX ? __builtin_amdgcn_exp2f(t - lse) : fabsf(t * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-t))) * inv;
}

// From the scores that the attention kernel left, a token to a lane: units of 256 tokens.
template <bool SOFTMAX, int USERS>
__global__ __launch_bounds__(256) void weigh8_saved_kernel(WeighParams<USERS> p) {
  const int lane = threadIdx.x & 63, unit = (int)blockIdx.x;
  const ScoredUser u = user_of(p.users, p.n_users, unit, lane, [](const ScoredUser& x) { return x.item0; });
  const int j = (unit - u.item0) * 256 + (int)threadIdx.x;
  if (j >= u.keys) return;
  const int64_t keys = u.saved_keys();
  const float* at = p.saved + u.saved0 + j;
  float sum = 0.f;
  for (int r = 0; r < u.rows; ++r) {
    const RowRange range = row_range(p.s, u, r);
    if (j >= range.pre && (j < range.lo || j >= range.hi)) continue;
    const float inv = 0.69314718055994531f / (float)range.count();
    const float* lse = p.lse + (int64_t)(u.row0 + r) * p.n_heads;
    for (int h = 0; h < p.n_heads; ++h) sum += weight_of<SOFTMAX>(at[((int64_t)h * u.rows + r) * keys], SOFTMAX ? lse[h] : 0.f, inv);
  }
  p.weight_out[u.token0 + j] = (p.weight_in ? p.weight_in[u.token0 + j] : 0.f) + sum;
}

// From K and q again: a workgroup to 32 tokens, whose wavefronts share the user's (head, row block) pairs and add up over them in registers.
constexpr int kWeighWaves = 8;
template <typename H, int DH, bool SOFTMAX, int USERS>
__global__ __launch_bounds__(kWeighWaves * 64) void weigh8_kernel(WeighParams<USERS> p) {
  constexpr int KS = DH / 16, KP = DH / 32, BLOCK = kTile * DH;
  __shared__ float join[kWeighWaves][32];
  const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, g = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), unit = (int)blockIdx.x;
  const ScoredUser u = user_of(p.users, p.n_users, unit, lane, [](const ScoredUser& x) { return x.item0; });
  const int half = unit - u.item0, t = half >> 1, kb = half & 1, first = half * 32, place = first + 4 * g;
  const bool inside = first + 32 <= u.keys;
  const char* tile = p.slab + (int64_t)u.page0 * p.page_bytes + (int64_t)t * p.tile_stride;
  const int blocks = (u.rows + 31) / 32;
  const int64_t pairs = (int64_t)blocks * p.n_heads;
  const int64_t at0 = pairs * wave / kWeighWaves, at1 = pairs * (wave + 1) / kWeighWaves;
  float sum[16];
#pragma unroll
  for (int e = 0; e < 16; ++e) sum[e] = 0.f;
  int head = (int)(at0 / blocks), block = (int)(at0 - (int64_t)head * blocks);
  u32x4_t kf[KS];
  float slope = 0.f;
  bool fresh = true;
  for (int64_t at = at0; at < at1; ++at) {
    if (fresh) {
      const char* codes = tile + (int64_t)head * (2 * BLOCK) + kb * KP * 1024;
      const float scale = *reinterpret_cast<const float*>(tile + p.scales_off + head * 8);
#pragma unroll
      for (int kp = 0; kp < KP; ++kp) {
        const uint4 c = load16<false>(codes + kp * 1024 + lane * 16);
        kf[2 * kp] = fp8_frag<H>(c.x, c.y, scale);
        kf[2 * kp + 1] = fp8_frag<H>(c.z, c.w, scale);
      }
      slope = p.s.slopes ? p.s.slopes[head] * 1.4426950408889634f : 0.f;
      fresh = false;
    }
    const int r = block * 32 + l32;
    const bool is_row = r < u.rows;
    const int i = is_row ? r : u.rows - 1;
    const RowRange range = row_range(p.s, u, i);
    // (a lane's tokens: whether its row sees all of the 32, or any)
    const bool all = first + 32 <= range.pre || (first + 32 <= range.hi && first >= range.from());
    const bool any = is_row && (first < range.pre || (first < range.hi && first + 32 > range.lo));
    if (__builtin_amdgcn_ballot_w64(any) != 0) {
      const uint16_t* qr = p.q + (int64_t)(u.row0 + i) * p.q_stride + head * DH + g * 8;
      f32x16_t s[1];
#pragma unroll
      for (int e = 0; e < 16; ++e) s[0][e] = 0.f;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) s[0] = H::mfma(kf[ks], *reinterpret_cast<const uint4*>(qr + ks * 16), s[0]);
      const float lse = SOFTMAX ? p.lse[(int64_t)(u.row0 + i) * p.n_heads + head] : 0.f, inv = 0.69314718055994531f / (float)range.count();
      scores_of<1>(p.s, s);
      if (p.s.slopes) {
        const int place_of[1] = {row_place(p.s, u, i)};
        bias_of<1>(p.s, u, slope, place_of, place, inside, s);
      }
      const bool masked = __builtin_amdgcn_ballot_w64(!all || !is_row) != 0;
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const float w = weight_of<SOFTMAX>(s[0][e], lse, inv);
        sum[e] += masked ? (is_row && sees(range, place, e) ? w : 0.f) : w;
      }
    }
    if (++block == blocks) { block = 0; ++head; fresh = true; }
  }
#pragma unroll
  for (int e = 0; e < 16; ++e) {
    const float x = lanes32_sum(sum[e]);
    if (l32 == 0) join[wave][8 * (e >> 2) + 4 * g + (e & 3)] = x;
  }
  __syncthreads();
  if (tid < 32 && first + tid < u.keys) {
    float x = 0.f;
#pragma unroll
    for (int w = 0; w < kWeighWaves; ++w) x += join[w][tid];
    const int64_t j = u.token0 + first + tid;
    p.weight_out[j] = (p.weight_in ? p.weight_in[j] : 0.f) + x;
  }
}

}  // namespace relaygr
