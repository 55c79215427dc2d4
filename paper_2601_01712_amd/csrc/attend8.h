// Attention of query rows over the 8-bit K/V cache (layout and conversions in kv8.h).  Row i of user u, which sees the first n_i tokens
// of the user's entry:
//     SiLU form     o_i = (1/n_i) sum_{j < n_i} SiLU(alpha <q_i, k_j>) v_j
//     softmax form  o_i = sum_{j < n_i} exp(alpha <q_i, k_j>) v_j / sum_{j < n_i} exp(alpha <q_i, k_j>)
// and o_i = 0 where n_i = 0.  The products are those of the 16-bit kernel (attention.h): S^T = K Q^T, whose accumulator layout is the operand
// layout of the next product, O^T += V^T P^T with P rounded to the storage type, as the MFMA takes it; scores, sums and outputs are fp32.
// Half a step, 2^-8 or 2^-11, of each weight at most, each by itself: where V has a mean the sum grows with the keys and the roundings do not,
// where V is centred on zero they stay beside it at any number of keys, as large together as the output's own (relative error against 64 bits, 20 to
// 2000 keys, bf16 0.0023 in the SiLU form and 0.0020 to 0.0022 in the softmax form, with V of SiLU's shape 0.0019 to 0.0016; the output's rounding
// alone 0.0017.  fp16: an eighth of that).  The rest of the weights in a product of its own would be half of the MFMAs again.  The softmax form's sums are of the rounded
// weights, so that a row is a mean of V whatever they round to: a weight that is most of its row's rounds in the numerator and in the denominator.
//
// What bounds it: few rows, the read of the codes (128 users of one row over 8192 keys, d = 512, 1.07 GB in 161 us: 6.7 TB/s, where a kernel that reads 1 to 4 GiB
// and does nothing else reaches 6.9 to 7.1); many rows, the vector ALU (16 users of 512 rows over 4096 keys, d = 512, SiLU: 68.7 GFLOP in 88 to 94 us by the card, 0.73
// to 0.78 PFLOP/s).  A 64 x 64 tile of scores is 472 vector instructions there, 128 of them exp and rcp; by the counters they issue for 2402 cycles of a SIMD, 4 an instruction
// and 8 an exp or rcp, 79 % of the 3034 that its compute unit is busy for it (the MFMAs' 1024 beside them; 1.77 wavefronts a SIMD of 2 in the mean, the others starting or
// done, 12 % of their time at waits).  A single row: the launch (7.9 us a call, 6.0 of them on the GPU).
// Tiles come straight to registers because nothing else is gained by LDS: codes staged there and converted once for 128 or 256 rows of an item took 96 and
// 99 us where this took 88.
#pragma once

#include "kv8.h"

namespace relaygr {

// Users of a launch: they travel in the kernel's arguments, as RowsParams' do.
constexpr int kAttendUsers = 128, kFewAttendUsers = 16;
constexpr int kAttendWaves = 4;        // wavefronts of a workgroup
struct AttendUser {
  int32_t page0;       // the entry's first page in the slab
  int32_t row0, rows;  // the user's rows in q and out
  int32_t keys;        // tokens that its last row sees (without `causal`: every row)
  int32_t item0;       // items of the launch's users before it, for one head
  int32_t part0;       // first of its rows in the table of partial sums
  uint32_t cut;        // pieces of its key sequence (7 bits), key tiles in each
  __host__ __device__ __forceinline__ int parts() const { return (int)(cut & 127); }
  __host__ __device__ __forceinline__ int per() const { return (int)(cut >> 7); }
};
static_assert(sizeof(AttendUser) == 28, "AttendUser layout");
template <int USERS> struct AttendParams {
  const uint16_t* q;
  uint16_t* out;
  int64_t q_stride, out_stride;      // elements between rows
  const char* slab;                  // of the pool, at the call's layer
  int64_t page_bytes, tile_stride, scales_off;   // bytes: of a page, between tiles, from a tile's codes to its layer's scales
  float* part;                       // [partial rows][d] sums of rows that are cut along the keys
  float* ml;                         // softmax form: [partial rows][n_heads][2] reference score (log2 units) and sum of weights
  int32_t n_users, n_items, d, n_heads, causal;
  float score_mul;                   // alpha * log2(e)
  uint32_t* arrived;                 // few users: pieces of a (row tile, head) that are done, zero between launches; null: a launch of its own joins them
  AttendUser users[USERS];
};
// Tokens that row i of the user sees.
__device__ __forceinline__ int attend_seen(const AttendUser& u, int i, int causal) { return causal ? max(u.keys - u.rows + 1 + i, 0) : u.keys; }

// NaN codes of four, as 0x01 in their bytes.
__device__ __forceinline__ uint32_t fp8_nans(uint32_t codes) { return (((codes & 0x7F7F7F7Fu) + 0x01010101u) >> 7) & 0x01010101u; }

// A tile that not every row sees whole: a weight of zero is no answer to a NaN in V (0 * NaN), which only rows that see its token may get.  NaN codes
// leave the V that the weights are multiplied with, and what is NaN times what is seen is added twice to the sums, as +inf and as -inf: products
// of powers of two beyond fp32 (in bf16 whatever the storage type; fp16 does not reach that far).  `chunk`: V codes (db, kb); vis: tokens of the tile
// that the lane's rows see, less 4g.
template <int NQ>
__device__ __forceinline__ void attend8_nans(uint4& chunk, int kb, f32x16_t (&o)[NQ], const int (&vis)[NQ]) {
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
      for (int j = 0; j < 4; ++j) {
        const int e = 8 * m + 2 * j, key = kb * 32 + 8 * (e >> 2) + (e & 3);
        see[j] = (key < vis[qb] ? big : 0u) | (key + 1 < vis[qb] ? big << 16 : 0u);
      }
      const uint4 sees = make_uint4(see[0], see[1], see[2], see[3]);
      o[qb] = Bf16::mfma(neg, sees, Bf16::mfma(pos, sees, o[qb]));
    }
    __builtin_amdgcn_sched_barrier(0);
  }
}

// An item of the launch: rows of one user, one head, one piece of the key sequence.
struct AttendItem {
  AttendUser u;
  int head, piece, first_row, n_rows;
  int most, least;      // tokens that the last and the first of its rows see
  int t0, t1;           // key tiles
};
// The workgroup's item (ROWS to an item); false: it has none.  Heads are dealt to the XCDs as in attention.h, so that the row tiles of one user and
// head share an L2.
template <int ROWS, int USERS>
__device__ __forceinline__ bool attend8_item(const AttendParams<USERS>& p, int lane, AttendItem* it) {
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
  it->u = user_of(p.users, p.n_users, item, lane, [](const AttendUser& x) { return x.item0; });
  const int row_tiles = (it->u.rows + ROWS - 1) / ROWS;
  it->piece = (item - it->u.item0) / row_tiles;
  it->first_row = (item - it->u.item0 - it->piece * row_tiles) * ROWS;
  it->n_rows = min(ROWS, it->u.rows - it->first_row);
  it->most = attend_seen(it->u, it->first_row + it->n_rows - 1, p.causal);
  it->least = attend_seen(it->u, it->first_row, p.causal);
  it->t0 = it->piece * it->u.per();
  it->t1 = min(it->t0 + it->u.per(), (it->most + kTile - 1) / kTile);
  return true;
}

// Writes a wavefront's 32 * NQ rows: sums over all their keys as outputs, sums of one piece as partial sums.  Element e of o[db][qb]: feature
// db*32 + 8*(e/4) + 4*g + e%4, row qb*32 + l32 of the wavefront's.
template <typename H, int DH, int NQ, bool SOFTMAX, int USERS>
__device__ __forceinline__ void attend8_store(const AttendParams<USERS>& p, const AttendItem& it, int row0, int lane, const int (&seen)[NQ], f32x16_t (&o)[DH / 32][NQ],
                                              const float (&mref)[NQ], const float (&lane_sum)[NQ]) {
  constexpr int DB = DH / 32;
  const int l32 = lane & 31, g = lane >> 5;
#pragma unroll
  for (int qb = 0; qb < NQ; ++qb) {
    const int r = row0 + qb * 32 + l32;
    const float lsum = SOFTMAX ? lane_sum[qb] + __shfl_xor(lane_sum[qb], 32, 64) : 0.f;
    if (r >= it.n_rows) continue;
    if (it.u.parts() == 1) {
      const float mul = SOFTMAX ? 1.0f / lsum : 0.69314718055994531f / (float)seen[qb];
      uint16_t* dst = p.out + (int64_t)(it.u.row0 + it.first_row + r) * p.out_stride + it.head * DH + 4 * g;
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int e4 = 0; e4 < 4; ++e4) {
          uint2 w = make_uint2(H::pack2(o[db][qb][4 * e4] * mul, o[db][qb][4 * e4 + 1] * mul), H::pack2(o[db][qb][4 * e4 + 2] * mul, o[db][qb][4 * e4 + 3] * mul));
          if (seen[qb] == 0) w = make_uint2(0, 0);
          *reinterpret_cast<uint2*>(dst + db * 32 + 8 * e4) = w;
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
        if (g == 0) *reinterpret_cast<float2*>(p.ml + (pr * p.n_heads + it.head) * 2) = make_float2(mref[qb], lsum);
      }
    }
  }
}

// The sums of a row's pieces, four features to a lane.  Pieces are added in 256 / DH groups (piece k in group k mod groups), in their order, and then
// the groups pairwise, lower to upper: one order, whichever of the two joins below a launch takes.
template <bool SOFTMAX> struct PieceSum {
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
  float M = -INFINITY, l = 0.f;
  __device__ __forceinline__ void add(const float4& x, float m, float w) {
    if constexpr (SOFTMAX) {
      const float mn = fmaxf(M, m), c0 = M == mn ? 1.0f : __builtin_amdgcn_exp2f(M - mn), c1 = m == mn ? 1.0f : __builtin_amdgcn_exp2f(m - mn);
      o = make_float4(fmaf(x.x, c1, o.x * c0), fmaf(x.y, c1, o.y * c0), fmaf(x.z, c1, o.z * c0), fmaf(x.w, c1, o.w * c0));
      l = fmaf(w, c1, l * c0);
      M = mn;
    } else {
      o = make_float4(o.x + x.x, o.y + x.y, o.z + x.z, o.w + x.w);
    }
  }
  template <typename H> __device__ __forceinline__ uint2 out(int seen) const {
    const float mul = SOFTMAX ? 1.0f / l : 0.69314718055994531f / (float)seen;
    return seen == 0 ? make_uint2(0, 0) : make_uint2(H::pack2(o.x * mul, o.y * mul), H::pack2(o.z * mul, o.w * mul));
  }
};

// Joins the pieces of an item's rows in the workgroup that is the last of them to arrive: every workgroup of the item comes here once its partial sums are
// stored by its wavefront 0.  Rows go to the wavefronts in turn, four at a time; a row's groups are side by side in a wavefront.
template <typename H, int DH, bool SOFTMAX, int USERS>
__device__ __forceinline__ void attend8_join_last(const AttendParams<USERS>& p, const AttendItem& it, int wave, int lane) {
  constexpr int LANES = DH / 4, GROUPS = 64 / LANES;
  __shared__ int last;
  if (wave == 0) {
    uint32_t* count = p.arrived + (it.u.item0 + it.first_row / 32) * p.n_heads + it.head;
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
    PieceSum<SOFTMAX> sum[4];
    for (int k = group; k < parts + group; k += GROUPS) {      // (as many turns for every lane)
      float4 x[4];
      float2 ml[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int64_t pr = it.u.part0 + min(k, parts - 1) * step + it.first_row + min(r0 + 4 * i, it.n_rows - 1);
        x[i] = *reinterpret_cast<const float4*>(p.part + pr * p.d + f);
        ml[i] = SOFTMAX ? *reinterpret_cast<const float2*>(p.ml + (pr * p.n_heads + it.head) * 2) : make_float2(0.f, 0.f);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (k < parts) sum[i].add(x[i], ml[i].x, ml[i].y);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
#pragma unroll
      for (int by = LANES; by < 64; by *= 2) {
        PieceSum<SOFTMAX>& a = sum[i];
        const float4 x = make_float4(__shfl_xor(a.o.x, by, 64), __shfl_xor(a.o.y, by, 64), __shfl_xor(a.o.z, by, 64), __shfl_xor(a.o.w, by, 64));
        a.add(x, SOFTMAX ? __shfl_xor(a.M, by, 64) : 0.f, SOFTMAX ? __shfl_xor(a.l, by, 64) : 0.f);
      }
      const int r = r0 + 4 * i;
      if (group == 0 && r < it.n_rows)
        *reinterpret_cast<uint2*>(p.out + (int64_t)(it.u.row0 + it.first_row + r) * p.out_stride + f) =
            sum[i].template out<H>(attend_seen(it.u, it.first_row + r, p.causal));
    }
  }
}

// One item: up to 32*NQ rows of one user, one head, one piece of the key sequence.  The workgroup's wavefronts take the piece's key tiles in turn, all
// for the same rows, each straight from memory to its registers (the codes are in operand order) with the next tile on its way while it
// works on one; their sums meet in LDS at the end.
//
// ONCE: no other item reads the same codes, and the launch reads more than the caches hold: the loads do not leave them there (attend_rules.h has both sides).
template <typename H, int DH, int NQ, bool SOFTMAX, bool ONCE, int USERS>
__global__ __launch_bounds__(kAttendWaves * 64, 2) void attend8_kernel(AttendParams<USERS> p) {
  constexpr int KS = DH / 16, KP = DH / 32, DB = DH / 32;
  constexpr int BLOCK = kTile * DH;            // bytes of codes of K, and of V
  __shared__ float join[kAttendWaves / 2][(DB * NQ * 16 + (SOFTMAX ? 2 * NQ : 0)) * 64];
  const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, g = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  AttendItem it;
  if (!attend8_item<32 * NQ>(p, lane, &it)) return;
  const AttendUser& u = it.u;
  const int head = it.head, first_row = it.first_row, n_rows = it.n_rows, least = it.least, t0 = it.t0, t1 = it.t1;

  int seen[NQ];
  uint4 qf[NQ][KS];
#pragma unroll
  for (int qb = 0; qb < NQ; ++qb) {
    const int r = qb * 32 + l32;
    const bool ok = r < n_rows;
    seen[qb] = ok ? attend_seen(u, first_row + r, p.causal) : 0;
    const uint16_t* qr = p.q + (int64_t)(u.row0 + first_row + (ok ? r : 0)) * p.q_stride + head * DH + g * 8;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) qf[qb][ks] = *reinterpret_cast<const uint4*>(qr + ks * 16);
  }
  f32x16_t oacc[DB][NQ];
  float mref[NQ], lsum[NQ];
#pragma unroll
  for (int qb = 0; qb < NQ; ++qb) {
    mref[qb] = -INFINITY; lsum[qb] = 0.f;
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

  // one tile, half by half; each piece of codes makes room for the wavefront's next tile as soon as it has been converted
  auto tile = [&](auto more_tag, int t) {
    constexpr bool MORE = decltype(more_tag)::value;
    const int tn = t + kAttendWaves;
    float2 sn = sc;
    if constexpr (MORE) sn = load_scales(tn);
    const bool masked = least < (t + 1) * kTile;
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
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
      // element e is key kb*32 + 8*(e/4) + 4*g + e%4 of the tile
      if (masked) {
        uint32_t any = 0;
#pragma unroll
        for (int qb = 0; qb < NQ; ++qb) {
          const int vis = seen[qb] - t * kTile - kb * 32 - 4 * g;
#pragma unroll
          for (int e = 0; e < 16; ++e) s[qb][e] = 8 * (e >> 2) + (e & 3) < vis ? s[qb][e] : (SOFTMAX ? -INFINITY : 0.f);   // (SiLU(0) = 0)
        }
#pragma unroll
        for (int db = 0; db < DB; ++db) any |= fp8_nans(vr[kb][db].x) | fp8_nans(vr[kb][db].y) | fp8_nans(vr[kb][db].z) | fp8_nans(vr[kb][db].w);
        if (__builtin_amdgcn_ballot_w64(any != 0) != 0) {
          int vis[NQ];
#pragma unroll
          for (int qb = 0; qb < NQ; ++qb) {
            vis[qb] = seen[qb] - t * kTile - 4 * g;
            asm volatile("" : "+v"(vis[qb]));      // (its compares are made here, not kept in registers from the ones above)
          }
#pragma unroll
          for (int db = 0; db < DB; ++db) attend8_nans<NQ>(vr[kb][db], kb, oacc[db], vis);
        }
      }
      uint32_t pk[NQ][8];
      if constexpr (SOFTMAX) {
        // the rows' reference scores follow the largest seen score at a distance of at most kAttendSlack, in which exp2 still fits either type
        constexpr float kAttendSlack = 8.0f;
        float mx[NQ];
        bool need = false;
#pragma unroll
        for (int qb = 0; qb < NQ; ++qb) {
          mx[qb] = -INFINITY;
#pragma unroll
          for (int e = 0; e < 16; ++e) mx[qb] = fmaxf(mx[qb], s[qb][e]);
          mx[qb] *= p.score_mul;
          need |= mx[qb] > mref[qb] + kAttendSlack;
        }
        if (__builtin_amdgcn_ballot_w64(need) != 0) {
#pragma unroll
          for (int qb = 0; qb < NQ; ++qb) {
            const float mn = fmaxf(mref[qb], fmaxf(mx[qb], __shfl_xor(mx[qb], 32, 64)));
            const float c = mn == mref[qb] ? 1.0f : __builtin_amdgcn_exp2f(mref[qb] - mn);     // from -inf: 0
            mref[qb] = mn;
            lsum[qb] *= c;
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
            const float a = __builtin_amdgcn_exp2f(fmaf(s[qb][e], p.score_mul, -m)), b = __builtin_amdgcn_exp2f(fmaf(s[qb][e + 1], p.score_mul, -m));
            pk[qb][e >> 1] = H::pack2(a, b);
            lsum[qb] = H::dot2(pk[qb][e >> 1], H::kOnes, lsum[qb]);       // of the weights that the second product takes
          }
        }
      } else {
#pragma unroll
        for (int qb = 0; qb < NQ; ++qb)
#pragma unroll
          for (int e = 0; e < 16; e += 2) {     // SiLU(s) / ln 2 with t = alpha s log2(e)
            const float ta = s[qb][e] * p.score_mul, tb = s[qb][e + 1] * p.score_mul;
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
  int t = t0 + wave;
  if (t < t1) {
    sc = load_scales(t);
    load_k(t, 0);
    load_v(t, 0);
    load_k(t, 1);
    load_v(t, 1);
    for (; t + kAttendWaves < t1; t += kAttendWaves) tile(std::true_type(), t);
    tile(std::false_type(), t);
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
          x[(DB * NQ * 16 + 2 * qb) * 64 + lane] = mref[qb];
          x[(DB * NQ * 16 + 2 * qb + 1) * 64 + lane] = lsum[qb];
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
          const float m1 = x[(DB * NQ * 16 + 2 * qb) * 64 + lane], M = fmaxf(mref[qb], m1);
          c0 = mref[qb] == M ? 1.0f : __builtin_amdgcn_exp2f(mref[qb] - M);
          c1 = m1 == M ? 1.0f : __builtin_amdgcn_exp2f(m1 - M);
          lsum[qb] = lsum[qb] * c0 + x[(DB * NQ * 16 + 2 * qb + 1) * 64 + lane] * c1;
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
  if (wave == 0) attend8_store<H, DH, NQ, SOFTMAX>(p, it, 0, lane, seen, oacc, mref, lsum);
  if constexpr (USERS <= kFewAttendUsers) {
    if (p.arrived != nullptr && u.parts() > 1) attend8_join_last<H, DH, SOFTMAX>(p, it, wave, lane);
  }
}

// The same as a launch of its own: one wavefront for 256 features of a row, pieces loaded eight at a time.
struct JoinUser {
  int32_t row0, rows, keys, part0, parts;
  int32_t cut0;        // rows of the launch's users before it
};
template <int USERS> struct JoinParams {
  uint16_t* out;
  int64_t out_stride;
  const float *part, *ml;
  int32_t n_users, n_rows, d, n_heads, causal;
  JoinUser users[USERS];
};
template <typename H, int DH, bool SOFTMAX, int USERS>
__global__ __launch_bounds__(256) void attend8_join_kernel(JoinParams<USERS> p) {
  constexpr int GROUPS = 256 / DH;
  const int lane = threadIdx.x & 63, segs_sh = max(__builtin_ctz(p.d) - 8, 0);
  const int unit = __builtin_amdgcn_readfirstlane((int)(blockIdx.x * 4 + (threadIdx.x >> 6)));
  const int row = unit >> segs_sh, f = (unit - (row << segs_sh)) * 256 + lane * 4;
  if (row >= p.n_rows) return;
  const JoinUser u = user_of(p.users, p.n_users, row, lane, [](const JoinUser& x) { return x.cut0; });
  const int r = row - u.cut0, seen = p.causal ? max(u.keys - u.rows + 1 + r, 0) : u.keys;
  const bool mine = f < p.d;           // (d = 128: half of the lanes)
  const int head = (mine ? f : 0) / DH;
  const float* x = p.part + ((int64_t)u.part0 + r) * p.d + (mine ? f : 0);
  const int64_t step = (int64_t)u.rows * p.d;      // between a row's pieces
  PieceSum<SOFTMAX> sum[GROUPS];
  for (int k0 = 0; k0 < u.parts; k0 += 8) {
    float4 v[8];
    float2 ml[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const int kk = min(k0 + k, u.parts - 1);
      v[k] = *reinterpret_cast<const float4*>(x + kk * step);
      ml[k] = SOFTMAX ? *reinterpret_cast<const float2*>(p.ml + (((int64_t)u.part0 + (int64_t)kk * u.rows + r) * p.n_heads + head) * 2) : make_float2(0.f, 0.f);
    }
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (k0 + k < u.parts) sum[k % GROUPS].add(v[k], ml[k].x, ml[k].y);
  }
#pragma unroll
  for (int by = 1; by < GROUPS; by *= 2)
#pragma unroll
    for (int i = 0; i < GROUPS; i += 2 * by) sum[i].add(sum[i + by].o, sum[i + by].M, sum[i + by].l);
  if (mine) *reinterpret_cast<uint2*>(p.out + (int64_t)(u.row0 + r) * p.out_stride + f) = sum[0].template out<H>(seen);
}

}  // namespace relaygr
