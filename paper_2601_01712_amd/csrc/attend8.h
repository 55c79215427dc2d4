// Attention of query rows over the 8-bit K/V cache (layout and conversions in kv8.h).  Row i of user u, which sees the first n_i tokens
// of the user's entry:
//     SiLU form     o_i = (1/n_i) sum_{j < n_i} SiLU(alpha <q_i, k_j>) v_j
//     softmax form  o_i = sum_{j < n_i} exp(alpha <q_i, k_j>) v_j / sum_{j < n_i} exp(alpha <q_i, k_j>)
// and o_i = 0 where n_i = 0.  The products are those of the 16-bit kernel (attention.h): S^T = K Q^T, whose accumulator layout is the operand
// layout of the next product, O^T += V^T P^T with P rounded to the storage type (half a step, 2^-8 or 2^-11 of each weight, signs at random); scores,
// weights' sums and outputs are fp32.
#pragma once

#include "kv8.h"

namespace relaygr {

constexpr int kAttendUsers = 64;       // of a launch: they travel in the kernel's arguments
constexpr int kAttendWaves = 4;        // wavefronts of a workgroup
struct AttendUser {
  const char* kv;      // codes of the entry's tile 0, head 0, in the call's layer
  int32_t row0, rows;  // the user's rows in q and out
  int32_t keys;        // tokens that its last row sees (without `causal`: every row)
  int32_t item0;       // items of the launch's users before it, for one head
  int32_t part0;       // first of its rows in the table of partial sums
  int32_t parts, per;  // pieces of its key sequence, key tiles in each
  int32_t pad_;
};
static_assert(sizeof(AttendUser) == 40, "AttendUser layout");
struct AttendParams {
  const uint16_t* q;
  uint16_t* out;
  int64_t q_stride, out_stride;      // elements between rows
  int64_t tile_stride, scales_off;   // bytes: between tiles, from a tile's codes to its layer's scales
  float* part;                       // [partial rows][d] sums of rows that are cut along the keys
  float* ml;                         // softmax form: [partial rows][n_heads][2] reference score (log2 units) and sum of weights
  int32_t n_users, n_items, d, n_heads, causal;
  float score_mul;                   // alpha * log2(e)
  AttendUser users[kAttendUsers];
};
// Tokens that row i of the user sees.
__device__ __forceinline__ int attend_seen(const AttendUser& u, int i, int causal) { return causal ? max(u.keys - u.rows + 1 + i, 0) : u.keys; }

// NaN codes of four, as 0x01 in their bytes.
__device__ __forceinline__ uint32_t fp8_nans(uint32_t codes) { return (((codes & 0x7F7F7F7Fu) + 0x01010101u) >> 7) & 0x01010101u; }

// A tile that not every row sees whole: a weight of zero is no answer to a NaN in V (0 * NaN), which only rows that see its token may get.  Where a
// tile holds any, they leave the tile's V, and what is NaN times what is seen is added twice to the sums, as +inf and as -inf: products
// of powers of two beyond fp32 (in bf16 whatever the storage type; fp16 does not reach that far).
template <int NQ, int DB>
__device__ __forceinline__ void attend8_nans(uint4 (&vr)[DB][2], f32x16_t (&oacc)[DB][NQ], const int (&vis)[NQ]) {
  const uint32_t big = 0x7180;          // 2^100 in bf16
#pragma unroll
  for (int kb = 0; kb < 2; ++kb)
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
      for (int db = 0; db < DB; ++db) {
        uint32_t w0 = m == 0 ? vr[db][kb].x : vr[db][kb].z, w1 = m == 0 ? vr[db][kb].y : vr[db][kb].w;
        const uint32_t n0 = fp8_nans(w0), n1 = fp8_nans(w1);
        w0 &= ~(n0 * 0xFFu); w1 &= ~(n1 * 0xFFu);
        if (m == 0) { vr[db][kb].x = w0; vr[db][kb].y = w1; } else { vr[db][kb].z = w0; vr[db][kb].w = w1; }
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
          oacc[db][qb] = Bf16::mfma(neg, sees, Bf16::mfma(pos, sees, oacc[db][qb]));
        }
        __builtin_amdgcn_sched_barrier(0);
      }
}

// One item: up to 32*NQ rows of one user, one head, one piece of the key sequence.  The workgroup's wavefronts take the piece's key tiles in turn, all
// for the same rows, each straight from memory to its registers (the codes are in operand order) with the next tile on its way while it
// works on one; their sums meet in LDS at the end.
template <typename H, int DH, int NQ, bool SOFTMAX>
__global__ __launch_bounds__(kAttendWaves * 64, 2) void attend8_kernel(AttendParams p) {
  constexpr int KS = DH / 16, KP = DH / 32, DB = DH / 32;
  constexpr int BLOCK = kTile * DH;            // bytes of codes of K, and of V
  __shared__ float join[kAttendWaves / 2][(DB * NQ * 16 + (SOFTMAX ? 2 * NQ : 0)) * 64];
  const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, g = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  // (heads dealt to the XCDs as in attention.h, so that the row tiles of one user and head share an L2)
  const int xcd = blockIdx.x & 7, turn = blockIdx.x >> 3, heads_sh = __builtin_ctz(p.n_heads);
  int head, item;
  if (p.n_heads >= 8) {
    const int sh = heads_sh - 3;
    head = (xcd << sh) + (turn & ((1 << sh) - 1));
    item = turn >> sh;
  } else {
    head = xcd & (p.n_heads - 1);
    item = (turn << (3 - heads_sh)) + (xcd >> heads_sh);
  }
  if (item >= p.n_items) return;
  const int at = __builtin_popcountll(__builtin_amdgcn_ballot_w64(lane < p.n_users && p.users[lane < p.n_users ? lane : 0].item0 <= item)) - 1;
  const AttendUser u = p.users[__builtin_amdgcn_readfirstlane(at)];
  const int row_tiles = (u.rows + 32 * NQ - 1) / (32 * NQ);
  const int piece = (item - u.item0) / row_tiles, first_row = (item - u.item0 - piece * row_tiles) * 32 * NQ;
  const int n_rows = min(32 * NQ, u.rows - first_row);

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
  const int most = attend_seen(u, first_row + n_rows - 1, p.causal), least = attend_seen(u, first_row, p.causal);   // of the item's rows
  const int t0 = piece * u.per, t1 = min(t0 + u.per, (most + kTile - 1) / kTile);

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

  const char* base = u.kv + (int64_t)head * (2 * BLOCK);
  const char* scales = u.kv + p.scales_off + head * 8;
  uint4 kr[2][KP], vr[DB][2];
  float2 sc;
  auto load = [&](int t, uint4 (&kx)[2][KP], uint4 (&vx)[DB][2], float2& s) {
    const char* tile = base + (int64_t)t * p.tile_stride;
    s = *reinterpret_cast<const float2*>(scales + (int64_t)t * p.tile_stride);
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int kp = 0; kp < KP; ++kp) kx[kb][kp] = *reinterpret_cast<const uint4*>(tile + (kb * KP + kp) * 1024 + lane * 16);
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) vx[db][kb] = *reinterpret_cast<const uint4*>(tile + BLOCK + (db * 2 + kb) * 1024 + lane * 16);
  };
  int t = t0 + wave;
  if (t < t1) load(t, kr, vr, sc);
  for (; t < t1; t += kAttendWaves) {
    uint4 kn[2][KP], vn[DB][2];
    float2 sn = sc;
    const int tn = t + kAttendWaves;
    load(tn < t1 ? tn : t, kn, vn, sn);
    // first product: the tile's 64 keys
    f32x16_t s[2][NQ];
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
#pragma unroll
      for (int qb = 0; qb < NQ; ++qb)
#pragma unroll
        for (int e = 0; e < 16; ++e) s[kb][qb][e] = 0.f;
#pragma unroll
      for (int kp = 0; kp < KP; ++kp) {
        const u32x4_t lo = fp8_frag<H>(kr[kb][kp].x, kr[kb][kp].y, sc.x), hi = fp8_frag<H>(kr[kb][kp].z, kr[kb][kp].w, sc.x);
#pragma unroll
        for (int qb = 0; qb < NQ; ++qb) s[kb][qb] = H::mfma(lo, qf[qb][2 * kp], s[kb][qb]);
#pragma unroll
        for (int qb = 0; qb < NQ; ++qb) s[kb][qb] = H::mfma(hi, qf[qb][2 * kp + 1], s[kb][qb]);
      }
    }
    // weights.  Element e of half kb is key kb*32 + 8*(e/4) + 4*g + e%4 of the tile
    const bool masked = least < (t + 1) * kTile;
    if (masked) {
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int qb = 0; qb < NQ; ++qb) {
          const int vis = seen[qb] - t * kTile - kb * 32 - 4 * g;
#pragma unroll
          for (int e = 0; e < 16; ++e) s[kb][qb][e] = 8 * (e >> 2) + (e & 3) < vis ? s[kb][qb][e] : (SOFTMAX ? -INFINITY : 0.f);   // (SiLU(0) = 0)
        }
    }
    uint32_t pk[2][NQ][8];
    if constexpr (SOFTMAX) {
      // the rows' reference scores follow the largest seen score at a distance of at most kAttendSlack, in which exp2 still fits either type
      constexpr float kAttendSlack = 8.0f;
      float mx[NQ];
      bool need = false;
#pragma unroll
      for (int qb = 0; qb < NQ; ++qb) {
        mx[qb] = -INFINITY;
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
          for (int e = 0; e < 16; ++e) mx[qb] = fmaxf(mx[qb], s[kb][qb][e]);
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
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
          for (int e = 0; e < 16; e += 2) {
            const float a = __builtin_amdgcn_exp2f(fmaf(s[kb][qb][e], p.score_mul, -m)), b = __builtin_amdgcn_exp2f(fmaf(s[kb][qb][e + 1], p.score_mul, -m));
            lsum[qb] += a + b;
            pk[kb][qb][e >> 1] = H::pack2(a, b);
          }
      }
    } else {
#pragma unroll
      for (int qb = 0; qb < NQ; ++qb)
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
          for (int e = 0; e < 16; e += 2) {     // SiLU(s) / ln 2 with t = alpha s log2(e)
            const float ta = s[kb][qb][e] * p.score_mul, tb = s[kb][qb][e + 1] * p.score_mul;
            pk[kb][qb][e >> 1] = H::pack2(ta * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-ta)), tb * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-tb)));
          }
    }
    if (masked) {
      uint32_t any = 0;
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) any |= fp8_nans(vr[db][kb].x) | fp8_nans(vr[db][kb].y) | fp8_nans(vr[db][kb].z) | fp8_nans(vr[db][kb].w);
      if (__builtin_amdgcn_ballot_w64(any != 0) != 0) {
        int vis[NQ];
#pragma unroll
        for (int qb = 0; qb < NQ; ++qb) {
          vis[qb] = seen[qb] - t * kTile - 4 * g;
          asm volatile("" : "+v"(vis[qb]));      // (its compares are made here, not kept in registers from the ones above)
        }
        attend8_nans<NQ, DB>(vr, oacc, vis);
      }
    }
    // second product
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int db = 0; db < DB; ++db) {
          const u32x4_t vf = m == 0 ? fp8_frag<H>(vr[db][kb].x, vr[db][kb].y, sc.y) : fp8_frag<H>(vr[db][kb].z, vr[db][kb].w, sc.y);
#pragma unroll
          for (int qb = 0; qb < NQ; ++qb)
            oacc[db][qb] = H::mfma(vf, make_uint4(pk[kb][qb][4 * m], pk[kb][qb][4 * m + 1], pk[kb][qb][4 * m + 2], pk[kb][qb][4 * m + 3]), oacc[db][qb]);
        }
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int kp = 0; kp < KP; ++kp) kr[kb][kp] = kn[kb][kp];
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) vr[db][kb] = vn[db][kb];
    sc = sn;
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
  if (wave != 0) return;

  // element e of oacc[db][qb]: feature db*32 + 8*(e/4) + 4*g + e%4, row l32 of block qb
#pragma unroll
  for (int qb = 0; qb < NQ; ++qb) {
    const int r = qb * 32 + l32;
    if constexpr (SOFTMAX) lsum[qb] += __shfl_xor(lsum[qb], 32, 64);
    if (r >= n_rows) continue;
    if (u.parts == 1) {
      const float mul = seen[qb] == 0 ? 0.f : SOFTMAX ? 1.0f / lsum[qb] : 0.69314718055994531f / (float)seen[qb];
      uint16_t* dst = p.out + (int64_t)(u.row0 + first_row + r) * p.out_stride + head * DH + 4 * g;
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int e4 = 0; e4 < 4; ++e4) {
          uint2 w = make_uint2(H::pack2(oacc[db][qb][4 * e4] * mul, oacc[db][qb][4 * e4 + 1] * mul), H::pack2(oacc[db][qb][4 * e4 + 2] * mul, oacc[db][qb][4 * e4 + 3] * mul));
          if (seen[qb] == 0) w = make_uint2(0, 0);
          *reinterpret_cast<uint2*>(dst + db * 32 + 8 * e4) = w;
        }
    } else {
      const int64_t pr = (int64_t)u.part0 + (int64_t)piece * u.rows + first_row + r;
      float* dst = p.part + pr * p.d + head * DH + 4 * g;
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int e4 = 0; e4 < 4; ++e4)
          *reinterpret_cast<float4*>(dst + db * 32 + 8 * e4) =
              make_float4(oacc[db][qb][4 * e4], oacc[db][qb][4 * e4 + 1], oacc[db][qb][4 * e4 + 2], oacc[db][qb][4 * e4 + 3]);
      if constexpr (SOFTMAX) {
        if (g == 0) *reinterpret_cast<float2*>(p.ml + (pr * p.n_heads + head) * 2) = make_float2(mref[qb], lsum[qb]);
      }
    }
  }
}

// Adds the pieces of rows that were cut along the keys, in their order, and writes the rows.  One thread for four features of a row.
template <typename H, bool SOFTMAX>
__global__ __launch_bounds__(256) void attend8_join_kernel(AttendParams p, int n_rows, int row_base) {
  const int lane = threadIdx.x & 63, per_row = p.d / 4;
  const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int row = row_base + (int)(id / per_row), f = (int)(id % per_row) * 4, head = f / (p.d / p.n_heads);
  if (row >= row_base + n_rows) return;
  int at = 0;
  for (int i = 1; i < p.n_users; ++i) at += p.users[i].row0 <= row ? 1 : 0;      // (users in the order of their rows)
  (void)lane;
  const AttendUser& u = p.users[at];
  if (u.parts <= 1 || row - u.row0 >= u.rows) return;
  const int seen = attend_seen(u, row - u.row0, p.causal);
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
  float M = -INFINITY, l = 0.f;
  for (int k = 0; k < u.parts; ++k) {
    const int64_t pr = (int64_t)u.part0 + (int64_t)k * u.rows + (row - u.row0);
    const float4 x = *reinterpret_cast<const float4*>(p.part + pr * p.d + f);
    if constexpr (SOFTMAX) {
      const float2 ml = *reinterpret_cast<const float2*>(p.ml + (pr * p.n_heads + head) * 2);
      const float mn = fmaxf(M, ml.x), c0 = M == mn ? 1.0f : __builtin_amdgcn_exp2f(M - mn), c1 = ml.x == mn ? 1.0f : __builtin_amdgcn_exp2f(ml.x - mn);
      o = make_float4(o.x * c0 + x.x * c1, o.y * c0 + x.y * c1, o.z * c0 + x.z * c1, o.w * c0 + x.w * c1);
      l = l * c0 + ml.y * c1;
      M = mn;
    } else {
      o = make_float4(o.x + x.x, o.y + x.y, o.z + x.z, o.w + x.w);
    }
  }
  const float mul = SOFTMAX ? 1.0f / l : 0.69314718055994531f / (float)seen;
  uint2 w = make_uint2(H::pack2(o.x * mul, o.y * mul), H::pack2(o.z * mul, o.w * mul));
  if (seen == 0) w = make_uint2(0, 0);
  *reinterpret_cast<uint2*>(p.out + (int64_t)row * p.out_stride + f) = w;
}

}  // namespace relaygr
