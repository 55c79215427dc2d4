// The 8-bit K/V cache: layout and conversions, and the kernels that write rows into it and read them back.
//
// A pool made for 8 bits stores K and V as e4m3 codes with one power-of-two scale for each block: the 64 tokens of a tile, of one
// head of K or of V, in one layer.  With a the largest finite magnitude of a block's values x,
//     e = max(floor(log2 a) - 8 + (a / 2^floor(log2 a) > 1.75 ? 1 : 0), -100)      the least e with a / 2^e <= 448, e4m3's largest
//     code = e4m3(x / 2^e), to nearest, ties to even                                a code stands for code * 2^e
// A value below 2^(e-6), 2^-14.8 of the block's largest or less, loses significant bits (e4m3's subnormals); every other is off by at most
// 2^-4 of itself, whatever the scale's mantissa would be: a float format gains nothing from scales between powers of two, and with these
//   - a code times its scale is exact in bf16 (and in fp16 for what came from fp16), so that attention works on exactly what a read returns;
//   - the conversion instruction applies the scale, and attention has no scale to multiply by;
//   - values that a block keeps while others join it are rounded again only where the larger scale makes them subnormal.
// Infinities and NaN are NaN codes (e4m3 has no infinity), and where 256 * 2^e is beyond the storage type (e = 8 in fp16, 120 in bf16:
// blocks within 1/8 of the type's largest value) codes stop at +-240, still within 2^-4.
//
// A tile block of the pool, in bytes: for every layer and head 64 * dh codes of K, then 64 * dh of V, at layer * 128 * d + head * 128 * dh; behind
// those of all layers the scales as fp32, [layer][head][K, V], padded to 128 bytes.  Codes are in the order in which the 32x32x16 MFMA takes
// its operands, two fragments to a lane's 16 bytes:
//     K chunk (kb, kp): lane (g, l32) holds token kb*32+l32, features (2kp+h)*16 + 8g + {0..7}, h = 0, 1
//     V chunk (db, kb): lane (g, l32) holds feature db*32+l32, tokens kb*32+16m+4g+{0..3}, kb*32+16m+8+4g+{0..3}, m = 0, 1
// (the halves are the 16-bit layout's fragments (kb, ks = 2kp+h) and (db, kb, m)).
#pragma once

#include "common.h"
#include "gemm.h"

namespace relaygr {

struct KvLayout8 {
  static __host__ __device__ __forceinline__ int k_off(int r, int f, int dh) {
    const int kb = r >> 5, l32 = r & 31, ks = f >> 4, g = (f >> 3) & 1, j = f & 7;
    return ((kb * (dh >> 5) + (ks >> 1)) * 64 + g * 32 + l32) * 16 + (ks & 1) * 8 + j;
  }
  static __host__ __device__ __forceinline__ int v_off(int r, int f, int dh) {
    const int db = f >> 5, l32 = f & 31, kb = r >> 5, m = (r >> 4) & 1, w = r & 15;
    const int g = (w >> 2) & 1, j = ((w >> 3) << 2) | (w & 3);
    return kTile * dh + ((db * 2 + kb) * 64 + g * 32 + l32) * 16 + m * 8 + j;
  }
};

// ---- conversions (each one instruction for two values; `scale` a power of two) -------------------------------------------------------
typedef short i16x2_t __attribute__((ext_vector_type(2)));

template <typename H> struct Fp8;
template <> struct Fp8<Bf16> {
  static constexpr uint32_t kInf = 0x7F80;        // the type's infinity, as bits
  static constexpr int kTopExp = 120;
  static __device__ __forceinline__ float bits_to_f32(uint32_t b) { return __uint_as_float(b << 16); }
  template <bool HI> static __device__ __forceinline__ uint32_t up(uint32_t codes, float scale) {    // codes 2*HI, 2*HI+1 of the word
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, HI));
  }
  static __device__ __forceinline__ uint32_t down4(uint32_t a, uint32_t b, float scale) {            // two packed pairs to four codes
    i16x2_t r = {0, 0};
    r = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(r, __builtin_bit_cast(bf16x2_t, a), scale, false);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(r, __builtin_bit_cast(bf16x2_t, b), scale, true);
    return __builtin_bit_cast(uint32_t, r);
  }
};
template <> struct Fp8<F16> {
  static constexpr uint32_t kInf = 0x7C00;
  static constexpr int kTopExp = 8;
  static __device__ __forceinline__ float bits_to_f32(uint32_t b) { return F16::to_f32((uint16_t)b); }
  template <bool HI> static __device__ __forceinline__ uint32_t up(uint32_t codes, float scale) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(codes, scale, HI));
  }
  static __device__ __forceinline__ uint32_t down4(uint32_t a, uint32_t b, float scale) {
    i16x2_t r = {0, 0};
    r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f16(r, __builtin_bit_cast(f16x2_t, a), scale, false);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f16(r, __builtin_bit_cast(f16x2_t, b), scale, true);
    return __builtin_bit_cast(uint32_t, r);
  }
};
// Eight codes of a fragment (two words) to the eight 16-bit values an MFMA operand holds.
template <typename H>
__device__ __forceinline__ u32x4_t fp8_frag(uint32_t w0, uint32_t w1, float scale) {
  return u32x4_t{Fp8<H>::template up<false>(w0, scale), Fp8<H>::template up<true>(w0, scale), Fp8<H>::template up<false>(w1, scale), Fp8<H>::template up<true>(w1, scale)};
}
__device__ __forceinline__ uint32_t fp8_down4_f32(float a, float b, float c, float d, float scale) {
  i16x2_t r = {0, 0};
  r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(r, a, b, scale, false);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(r, c, d, scale, true);
  return __builtin_bit_cast(uint32_t, r);
}
// Four codes under another scale.
__device__ __forceinline__ uint32_t fp8_rescale4(uint32_t codes, float from, float to) {
  const f32x2_t a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(codes, from, false), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(codes, from, true);
  return fp8_down4_f32(a[0], a[1], b[0], b[1], to);
}
// Exponent of a block's scale from its largest finite magnitude.
__device__ __forceinline__ int fp8_exponent(float amax) {
  const uint32_t b = __float_as_uint(amax) & 0x7FFFFFFFu;
  const int e = (int)(b >> 23) - 127 - 8 + ((b & 0x7FFFFFu) > 0x600000u ? 1 : 0);
  return min(max(e, -100), 120);
}
__device__ __forceinline__ float pow2f(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }

// Largest magnitude of packed 16-bit pairs, as bits (pairs of unsigned maxima).
__device__ __forceinline__ uint32_t max_u16x2(uint32_t a, uint32_t b) {
  typedef unsigned short u16x2_t __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2_t, a), __builtin_bit_cast(u16x2_t, b)));
}
// Largest of an unsigned value over the wavefront, in a scalar.
__device__ __forceinline__ uint32_t wave_max_u32(uint32_t v) {
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xB1, 0xF, 0xF, true));
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x4E, 0xF, 0xF, true));
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x141, 0xF, 0xF, true));
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x140, 0xF, 0xF, true));
  return max(max((uint32_t)__builtin_amdgcn_readlane((int)v, 0), (uint32_t)__builtin_amdgcn_readlane((int)v, 16)),
             max((uint32_t)__builtin_amdgcn_readlane((int)v, 32), (uint32_t)__builtin_amdgcn_readlane((int)v, 48)));
}

// Largest finite magnitude of a wavefront's 16-byte pieces of a block.
template <typename H, int N>
__device__ __forceinline__ float kv8_top(const uint4 (&x)[N]) {
  uint32_t top2 = 0;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    top2 = max_u16x2(top2, x[i].x & 0x7FFF7FFFu); top2 = max_u16x2(top2, x[i].y & 0x7FFF7FFFu);
    top2 = max_u16x2(top2, x[i].z & 0x7FFF7FFFu); top2 = max_u16x2(top2, x[i].w & 0x7FFF7FFFu);
  }
  uint32_t top = wave_max_u32(max(top2 & 0xFFFFu, top2 >> 16));
  if (top >= Fp8<H>::kInf) {     // infinities or NaN among them: leave those out
    uint32_t t = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const uint32_t w[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint32_t lo = w[j] & 0x7FFFu, hi = (w[j] >> 16) & 0x7FFFu;
        t = max(t, max(lo >= Fp8<H>::kInf ? 0u : lo, hi >= Fp8<H>::kInf ? 0u : hi));
      }
    }
    top = wave_max_u32(t);
  }
  return Fp8<H>::bits_to_f32(top);
}
// Eight values to eight codes.
template <typename H>
__device__ __forceinline__ uint2 kv8_quantise(const uint4& a, float scale) {
  if (scale != pow2f(Fp8<H>::kTopExp)) return make_uint2(Fp8<H>::down4(a.x, a.y, scale), Fp8<H>::down4(a.z, a.w, scale));
  constexpr float inv = Fp8<H>::kTopExp == 8 ? 0x1p-8f : 0x1p-120f;       // 256 * scale would be beyond the type: clamped in fp32
  float y[8];
  const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float v = H::of_word(w[i >> 1], i) * inv;
    y[i] = fabsf(v) > 240.0f && fabsf(v) < 256.0f ? copysignf(240.0f, v) : v;      // (infinities and NaN stay)
  }
  return make_uint2(fp8_down4_f32(y[0], y[1], y[2], y[3], 1.0f), fp8_down4_f32(y[4], y[5], y[6], y[7], 1.0f));
}

// ---- rows into the cache, and back ------------------------------------------------------------------------------------------------
// The users of a launch travel in the kernel's arguments: no staging, no scratch, nothing for two calls to share.  A launch with 2.6 KB of
// arguments takes 4.3 us of the host, one with 650 bytes 3.2, so that launches of few users take kernels with room for few.
constexpr int kRowUsers = 64, kFewRowUsers = 14;
struct RowsUser {
  char* tile0;       // the user's tile 0 (all layers)
  int32_t first;     // token that the user's first row is
  int32_t rows;
  int64_t row0;      // its first row in k and v
  int32_t unit0;     // touched tiles of the launch's users before it
  int32_t pad_;
};
template <int USERS> struct RowsParams {
  void* k;           // [rows][stride] in the storage type: sources of a write, targets of a read
  void* v;
  int64_t k_stride, v_stride;   // elements between rows
  int64_t tile_stride;          // bytes between the tiles of an entry
  int64_t codes_off, scales_off;   // of the layer in a tile
  int32_t n_users, n_tiles, n_heads, pad_;
  RowsUser users[USERS];
};

// A wavefront's unit of a launch: the K or the V block of one head in one touched tile.
struct RowsUnit {
  bool is_v;
  int head, r0, r1;   // the tile's tokens [r0, r1) are rows of the call
  int64_t row;        // row that token r0 is
  char* tile;
};
template <int USERS>
__device__ __forceinline__ bool rows_unit(const RowsParams<USERS>& p, int lane, RowsUnit* u) {
  const int unit = __builtin_amdgcn_readfirstlane((int)(blockIdx.x * 4 + (threadIdx.x >> 6)));
  u->is_v = unit & 1;
  const int t = (unit >> 1) / p.n_heads;
  u->head = (unit >> 1) - t * p.n_heads;
  if (t >= p.n_tiles) return false;
  const int at = __builtin_popcountll(__builtin_amdgcn_ballot_w64(lane < p.n_users && p.users[lane < p.n_users ? lane : 0].unit0 <= t)) - 1;
  const RowsUser& us = p.users[at];
  const int tile = us.first / kTile + (t - us.unit0);
  u->r0 = max(us.first - tile * kTile, 0);
  u->r1 = min(us.first + us.rows - tile * kTile, kTile);
  u->row = us.row0 + (tile * kTile + u->r0 - us.first);
  u->tile = us.tile0 + (int64_t)tile * p.tile_stride;
  return true;
}

// Writes: quantises the block anew from the tokens before r0 that it keeps and the rows of the call; tokens from r1 on become zero.
// One wavefront a block.  What bounds it is HBM: 2 bytes in and 1 out per value.  K rows are loaded in the order of the codes (a lane's
// 16 codes are two 16-byte runs of one token); V codes have their lanes along the features and 16 tokens to a lane, so that V goes through LDS
// as bytes, [token][feature].
template <typename H, int DH, int USERS>
__global__ __launch_bounds__(256) void kv8_write_kernel(RowsParams<USERS> p) {
  constexpr int NL = DH / 8;                 // 16-byte loads of a lane: a block is 64 * DH values
  constexpr int LROW = DH + 8;               // bytes between tokens in LDS
  __shared__ __attribute__((aligned(16))) uint8_t turn[2][kTile * LROW];
  const int lane = threadIdx.x & 63, l32 = lane & 31, g = lane >> 5;
  RowsUnit u;
  if (!rows_unit(p, lane, &u)) return;       // (no barrier below: a wavefront's LDS is its own)
  uint8_t* lds = turn[(threadIdx.x >> 7)];   // wavefronts come in pairs of K and V
  const uint16_t* src = reinterpret_cast<const uint16_t*>(u.is_v ? p.v : p.k) + (u.is_v ? p.v_stride : p.k_stride) * u.row + u.head * DH;
  const int64_t stride = u.is_v ? p.v_stride : p.k_stride;
  char* codes = u.tile + p.codes_off + (int64_t)u.head * (2 * kTile * DH) + (u.is_v ? kTile * DH : 0);
  float* scale_at = reinterpret_cast<float*>(u.tile + p.scales_off) + 2 * u.head + (u.is_v ? 1 : 0);

  // the rows: load i of a lane is token tok(i), features feat(i) .. +7
  auto tok = [&](int i) { return u.is_v ? (i * 64 + lane) / (DH / 8) : (i / (DH / 16)) * 32 + l32; };
  auto feat = [&](int i) { return u.is_v ? (i * 64 + lane) % (DH / 8) * 8 : (i % (DH / 16)) * 16 + g * 8; };
  uint4 x[NL];
#pragma unroll
  for (int i = 0; i < NL; ++i) {
    const int r = tok(i);
    x[i] = make_uint4(0, 0, 0, 0);
    if (r >= u.r0 && r < u.r1) x[i] = *reinterpret_cast<const uint4*>(src + (int64_t)(r - u.r0) * stride + feat(i));
  }
  // codes that stay: tokens before r0 (their chunks are in the order of the output)
  uint4 old[NL / 2];
  float old_scale = 1.0f;
  if (u.r0 > 0) {
    old_scale = *scale_at;
#pragma unroll
    for (int c = 0; c < NL / 2; ++c) old[c] = *reinterpret_cast<const uint4*>(codes + (c * 64 + lane) * 16);
  }
  // which bytes of word w of output chunk c stay
  auto kept = [&](int c, int w) -> uint32_t {
    if (!u.is_v) return (c / (DH / 32)) * 32 + l32 < u.r0 ? 0xFFFFFFFFu : 0u;
    const int t0 = (c & 1) * 32 + (w >> 1) * 16 + (w & 1) * 8 + 4 * g;      // chunk (db, kb): kb = c & 1; word w: m = w / 2
    const int n = min(max(u.r0 - t0, 0), 4);
    return n == 4 ? 0xFFFFFFFFu : (1u << (8 * n)) - 1u;
  };

  float amax = kv8_top<H, NL>(x);
  if (u.r0 > 0) {
    uint32_t t = 0;
#pragma unroll
    for (int c = 0; c < NL / 2; ++c) {
      const uint32_t w[4] = {old[c].x, old[c].y, old[c].z, old[c].w};
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint32_t m = w[j] & kept(c, j) & 0x7F7F7F7Fu;
#pragma unroll
        for (int b = 0; b < 4; ++b) { const uint32_t code = (m >> (8 * b)) & 0x7Fu; t = max(t, code == 0x7Fu ? 0u : code); }
      }
    }
    t = wave_max_u32(t);
    const f32x2_t kept_top = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(t, old_scale, false);
    amax = fmaxf(amax, kept_top[0]);
  }
  const float scale = pow2f(fp8_exponent(amax));
  uint4 out[NL / 2];
  if (!u.is_v) {
#pragma unroll
    for (int c = 0; c < NL / 2; ++c) {
      const uint2 lo = kv8_quantise<H>(x[2 * c], scale), hi = kv8_quantise<H>(x[2 * c + 1], scale);
      out[c] = make_uint4(lo.x, lo.y, hi.x, hi.y);
    }
  } else {
#pragma unroll
    for (int i = 0; i < NL; ++i) *reinterpret_cast<uint2*>(lds + tok(i) * LROW + feat(i)) = kv8_quantise<H>(x[i], scale);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int c = 0; c < NL / 2; ++c) {
      uint32_t w[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint8_t* at = lds + ((c & 1) * 32 + (j >> 1) * 16 + (j & 1) * 8 + 4 * g) * LROW + (c >> 1) * 32 + l32;
        w[j] = (uint32_t)at[0] | (uint32_t)at[LROW] << 8 | (uint32_t)at[2 * LROW] << 16 | (uint32_t)at[3 * LROW] << 24;
      }
      out[c] = make_uint4(w[0], w[1], w[2], w[3]);
    }
  }
  if (u.r0 > 0) {
    const bool same = scale == old_scale;
#pragma unroll
    for (int c = 0; c < NL / 2; ++c) {
      uint32_t o[4] = {out[c].x, out[c].y, out[c].z, out[c].w};
      const uint32_t w[4] = {old[c].x, old[c].y, old[c].z, old[c].w};
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint32_t stay = kept(c, j);
        o[j] |= (same ? w[j] : fp8_rescale4(w[j], old_scale, scale)) & stay;    // (the call's rows left zero there)
      }
      out[c] = make_uint4(o[0], o[1], o[2], o[3]);
    }
  }
#pragma unroll
  for (int c = 0; c < NL / 2; ++c) *reinterpret_cast<uint4*>(codes + (c * 64 + lane) * 16) = out[c];
  if (lane == 0) *scale_at = scale;
}

// Quantises whole tiles that are already in the order of the 16-bit layout: a pre-inference's K and V of one layer, from its scratch tiles into the
// pool.  One wavefront a block; a lane's output chunk is its pieces of two consecutive fragments, so that nothing changes lanes.
struct TilesUser {
  char* tile0;             // of the pool entry
  const uint16_t* src;     // the user's tile 0 in scratch, head 0
  int32_t unit0, pad_;     // tiles of the launch's users before it
};
struct TilesParams {
  int64_t tile_stride, src_stride;   // bytes between the entry's tiles; elements between scratch tiles
  int64_t codes_off, scales_off;
  int32_t n_users, n_tiles, n_heads, pad_;
  TilesUser users[kRowUsers];
};
template <typename H, int DH>
__global__ __launch_bounds__(256) void kv8_tiles_kernel(TilesParams p) {
  constexpr int NL = DH / 8;
  const int lane = threadIdx.x & 63;
  const int unit = __builtin_amdgcn_readfirstlane((int)(blockIdx.x * 4 + (threadIdx.x >> 6)));
  const int is_v = unit & 1, t = (unit >> 1) / p.n_heads, head = (unit >> 1) - t * p.n_heads;
  if (t >= p.n_tiles) return;
  const int at = __builtin_popcountll(__builtin_amdgcn_ballot_w64(lane < p.n_users && p.users[lane < p.n_users ? lane : 0].unit0 <= t)) - 1;
  const TilesUser& us = p.users[__builtin_amdgcn_readfirstlane(at)];
  const uint4* src = reinterpret_cast<const uint4*>(us.src + (int64_t)(t - us.unit0) * p.src_stride + (2 * head + is_v) * (kTile * DH));
  char* tile = us.tile0 + (int64_t)(t - us.unit0) * p.tile_stride;
  uint4 x[NL];
#pragma unroll
  for (int i = 0; i < NL; ++i) x[i] = src[i * 64 + lane];
  const float scale = pow2f(fp8_exponent(kv8_top<H, NL>(x)));
#pragma unroll
  for (int c = 0; c < NL / 2; ++c) {
    const uint2 lo = kv8_quantise<H>(x[2 * c], scale), hi = kv8_quantise<H>(x[2 * c + 1], scale);
    *reinterpret_cast<uint4*>(tile + p.codes_off + (2 * head + is_v) * (kTile * DH) + (c * 64 + lane) * 16) = make_uint4(lo.x, lo.y, hi.x, hi.y);
  }
  if (lane == 0) reinterpret_cast<float*>(tile + p.scales_off)[2 * head + is_v] = scale;
}

// Reads: the values that tokens [r0, r1) of the block stand for, into their rows.  One wavefront a block, 1 byte in and 2 out per value.
template <typename H, int DH, int USERS>
__global__ __launch_bounds__(256) void kv8_read_kernel(RowsParams<USERS> p) {
  constexpr int NL = DH / 8, LROW = DH + 8;
  __shared__ __attribute__((aligned(16))) uint8_t turn[2][kTile * LROW];
  const int lane = threadIdx.x & 63, l32 = lane & 31, g = lane >> 5;
  RowsUnit u;
  if (!rows_unit(p, lane, &u)) return;
  uint8_t* lds = turn[(threadIdx.x >> 7)];
  uint16_t* dst = reinterpret_cast<uint16_t*>(u.is_v ? p.v : p.k) + (u.is_v ? p.v_stride : p.k_stride) * u.row + u.head * DH;
  const int64_t stride = u.is_v ? p.v_stride : p.k_stride;
  const char* codes = u.tile + p.codes_off + (int64_t)u.head * (2 * kTile * DH) + (u.is_v ? kTile * DH : 0);
  const float scale = reinterpret_cast<const float*>(u.tile + p.scales_off)[2 * u.head + (u.is_v ? 1 : 0)];
  uint4 x[NL / 2];
#pragma unroll
  for (int c = 0; c < NL / 2; ++c) x[c] = *reinterpret_cast<const uint4*>(codes + (c * 64 + lane) * 16);
  auto store = [&](int r, int f, uint32_t w0, uint32_t w1) {
    if (r >= u.r0 && r < u.r1) *reinterpret_cast<u32x4_t*>(dst + (int64_t)(r - u.r0) * stride + f) = fp8_frag<H>(w0, w1, scale);
  };
  if (!u.is_v) {
#pragma unroll
    for (int c = 0; c < NL / 2; ++c) {
      const int r = (c / (DH / 32)) * 32 + l32, f = (c % (DH / 32)) * 32 + g * 8;
      store(r, f, x[c].x, x[c].y);
      store(r, f + 16, x[c].z, x[c].w);
    }
  } else {
#pragma unroll
    for (int c = 0; c < NL / 2; ++c) {
      const uint32_t w[4] = {x[c].x, x[c].y, x[c].z, x[c].w};
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        uint8_t* at = lds + ((c & 1) * 32 + (j >> 1) * 16 + (j & 1) * 8 + 4 * g) * LROW + (c >> 1) * 32 + l32;
#pragma unroll
        for (int b = 0; b < 4; ++b) at[b * LROW] = (uint8_t)(w[j] >> (8 * b));
      }
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      const int r = (i * 64 + lane) / (DH / 8), f = (i * 64 + lane) % (DH / 8) * 8;
      const uint2 w = *reinterpret_cast<const uint2*>(lds + r * LROW + f);
      store(r, f, w.x, w.y);
    }
  }
}

}  // namespace relaygr
