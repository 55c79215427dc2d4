// The 8-bit K/V cache: layout and conversions, and the kernels that write rows into it and read them back.
//
// A pool made for 8 bits stores K and V as e4m3 codes with one power-of-two scale for each block: the 64 tokens of a tile, of one
// head of K or of V, in one layer.  With a the largest finite magnitude of a block's values x,
//     e = max(floor(log2 a) - 8 + (a / 2^floor(log2 a) > 1.75 ? 1 : 0), -100)      the least e with a / 2^e <= 448, e4m3's largest
//     code = e4m3(x / 2^e), to nearest, ties to even                                a code stands for code * 2^e
// A value below 2^(e-6), which is 2^-14.8 to 2^-13.8 of the block's largest by where that stands in (224 * 2^e, 448 * 2^e], loses significant bits (e4m3's
// subnormals); every other is off by at most 2^-4 of itself, whatever the scale's mantissa would be: a float format gains nothing from scales between powers of two, and with these
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

#include <type_traits>

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

// Largest of an unsigned value over the lanes that share a head, where lanes have eight features each: groups of GROUP adjacent lanes in each run of RUN.
template <int GROUP, int RUN>
__device__ __forceinline__ uint32_t head_max_u32(uint32_t v) {
  if constexpr (GROUP == 64) return wave_max_u32(v);
  auto dpp = [&](auto ctrl) { v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, decltype(ctrl)::value, 0xF, 0xF, true)); };
  dpp(std::integral_constant<int, 0xB1>());
  dpp(std::integral_constant<int, 0x4E>());
  if constexpr (GROUP >= 8) dpp(std::integral_constant<int, 0x141>());
  if constexpr (GROUP >= 16) dpp(std::integral_constant<int, 0x140>());
  if constexpr (RUN <= 4) v = max(v, (uint32_t)__shfl_xor((int)v, 4, 64));
  if constexpr (RUN <= 8) v = max(v, (uint32_t)__shfl_xor((int)v, 8, 64));
  v = max(v, (uint32_t)__shfl_xor((int)v, 16, 64));
  return max(v, (uint32_t)__shfl_xor((int)v, 32, 64));
}
// Largest finite magnitude of the 16-byte pieces of the lane's head (GROUP, RUN: head_max_u32).
template <typename H, int N, int GROUP, int RUN>
__device__ __forceinline__ float kv8_top(const uint4 (&x)[N]) {
  uint32_t top2 = 0;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    top2 = max_u16x2(top2, x[i].x & 0x7FFF7FFFu); top2 = max_u16x2(top2, x[i].y & 0x7FFF7FFFu);
    top2 = max_u16x2(top2, x[i].z & 0x7FFF7FFFu); top2 = max_u16x2(top2, x[i].w & 0x7FFF7FFFu);
  }
  uint32_t top = head_max_u32<GROUP, RUN>(max(top2 & 0xFFFFu, top2 >> 16));
  if (__builtin_amdgcn_ballot_w64(top >= Fp8<H>::kInf) != 0) {     // infinities or NaN among them: leave those out
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
    top = head_max_u32<GROUP, RUN>(t);
  }
  return Fp8<H>::bits_to_f32(top);
}
// Eight values to eight codes.
template <typename H>
__device__ __forceinline__ uint2 kv8_quantise(const uint4& a, float scale) {
  if (__builtin_amdgcn_ballot_w64(scale == pow2f(Fp8<H>::kTopExp)) == 0) return make_uint2(Fp8<H>::down4(a.x, a.y, scale), Fp8<H>::down4(a.z, a.w, scale));
  const float inv = __uint_as_float((254u << 23) - __float_as_uint(scale));      // 1 / scale
  const bool top = scale == pow2f(Fp8<H>::kTopExp);       // 256 * scale would be beyond the type: clamped in fp32
  float y[8];
  const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float v = H::of_word(w[i >> 1], i) * inv;
    y[i] = top && fabsf(v) > 240.0f && fabsf(v) < 256.0f ? copysignf(240.0f, v) : v;      // (infinities and NaN stay)
  }
  return make_uint2(fp8_down4_f32(y[0], y[1], y[2], y[3], 1.0f), fp8_down4_f32(y[4], y[5], y[6], y[7], 1.0f));
}

// ---- rows into the cache, and back ------------------------------------------------------------------------------------------------
// The users of a launch travel in the kernel's arguments: no staging, no scratch, nothing for two calls to share.  A launch with 2.6 KB of
// arguments takes 4.3 us of the host, one with 650 bytes 3.2, so that launches of few users take kernels with room for few.
constexpr int kRowUsers = 128, kFewRowUsers = 28;
struct RowsUser {
  int32_t page0;     // the entry's first page in the slab
  int32_t first;     // token that the user's first row is
  int32_t rows;
  int32_t row0;      // its first row in k and v
  int32_t unit0;     // touched tiles of the launch's users before it
};
// Of n users with ascending starts the last whose `start` is at most x (the first one's is).  A launch of one has its first user from the arguments
// at once, without the look at the starts in between.
template <int USERS, class User, class Start>
__device__ __forceinline__ User user_of(const User (&users)[USERS], int n, int x, int lane, Start start) {
  User u = users[0];
  if (n > 1) {
    int at = -1;
#pragma unroll
    for (int u0 = 0; u0 < USERS; u0 += 64) {
      const bool there = u0 + lane < n;
      at += __builtin_popcountll(__builtin_amdgcn_ballot_w64(there && start(users[there ? u0 + lane : 0]) <= x));
    }
    u = users[__builtin_amdgcn_readfirstlane(at)];
  }
  return u;
}
template <int USERS> struct RowsParams {
  void* k;           // [rows][stride] in the storage type: sources of a write, targets of a read
  void* v;
  int64_t k_stride, v_stride;   // elements between rows
  char* slab;
  int64_t page_bytes, tile_stride;   // of a page; between the tiles of an entry
  int64_t codes_off, scales_off;     // of the layer in a tile
  int32_t n_users, n_tiles, d, pad_;
  RowsUser users[USERS];
};

// A wavefront's unit of a launch: FW features of K or of V, one head or several, of the tokens of one touched tile.
struct RowsUnit {
  int is_v, f0;       // first feature
  int r0, r1;         // the tile's tokens [r0, r1) are rows of the call
  int64_t row;        // row that token r0 is
  char* tile;
};
template <int FW, int USERS>
__device__ __forceinline__ bool rows_unit(const RowsParams<USERS>& p, int lane, RowsUnit* u) {
  const int unit = __builtin_amdgcn_readfirstlane((int)(blockIdx.x * 4 + (threadIdx.x >> 6)));
  const int of_tile_sh = __builtin_ctz(p.d / FW) + 1;       // log2 of the units of a tile
  const int t = unit >> of_tile_sh, in_tile = unit - (t << of_tile_sh);
  u->is_v = in_tile & 1;
  u->f0 = (in_tile >> 1) * FW;
  if (t >= p.n_tiles) return false;
  const RowsUser us = user_of(p.users, p.n_users, t, lane, [](const RowsUser& x) { return x.unit0; });
  const int tile = us.first / kTile + (t - us.unit0);
  u->r0 = max(us.first - tile * kTile, 0);
  u->r1 = min(us.first + us.rows - tile * kTile, kTile);
  u->row = (int64_t)us.row0 + (tile * kTile + u->r0 - us.first);
  u->tile = p.slab + us.page0 * p.page_bytes + tile * p.tile_stride;
  return true;
}
template <bool ONCE>
__device__ __forceinline__ uint4 load16(const void* p) {
  const u32x4_t* x = reinterpret_cast<const u32x4_t*>(p);
  return __builtin_bit_cast(uint4, ONCE ? __builtin_nontemporal_load(x) : *x);
}

// The two orders of a unit's codes.  Rows: a lane has eight adjacent features (the same in every row) of every (512 / FW)th token.  Codes: chunk c (of FW / 16,
// head by head) as in the cache.  They meet in the wavefront's LDS, [token][feature]; V's chunks take their 16 tokens byte by byte.
template <int DH, int FW> struct UnitLayout {
  static constexpr int N = FW / 8, CHUNKS = FW / 16, PER_HEAD = DH / 16, LROW = FW + 8;
  static __device__ __forceinline__ int tok(int i, int lane) { return (i * 64 + lane) / (FW / 8); }
  static __device__ __forceinline__ int feat(int lane) { return lane % (FW / 8) * 8; }
  static __device__ __forceinline__ int64_t chunk_off(int c, int lane) { return (int64_t)(c / PER_HEAD) * (2 * kTile * DH) + (c % PER_HEAD * 64 + lane) * 16; }
  static __device__ __forceinline__ uint8_t* k_at(uint8_t* lds, int c, int lane) {      // 8 bytes here and 16 further on
    const int h = c / PER_HEAD, ch = c % PER_HEAD;
    return lds + ((ch / (DH / 32)) * 32 + (lane & 31)) * LROW + h * DH + (ch % (DH / 32)) * 32 + (lane >> 5) * 8;
  }
  static __device__ __forceinline__ uint8_t* v_at(uint8_t* lds, int c, int w, int lane) {     // word w's four tokens, LROW apart
    const int h = c / PER_HEAD, ch = c % PER_HEAD;
    return lds + ((ch & 1) * 32 + (w >> 1) * 16 + (w & 1) * 8 + 4 * (lane >> 5)) * LROW + h * DH + (ch >> 1) * 32 + (lane & 31);
  }
};
// (a wavefront's LDS is its own: its reads come behind its writes without a barrier)
__device__ __forceinline__ void wave_lds_done() {
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  __builtin_amdgcn_wave_barrier();
}

// Writes: quantises the unit's blocks anew from the tokens before r0 that they keep and the rows of the call; tokens from r1 on become zero.
// What bounds it is HBM, 2 bytes in and 1 out per value; loads are runs of FW * 2 bytes of a row (d = 512, 32 users of 8192 tokens, us: K in the codes' order, 32 bytes
// of a row at a time 175, runs of 128 bytes 157, and 137 with nothing left in the caches: 5.9 TB/s).  ONCE: more than the caches hold.
template <typename H, int DH, int FW, bool ONCE, int USERS>
__global__ __launch_bounds__(256) void kv8_write_kernel(RowsParams<USERS> p) {
  using L = UnitLayout<DH, FW>;
  constexpr int HEADS = FW / DH;
  __shared__ __attribute__((aligned(16))) uint8_t turn[4][kTile * L::LROW];
  const int lane = threadIdx.x & 63, l32 = lane & 31, g = lane >> 5;
  RowsUnit u;
  if (!rows_unit<FW>(p, lane, &u)) return;       // (no barrier below)
  uint8_t* lds = turn[threadIdx.x >> 6];
  const int64_t stride = u.is_v ? p.v_stride : p.k_stride;
  const uint16_t* src = reinterpret_cast<const uint16_t*>(u.is_v ? p.v : p.k) + stride * u.row + u.f0 + L::feat(lane);
  char* codes = u.tile + p.codes_off + (int64_t)u.f0 * (2 * kTile) + u.is_v * (kTile * DH);
  float* scale_at = reinterpret_cast<float*>(u.tile + p.scales_off) + 2 * (u.f0 / DH) + u.is_v;

  uint4 x[L::N];
#pragma unroll
  for (int i = 0; i < L::N; ++i) {
    const int r = L::tok(i, lane);
    x[i] = make_uint4(0, 0, 0, 0);
    if (r >= u.r0 && r < u.r1) x[i] = load16<ONCE>(src + (int64_t)(r - u.r0) * stride);
  }
  // codes that stay: tokens before r0
  uint4 old[L::CHUNKS];
  float old_scale[HEADS];
  if (u.r0 > 0) {
#pragma unroll
    for (int h = 0; h < HEADS; ++h) old_scale[h] = scale_at[2 * h];
#pragma unroll
    for (int c = 0; c < L::CHUNKS; ++c) old[c] = *reinterpret_cast<const uint4*>(codes + L::chunk_off(c, lane));
  }
  // which bytes of word w of chunk c stay
  auto kept = [&](int c, int w) -> uint32_t {
    const int ch = c % L::PER_HEAD;
    if (!u.is_v) return (ch / (DH / 32)) * 32 + l32 < u.r0 ? 0xFFFFFFFFu : 0u;
    const int n = min(max(u.r0 - ((ch & 1) * 32 + (w >> 1) * 16 + (w & 1) * 8 + 4 * g), 0), 4);
    return n == 4 ? 0xFFFFFFFFu : (1u << (8 * n)) - 1u;
  };

  float amax = kv8_top<H, L::N, DH / 8, FW / 8>(x);     // of the lane's head
  const int my_head = L::feat(lane) / DH;
  if (u.r0 > 0) {
#pragma unroll
    for (int h = 0; h < HEADS; ++h) {
      uint32_t t = 0;
#pragma unroll
      for (int c = h * L::PER_HEAD; c < (h + 1) * L::PER_HEAD; ++c) {
        const uint32_t w[4] = {old[c].x, old[c].y, old[c].z, old[c].w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint32_t m = w[j] & kept(c, j) & 0x7F7F7F7Fu;
#pragma unroll
          for (int b = 0; b < 4; ++b) { const uint32_t code = (m >> (8 * b)) & 0x7Fu; t = max(t, code == 0x7Fu ? 0u : code); }
        }
      }
      const f32x2_t kept_top = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(wave_max_u32(t), old_scale[h], false);
      amax = my_head == h ? fmaxf(amax, kept_top[0]) : amax;
    }
  }
  const float scale = pow2f(fp8_exponent(amax));
  float scales[HEADS];
#pragma unroll
  for (int h = 0; h < HEADS; ++h) scales[h] = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(scale), h * (DH / 8)));

#pragma unroll
  for (int i = 0; i < L::N; ++i) *reinterpret_cast<uint2*>(lds + L::tok(i, lane) * L::LROW + L::feat(lane)) = kv8_quantise<H>(x[i], scale);
  wave_lds_done();
#pragma unroll
  for (int c = 0; c < L::CHUNKS; ++c) {
    uint32_t o[4];
    if (!u.is_v) {
      const uint8_t* at = L::k_at(lds, c, lane);
      const uint2 lo = *reinterpret_cast<const uint2*>(at), hi = *reinterpret_cast<const uint2*>(at + 16);
      o[0] = lo.x; o[1] = lo.y; o[2] = hi.x; o[3] = hi.y;
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint8_t* at = L::v_at(lds, c, j, lane);
        o[j] = (uint32_t)at[0] | (uint32_t)at[L::LROW] << 8 | (uint32_t)at[2 * L::LROW] << 16 | (uint32_t)at[3 * L::LROW] << 24;
      }
    }
    if (u.r0 > 0) {
      const uint32_t w[4] = {old[c].x, old[c].y, old[c].z, old[c].w};
      const float from = old_scale[c / L::PER_HEAD], to = scales[c / L::PER_HEAD];
#pragma unroll
      for (int j = 0; j < 4; ++j) o[j] |= (from == to ? w[j] : fp8_rescale4(w[j], from, to)) & kept(c, j);     // (the call's rows left zero there)
    }
    *reinterpret_cast<uint4*>(codes + L::chunk_off(c, lane)) = make_uint4(o[0], o[1], o[2], o[3]);
  }
  if (lane < HEADS) {
    float mine = scales[0];
#pragma unroll
    for (int h = 1; h < HEADS; ++h) mine = lane == h ? scales[h] : mine;
    scale_at[2 * lane] = mine;
  }
}

// Reads: the values that the unit's tokens [r0, r1) stand for, into their rows; 1 byte in and 2 out per value (32 users of 8192 tokens, d = 512: 806 MB in 148 us,
// 5.4 TB/s; one user of 1001 tokens, 6.2 MB, 8.8, which is the launch).
template <typename H, int DH, int FW, bool ONCE, int USERS>
__global__ __launch_bounds__(256) void kv8_read_kernel(RowsParams<USERS> p) {
  using L = UnitLayout<DH, FW>;
  __shared__ __attribute__((aligned(16))) uint8_t turn[4][kTile * L::LROW];
  const int lane = threadIdx.x & 63;
  RowsUnit u;
  if (!rows_unit<FW>(p, lane, &u)) return;
  uint8_t* lds = turn[threadIdx.x >> 6];
  const int64_t stride = u.is_v ? p.v_stride : p.k_stride;
  uint16_t* dst = reinterpret_cast<uint16_t*>(u.is_v ? p.v : p.k) + stride * u.row + u.f0 + L::feat(lane);
  const char* codes = u.tile + p.codes_off + (int64_t)u.f0 * (2 * kTile) + u.is_v * (kTile * DH);
  const float scale = reinterpret_cast<const float*>(u.tile + p.scales_off)[2 * ((u.f0 + L::feat(lane)) / DH) + u.is_v];
  uint4 x[L::CHUNKS];
#pragma unroll
  for (int c = 0; c < L::CHUNKS; ++c) x[c] = load16<ONCE>(codes + L::chunk_off(c, lane));
#pragma unroll
  for (int c = 0; c < L::CHUNKS; ++c) {
    const uint32_t w[4] = {x[c].x, x[c].y, x[c].z, x[c].w};
    if (!u.is_v) {
      uint8_t* at = L::k_at(lds, c, lane);
      *reinterpret_cast<uint2*>(at) = make_uint2(w[0], w[1]);
      *reinterpret_cast<uint2*>(at + 16) = make_uint2(w[2], w[3]);
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        uint8_t* at = L::v_at(lds, c, j, lane);
#pragma unroll
        for (int b = 0; b < 4; ++b) at[b * L::LROW] = (uint8_t)(w[j] >> (8 * b));
      }
    }
  }
  wave_lds_done();
#pragma unroll
  for (int i = 0; i < L::N; ++i) {
    const int r = L::tok(i, lane);
    if (r < u.r0 || r >= u.r1) continue;
    const uint2 w = *reinterpret_cast<const uint2*>(lds + r * L::LROW + L::feat(lane));
    u32x4_t* to = reinterpret_cast<u32x4_t*>(dst + (int64_t)(r - u.r0) * stride);
    if constexpr (ONCE) __builtin_nontemporal_store(fp8_frag<H>(w.x, w.y, scale), to);
    else *to = fp8_frag<H>(w.x, w.y, scale);
  }
}

// Quantises whole tiles that are already in the order of the 16-bit layout: a pre-inference's K and V of one layer, from its scratch tiles into the
// pool.  One wavefront a block; a lane's output chunk is its pieces of two consecutive fragments, so that nothing changes lanes.  HBM and the last-level cache bound it: 16 users
// of 4096 tokens, d = 512, 134 MB in and 67 out in 33 us a layer, 6.1 TB/s.
constexpr int kTilesUsers = 64;
struct TilesUser {
  char* tile0;             // of the pool entry
  const uint16_t* src;     // the user's tile 0 in scratch, head 0
  int32_t unit0, pad_;     // tiles of the launch's users before it
};
struct TilesParams {
  int64_t tile_stride, src_stride;   // bytes between the entry's tiles; elements between scratch tiles
  int64_t codes_off, scales_off;
  int32_t n_users, n_tiles, n_heads, pad_;
  TilesUser users[kTilesUsers];
};
template <typename H, int DH>
__global__ __launch_bounds__(256) void kv8_tiles_kernel(TilesParams p) {
  constexpr int NL = DH / 8;
  const int lane = threadIdx.x & 63;
  const int unit = __builtin_amdgcn_readfirstlane((int)(blockIdx.x * 4 + (threadIdx.x >> 6)));
  const int is_v = unit & 1, t = (unit >> 1) / p.n_heads, head = (unit >> 1) - t * p.n_heads;
  if (t >= p.n_tiles) return;
  const TilesUser us = user_of(p.users, p.n_users, t, lane, [](const TilesUser& x) { return x.unit0; });
  const uint4* src = reinterpret_cast<const uint4*>(us.src + (int64_t)(t - us.unit0) * p.src_stride + (2 * head + is_v) * (kTile * DH));
  char* tile = us.tile0 + (int64_t)(t - us.unit0) * p.tile_stride;
  uint4 x[NL];
#pragma unroll
  for (int i = 0; i < NL; ++i) x[i] = src[i * 64 + lane];
  const float scale = pow2f(fp8_exponent(kv8_top<H, NL, 64, 64>(x)));
#pragma unroll
  for (int c = 0; c < NL / 2; ++c) {
    const uint2 lo = kv8_quantise<H>(x[2 * c], scale), hi = kv8_quantise<H>(x[2 * c + 1], scale);
    *reinterpret_cast<uint4*>(tile + p.codes_off + (2 * head + is_v) * (kTile * DH) + (c * 64 + lane) * 16) = make_uint4(lo.x, lo.y, hi.x, hi.y);
  }
  if (lane == 0) reinterpret_cast<float*>(tile + p.scales_off)[2 * head + is_v] = scale;
}

}  // namespace relaygr
