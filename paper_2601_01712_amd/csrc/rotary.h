// Rotary positions: pairs (a, b) of the first features of each head turn by an angle that grows with the row's position,
//     a' = g (a cos t - b sin t),   b' = g (a sin t + b cos t),   t = position * f_i
// for pair i of `dim / 2` pairs, (i, i + dim/2) in the half layout and (2i, 2i + 1) in the interleaved one; the features from `dim` on are copied.  The
// transposed form turns by -t: the gradient of the above, and (at g = 1) its inverse.
//
// Angles are exact whatever the position: f_i is kept as the fraction of a turn per position, times 2^64, and position times that, modulo 2^64, is the
// fraction of a turn with nothing lost but f_i's own rounding (2^-34 of a turn at position 2^31).  Its top 32 bits are cut at the nearest quarter turn, and
// sine and cosine of what is left, at most pi/4, are their power series (to x^9 and x^10: 2e-9 and 1e-10 off there, below fp32's own rounding).
#pragma once

#include "common.h"
#include "gemm.h"

namespace relaygr {

constexpr int kRotaryPairs = 64;
enum RotaryUnit { kRotaryHalf, kRotaryLanes, kRotaryInterleaved, kRotaryOdd };     // what a lane takes: two chunks half the pairs apart; a chunk whose partners are another lane's; a chunk; a chunk whose partners are not a chunk
struct RotaryArray { const char* in; char* out; int64_t in_stride, out_stride; };      // bytes between rows; in null: there is none
struct RotaryParams {
  RotaryArray x[2];
  const int32_t* position;
  int32_t n_rows, n_heads, dh, dim, units_sh, heads_per;      // log2 of the lanes of a row; heads that a lane takes
  int32_t transposed;
  float gain;
  uint64_t turns[kRotaryPairs];
};

// sin and cos of 2 pi t / 2^32.
__device__ __forceinline__ void sincos_turns(uint32_t t, float* sin_out, float* cos_out) {
  const uint32_t quarter = (t + 0x20000000u) >> 30;
  const float x = (float)(int32_t)(t - (quarter << 30)) * 1.4629180792671596e-9f, y = x * x;      // 2 pi / 2^32
  const float s = fmaf(x * y, fmaf(y, fmaf(y, fmaf(y, 2.7557319e-6f, -1.9841270e-4f), 8.3333333e-3f), -1.6666667e-1f), x);
  const float c = fmaf(y, fmaf(y, fmaf(y, fmaf(y, fmaf(y, -2.7557319e-7f, 2.4801587e-5f), -1.3888889e-3f), 4.1666667e-2f), -0.5f), 1.0f);
  const bool odd = quarter & 1;
  const float a = odd ? c : s, b = odd ? s : c;
  *sin_out = quarter & 2 ? -a : a;
  *cos_out = (quarter + 1) & 2 ? -b : b;
}

// The storage types, 16 bytes at a time.
template <class T> struct RotaryType;
template <> struct RotaryType<float> {
  static constexpr int E = 4;
  static __device__ __forceinline__ void up(const u32x4_t& w, float (&x)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = __uint_as_float(w[i]);
  }
  static __device__ __forceinline__ u32x4_t down(const float (&x)[4]) {
    return u32x4_t{__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3])};
  }
  static __device__ __forceinline__ float one(const char* p) { return *reinterpret_cast<const float*>(p); }
};
template <class H> struct RotaryType16 {
  static constexpr int E = 8;
  static __device__ __forceinline__ void up(const u32x4_t& w, float (&x)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = H::of_word(w[i >> 1], i);
  }
  static __device__ __forceinline__ u32x4_t down(const float (&x)[8]) {
    return u32x4_t{H::pack2(x[0], x[1]), H::pack2(x[2], x[3]), H::pack2(x[4], x[5]), H::pack2(x[6], x[7])};
  }
  static __device__ __forceinline__ float one(const char* p) { return H::to_f32(*reinterpret_cast<const uint16_t*>(p)); }
};
template <> struct RotaryType<Bf16> : RotaryType16<Bf16> {};
template <> struct RotaryType<F16> : RotaryType16<F16> {};

// A lane's unit of a row, in `heads_per` heads of every array: the angles are worked out once for all of them, while the first four heads are on their way.  A head's lanes are in
// one wavefront and read all that they turn before they write any of it, so that `out` may be `in`.  What bounds it is HBM, or the launch: q and k of 65 536 rows of 512 bf16, 268 MB,
// 53 us (5.1 TB/s; a copy of 1 GiB reaches 5.0), of 16 384 15.9; one row 3.8.  Half-layout pairs that are no 16-byte pieces (kRotaryOdd: `dim` / 2 not a multiple of 8, of 4 in fp32) take each
// partner by a load of its own, and these loads bound it: 60 of 64 features of the 65 536 rows 110 us where 64 of 64 take 46 on the same card, of 2048 rows 12.1 and 4.5; in fp32, at half as many
// of them for a byte, 104 and 106.
template <class T, RotaryUnit UNIT>
__global__ __launch_bounds__(256) void rotary_kernel(RotaryParams p) {
  using R = RotaryType<T>;
  constexpr int E = R::E, BYTES = 16 / E, CHUNKS = UNIT == kRotaryHalf ? 2 : 1, AT_ONCE = 4;
  const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int64_t row = id >> p.units_sh;
  const int unit = (int)(id & ((1 << p.units_sh) - 1)), half = p.dim >> 1;
  const int turned = UNIT == kRotaryHalf ? half / E : (p.dim + E - 1) / E;       // units that turn something; the others copy
  const int units = UNIT == kRotaryHalf ? turned + (p.dh - p.dim) / E : p.dh / E;
  if (row >= p.n_rows || unit >= units) return;
  const bool turns = unit < turned;
  const int f0 = UNIT == kRotaryHalf && !turns ? p.dim + (unit - turned) * E : unit * E;
  const int lane = threadIdx.x & 63, partner = !turns ? lane : f0 < half ? lane + half / E : lane - half / E;      // (kRotaryLanes: a row's lanes are side by side)
  const int head0 = blockIdx.y * p.heads_per, head1 = min(head0 + p.heads_per, p.n_heads);
  const int head_bytes = p.dh * BYTES;
  const int of_array = (head1 - head0 + AT_ONCE - 1) / AT_ONCE, batches = p.x[1].in ? 2 * of_array : of_array;
  // four heads of one array at a time, the next four on their way
  u32x4_t w[2][AT_ONCE][CHUNKS];
  float odd[2][UNIT == kRotaryOdd ? AT_ONCE : 1][E];
  auto load = [&](int batch, int slot) {
    const RotaryArray& x = p.x[batch >= of_array];
    const int h0 = head0 + (batch >= of_array ? batch - of_array : batch) * AT_ONCE;
    const char* in = x.in + row * x.in_stride + f0 * BYTES;
#pragma unroll
    for (int j = 0; j < AT_ONCE; ++j) {
      const char* at = in + (int64_t)min(h0 + j, head1 - 1) * head_bytes;
      w[slot][j][0] = *reinterpret_cast<const u32x4_t*>(at);
      if (CHUNKS == 2) w[slot][j][CHUNKS - 1] = *reinterpret_cast<const u32x4_t*>(turns ? at + half * BYTES : at);
      if constexpr (UNIT == kRotaryOdd) {
#pragma unroll
        for (int i = 0; i < E; ++i) {
          const int f = f0 + i, other = f >= p.dim ? 0 : f < half ? half : -half;
          odd[slot][j][i] = turns ? R::one(at + (i + other) * BYTES) : 0.0f;
        }
      }
    }
  };
  load(0, 0);
  float cs[E], sn[E];
#pragma unroll
  for (int i = 0; i < E; ++i) { cs[i] = 1.0f; sn[i] = 0.0f; }
  if (turns) {
    const uint64_t at = (uint64_t)(int64_t)p.position[row];
#pragma unroll
    for (int i = 0; i < E; ++i) {
      const int f = f0 + i;
      if (UNIT != kRotaryHalf && f >= p.dim) continue;
      if (UNIT == kRotaryInterleaved && (i & 1)) { cs[i] = cs[i - 1]; sn[i] = -sn[i - 1]; continue; }
      const int pair = UNIT == kRotaryInterleaved ? f >> 1 : UNIT != kRotaryHalf && f >= half ? f - half : f;
      float s, c;
      sincos_turns((uint32_t)((at * p.turns[pair]) >> 32), &s, &c);
      s = p.transposed ? -s : s;
      cs[i] = c * p.gain;
      sn[i] = (UNIT == kRotaryHalf || f < half || UNIT == kRotaryInterleaved ? -s : s) * p.gain;      // of the partner, in this element
    }
  }
  auto turn = [&](int batch, int slot) {
    const RotaryArray& x = p.x[batch >= of_array];
    const int h0 = head0 + (batch >= of_array ? batch - of_array : batch) * AT_ONCE;
    if (UNIT != kRotaryLanes && !turns && x.in == x.out) return;
    char* out = x.out + row * x.out_stride + f0 * BYTES;
#pragma unroll
    for (int j = 0; j < AT_ONCE; ++j) {
      if (h0 + j >= head1) break;
      char* at = out + (int64_t)(h0 + j) * head_bytes;
      u32x4_t other;
      if constexpr (UNIT == kRotaryLanes) {
#pragma unroll
        for (int i = 0; i < 4; ++i) other[i] = (uint32_t)__shfl((int)w[slot][j][0][i], partner, 64);
      }
      if (!turns) { *reinterpret_cast<u32x4_t*>(at) = w[slot][j][0]; continue; }
      float u[E], v[E], y[E];
      R::up(w[slot][j][0], u);
      if constexpr (UNIT == kRotaryHalf) {
        float z[E];
        R::up(w[slot][j][1], v);
#pragma unroll
        for (int i = 0; i < E; ++i) { y[i] = fmaf(u[i], cs[i], v[i] * sn[i]); z[i] = fmaf(v[i], cs[i], -u[i] * sn[i]); }
        *reinterpret_cast<u32x4_t*>(at) = R::down(y);
        *reinterpret_cast<u32x4_t*>(at + half * BYTES) = R::down(z);
      } else if constexpr (UNIT == kRotaryLanes) {
        R::up(other, v);
#pragma unroll
        for (int i = 0; i < E; ++i) y[i] = fmaf(u[i], cs[i], v[i] * sn[i]);
        *reinterpret_cast<u32x4_t*>(at) = R::down(y);
      } else {
#pragma unroll
        for (int i = 0; i < E; ++i) y[i] = fmaf(u[i], cs[i], (UNIT == kRotaryOdd ? odd[slot][j][i] : u[i ^ 1]) * sn[i]);
        u32x4_t o = R::down(y);
        if (f0 + E > p.dim) {       // (features that stay keep their bits, NaN's too)
#pragma unroll
          for (int i = 0; i < E; ++i)
            if (f0 + i >= p.dim) {
              const uint32_t keep = E == 4 ? 0xFFFFFFFFu : 0xFFFFu << (16 * (i & 1));
              const int word = E == 4 ? i : i >> 1;
              o[word] = (o[word] & ~keep) | (w[slot][j][0][word] & keep);
            }
        }
        *reinterpret_cast<u32x4_t*>(at) = o;
      }
    }
  };
  for (int batch = 0; batch < batches; batch += 2) {
    if (batch + 1 < batches) load(batch + 1, 1);
    turn(batch, 0);
    if (batch + 1 >= batches) break;
    if (batch + 2 < batches) load(batch + 2, 0);
    turn(batch + 1, 1);
  }
}

}  // namespace relaygr
