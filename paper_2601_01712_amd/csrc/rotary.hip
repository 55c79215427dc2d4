// C-ABI entry points of rotary positions (rotary.h).
#include "rotary.h"

#include <math.h>

#include <algorithm>

#include "../../include/relaygr.h"
#include "cache_rows.h"
#include "errors.h"

using namespace relaygr;

namespace {

// Numbers hi + lo of some 120 bits, for frequencies: of one that turns often only the fraction of a turn counts, and positions multiply what is lost of it.  (64 bits
// alone were off by 2^-48 of a turn at a base of 1e-6, 6e-5 in the angle at position 2^31.)
struct Wide { long double hi, lo; };
Wide sum(long double a, long double b) {
  const long double s = a + b, x = s - a;
  return {s, (a - (s - x)) + (b - x)};
}
Wide operator+(const Wide& a, const Wide& b) {
  const Wide s = sum(a.hi, b.hi);
  return sum(s.hi, s.lo + (a.lo + b.lo));
}
// (halves of 32 bits, whose products are exact)
Wide halves(long double x) {
  const long double y = x * 0x100000001p0L, hi = y - (y - x);
  return {hi, x - hi};
}
Wide operator*(const Wide& a, const Wide& b) {
  const long double p = a.hi * b.hi;
  const Wide x = halves(a.hi), y = halves(b.hi);
  const long double rest = ((x.hi * y.hi - p) + x.hi * y.lo + x.lo * y.hi) + x.lo * y.lo;
  return sum(p, rest + (a.hi * b.lo + a.lo * b.hi));
}
Wide operator/(const Wide& a, const Wide& b) {
  const long double q = a.hi / b.hi;
  const Wide rest = a + b * Wide{-q, 0};
  return sum(q, (rest.hi + rest.lo) / b.hi);
}

// base^(-1 / n), 0 < n <= 64: with base = m 2^e the n-th root of 2^r / m, times 2^k, k n + r = -e; the root from powl's (off by some 2^-62), of which the n-th power is off by c:
// times (1 + c)^(1 / n), to its square.
Wide root_of(double base, int n) {
  int e;
  const double m = frexp(base, &e);
  int k = -e / n, r = -e % n;
  if (r < 0) { r += n; --k; }
  const Wide of = Wide{ldexpl(1, r), 0} / Wide{m, 0};
  const long double root = powl(of.hi, 1.0L / n);
  Wide x = {root, 0}, power = {1, 0};
  for (int j = n; j > 0; j >>= 1, x = x * x)
    if (j & 1) power = power * x;
  const long double c = (of / power + Wide{-1, 0}).hi / n;
  const Wide f = sum(root, root * (c - (n - 1) / 2.0L * c * c));
  return {ldexpl(f.hi, k), ldexpl(f.lo, k)};
}

}  // namespace

extern "C" int relaygr_rope_init(relaygr_rope* out, int32_t dim, int32_t layout, double base, double factor, int32_t original_len, double low, double high,
                                 float gain) {
  static const char* what = "rope_init";
  if (!out) return fail(RELAYGR_EINVAL, "%s: null argument", what);
  if (dim < 2 || dim > 2 * kRotaryPairs || dim % 2) return fail(RELAYGR_EINVAL, "%s: %d features are not pairs of a head", what, dim);
  if (layout != RELAYGR_ROPE_HALF && layout != RELAYGR_ROPE_INTERLEAVED) return fail(RELAYGR_EINVAL, "%s: unknown layout %d", what, layout);
  if (!(base > 0) || !isfinite(base) || !(factor > 0) || !isfinite(factor) || !isfinite(gain)) return fail(RELAYGR_EINVAL, "%s: base, factor or gain", what);
  if (original_len < 0 || (original_len > 0 && (!isfinite(low) || !isfinite(high) || !(low < high)))) return fail(RELAYGR_EINVAL, "%s: original length, low or high", what);
  *out = relaygr_rope();
  out->dim = dim; out->layout = layout; out->gain = gain;
  const Wide per_turn = {0xa2f9836e4e44152ap-66L, -0x3d8a82e0acb223fp-130L};      // 1 / 2 pi
  const Wide step = root_of(base, dim / 2), shorter = Wide{1, 0} / Wide{factor, 0};
  Wide frequency = {1, 0};
  for (int i = 0; i < dim / 2; ++i, frequency = frequency * step) {
    Wide turns = frequency * per_turn, keep = {0, 0};
    if (original_len > 0) {
      keep = (turns * Wide{(long double)original_len, 0} + Wide{-(long double)low, 0}) / sum(high, -(long double)low);
      keep = keep.hi < 0 ? Wide{0, 0} : keep.hi >= 1 ? Wide{1, 0} : keep;
    }
    turns = turns * (keep + (Wide{1, 0} + Wide{-keep.hi, -keep.lo}) * shorter);
    if (!(turns.hi < 0x1p48L)) return fail(RELAYGR_EINVAL, "%s: a frequency of %Lg turns a position", what, turns.hi);      // (beyond, its fraction would be known to fewer than 64 bits)
    const Wide fraction = sum(turns.hi - floorl(turns.hi), turns.lo);
    const long double scaled = ldexpl(fraction.hi, 64), whole = floorl(scaled);
    const long double rounded = whole + floorl(scaled - whole + ldexpl(fraction.lo, 64) + 0.5L);
    out->turns[i] = rounded >= 0x1p64L ? 0 : (uint64_t)(rounded < 0 ? rounded + 0x1p64L : rounded);
  }
  return RELAYGR_OK;
}

namespace {

// Halves of pairs that are pieces of a cache line (fewer than 128 bytes): a lane takes both, each of 16 bytes, or one of them and its partners from another lane, so that lines are read and written whole.
// That costs twice the angles and a turn by way of the lanes, and is for what the caches do not hold.  us, both / one (q and k, read and written): halves of 64 bytes, 65 536 rows of 512 bf16
// (268 MB) 59.4 / 52.6, of 256 fp32 59.7 / 50.5, of 256 bf16 (134 MB) 27.6 / 29.4, 2048 of 512 5.4 / 5.9; of 32 bytes, 65 536 of 256 36.1 / 29.1, 16 384 (34 MB) 11.9 / 10.4, 4700 (10 MB) 6.9 / 6.9.
bool by_lanes(int half_bytes, int64_t bytes) { return half_bytes < 128 && bytes >= (half_bytes < 64 ? (int64_t)16 << 20 : (int64_t)192 << 20); }

// Lanes take all heads of a row while that leaves the chip enough of them: the angles are a lane's first work, some 25 instructions each, and rows that are read and written
// whole are what the memory likes.  us, eight heads a lane / four (q and k of 8 heads): 65 536 rows of 512 bf16 59.0 / 64.4, of 1024 fp32 224 / 283; 16 384 rows (131 072 lanes at
// eight) of 1024 bf16 28.9 / 25.2, of 512 fp32 28.4 / 25.0; four a lane / one: 2048 rows of 512 bf16 6.1 / 5.4, 4700 10.9 / 8.6.
template <class T>
void launch_rotary(RotaryParams p, hipStream_t st) {
  constexpr int E = RotaryType<T>::E;
  const int64_t bytes = (int64_t)p.n_rows * p.n_heads * p.dh * (16 / E) * (p.x[1].in ? 4 : 2);      // read and written
  const RotaryUnit unit = p.units_sh == 0 ? kRotaryInterleaved : (p.dim / 2) % E ? kRotaryOdd : by_lanes(p.dim / 2 * (16 / E), bytes) ? kRotaryLanes : kRotaryHalf;      // (units_sh carries the layout here)
  const int units = unit == kRotaryHalf ? p.dim / 2 / E + (p.dh - p.dim) / E : p.dh / E;
  p.units_sh = 0;
  while (1 << p.units_sh < units) ++p.units_sh;
  const int64_t lanes = (int64_t)p.n_rows << p.units_sh;
  p.heads_per = p.n_heads;
  while (p.heads_per > 1 && lanes * ((p.n_heads + p.heads_per - 1) / p.heads_per) < (p.heads_per > 4 ? 4096 : 2048) * 64) p.heads_per = (p.heads_per + 1) / 2;
  const int32_t rows = p.n_rows;
  for (int32_t row = 0; row < rows; row += p.n_rows) {
    p.n_rows = (int32_t)std::min<int64_t>(rows - row, (1ll << 31) >> p.units_sh);      // (a launch counts its threads in 32 bits)
    const dim3 grid((unsigned)((((int64_t)p.n_rows << p.units_sh) + 255) / 256), (unsigned)((p.n_heads + p.heads_per - 1) / p.heads_per));
    switch (unit) {
      case kRotaryHalf: hipLaunchKernelGGL((rotary_kernel<T, kRotaryHalf>), grid, dim3(256), 0, st, p); break;
      case kRotaryLanes: hipLaunchKernelGGL((rotary_kernel<T, kRotaryLanes>), grid, dim3(256), 0, st, p); break;
      case kRotaryInterleaved: hipLaunchKernelGGL((rotary_kernel<T, kRotaryInterleaved>), grid, dim3(256), 0, st, p); break;
      default: hipLaunchKernelGGL((rotary_kernel<T, kRotaryOdd>), grid, dim3(256), 0, st, p); break;
    }
    p.position += p.n_rows;
    for (RotaryArray& x : p.x) { x.in += x.in ? p.n_rows * x.in_stride : 0; x.out += x.in ? p.n_rows * x.out_stride : 0; }
  }
}

}  // namespace

extern "C" int relaygr_rotary(const relaygr_model_config* cfg, const relaygr_rope* rope, int32_t n_rows, const int32_t* positions, int32_t transposed,
                              const void* q, int64_t q_stride, void* q_out, int64_t q_out_stride, const void* k, int64_t k_stride, void* k_out,
                              int64_t k_out_stride, void* hip_stream) {
  static const char* what = "rotary";
  if (!cfg || !rope) return fail(RELAYGR_EINVAL, "%s: null argument", what);
  if (relaygr_kv_footprint_bytes(cfg, 1) == 0) return fail(RELAYGR_EINVAL, "%s: unsupported model configuration", what);
  const int d = cfg->d_model, dh = d / cfg->n_heads, e = elem_bytes(*cfg);
  if (rope->dim < 2 || rope->dim % 2 || rope->dim > dh) return fail(RELAYGR_EINVAL, "%s: %d features of a head of %d", what, rope->dim, dh);
  if (rope->layout != RELAYGR_ROPE_HALF && rope->layout != RELAYGR_ROPE_INTERLEAVED) return fail(RELAYGR_EINVAL, "%s: unknown layout %d", what, rope->layout);
  if (n_rows < 0) return fail(RELAYGR_EINVAL, "%s: n_rows < 0", what);
  if (n_rows == 0) return RELAYGR_OK;
  if (!positions || ((uintptr_t)positions & 3)) return fail(RELAYGR_EINVAL, "%s: positions are null or not aligned", what);
  if (!k != !k_out) return fail(RELAYGR_EINVAL, "%s: k without k_out, or k_out without k", what);
  int rc;
  if ((rc = check_rows_array(what, "q", q, q_stride, d, e)) != RELAYGR_OK || (rc = check_rows_array(what, "q_out", q_out, q_out_stride, d, e)) != RELAYGR_OK) return rc;
  if (k && ((rc = check_rows_array(what, "k", k, k_stride, d, e)) != RELAYGR_OK || (rc = check_rows_array(what, "k_out", k_out, k_out_stride, d, e)) != RELAYGR_OK)) return rc;
  if ((q == q_out && q_stride != q_out_stride) || (k && k == k_out && k_stride != k_out_stride))
    return fail(RELAYGR_EINVAL, "%s: rows in place must stay where they are", what);
  RotaryParams p = {};
  p.x[0] = {(const char*)q, (char*)q_out, q_stride * e, q_out_stride * e};
  p.x[1] = {(const char*)k, (char*)k_out, k_stride * e, k_out_stride * e};
  p.position = positions;
  p.n_rows = n_rows; p.n_heads = cfg->n_heads; p.dh = dh; p.dim = rope->dim;
  p.units_sh = rope->layout == RELAYGR_ROPE_INTERLEAVED ? 0 : 1;
  p.transposed = transposed ? 1 : 0; p.gain = rope->gain;
  for (int i = 0; i < kRotaryPairs; ++i) p.turns[i] = rope->turns[i];
  (void)hipGetLastError();
  hipStream_t st = (hipStream_t)hip_stream;
  if (cfg->dtype == RELAYGR_DTYPE_FP32) launch_rotary<float>(p, st);
  else if (cfg->dtype == RELAYGR_DTYPE_FP16) launch_rotary<F16>(p, st);
  else launch_rotary<Bf16>(p, st);
  hipError_t err = hipGetLastError();
  if (err != hipSuccess) return fail(RELAYGR_EHIP, "launch %s: %s", what, hipGetErrorString(err));
  return RELAYGR_OK;
}
