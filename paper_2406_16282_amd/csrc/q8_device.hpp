// Rows in 8 bits: the arithmetic shared by the kernels that make them (gfx950, wave64).
//
// Of a row t (fp32): a = max(max |t|, 2^-100), r = fl(127 / a), q = t r rounded half to even,
// and the row stands for q scale with scale = a / 127. The row's own largest value maps to
// +-127 (t r is at most 127 (1 + 2^-24), which rounds to 127), so nothing is clamped. The
// smallest a keeps r finite and gives a row of zeros the same path. r is the only rounding
// before q: t r is formed and rounded to a whole number in one fused multiply-add (to_q8),
// so a product that lies next to a half falls on its own side of it.
// A row that holds an infinity or a NaN gets scale NaN and q = 0: every result that is
// formed from it is then NaN.
#pragma once

#include "lmbp_device.hpp"

namespace lmbp {

constexpr float kQ8Least = 0x1p-100f;

// Largest magnitude as a bit pattern: patterns of magnitudes are ordered as the values are,
// an infinity above every number and a NaN above an infinity.
__device__ inline uint32_t magnitude(float v) { return __float_as_uint(v) & 0x7fffffffu; }
__device__ inline uint32_t umax(uint32_t a, uint32_t b) { return a > b ? a : b; }
__device__ inline uint32_t wave_umax(uint32_t v) {
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) v = umax(v, uint32_t(__shfl_xor(int(v), off, kWave)));
  return v;
}

struct Q8Row {
  float a;   // largest magnitude, at least kQ8Least; NaN for a row that is not finite
  float r;   // fl(127 / a); 0 for a row that is not finite
  bool finite;
};
__device__ inline Q8Row q8_row(uint32_t most) {
  Q8Row w;
  w.finite = most < 0x7f800000u;
  const float m = __uint_as_float(most);
  w.a = w.finite ? (m > kQ8Least ? m : kQ8Least) : __uint_as_float(0x7fc00000u);
  w.r = w.finite ? 127.0f / w.a : 0.0f;
  return w;
}

// t r as a whole number in the low byte of the result (two's complement): 1.5 * 2^23 + t r
// has a unit of 1 in the last place, so the one rounding of the multiply-add is the rounding
// to a whole number, ties to even.
__device__ inline uint32_t to_q8(float t, float r) {
  return __float_as_uint(__builtin_fmaf(t, r, 12582912.0f));
}

}  // namespace lmbp
