// e4m3 blocks (gfx950): 8-bit floats of 4 exponent and 3 mantissa bits, largest
// value 448, no infinity, with a float32 scale per block of 128 columns.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace wam {

constexpr int kScaleBlock = 128;
constexpr float kE4m3Max = 448.0f;
constexpr float kMinScale = 1.17549435e-38f;  // 2^-126: x / scale stays finite

// |x| as bits: its order as an unsigned integer is that of the magnitudes, with
// infinity above every number and NaN above infinity, so a maximum keeps both
__device__ __forceinline__ uint32_t abs_bits(float x) { return __float_as_uint(x) & 0x7fffffffu; }

__device__ __forceinline__ uint32_t wave_max(uint32_t v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v = max(v, (uint32_t)__shfl_xor((int)v, o, 64));
  return v;
}

// Maximum over aligned groups of N = 8 or 16 lanes, in every lane of the group,
// on the data-parallel crossbar (lane ^ 1, lane ^ 2, mirrored 8, mirrored 16).
template <int CTRL>
__device__ __forceinline__ uint32_t dpp(uint32_t v) {
  return (uint32_t)__builtin_amdgcn_mov_dpp((int)v, CTRL, 0xf, 0xf, false);
}
template <int N>
__device__ __forceinline__ uint32_t group_max(uint32_t v) {
  static_assert(N == 8 || N == 16, "group size");
  v = max(v, dpp<0xb1>(v));
  v = max(v, dpp<0x4e>(v));
  v = max(v, dpp<0x141>(v));
  if constexpr (N == 16) v = max(v, dpp<0x140>(v));
  return v;
}

// x / s rounded to float32 from the rounded reciprocal of s: the quotient
// estimate corrected by its exact remainder (three instructions; the compiler's
// division takes ten).  The remainder is exact above 2^-149 only, so with a small
// s both sides are first raised by 2^64.  Where s is infinite or NaN the result is
// NaN.  Its rounding comes before that to e4m3: 4 of 10^7 values (normal ones, float32
// blocks) lie so near to a border between two e4m3 values that one rounding would
// have gone to the other side, as in any form that divides in float32.
struct Divisor {
  float s, r, raise;
};
__device__ __forceinline__ Divisor divisor(float s) {
  const float raise = s < 5.421010862e-20f ? 1.8446744073709552e19f : 1.0f;  // 2^-64, 2^64
  s *= raise;
  return {s, 1.0f / s, raise};
}
__device__ __forceinline__ float divide_by(float x, const Divisor& d) {
  x *= d.raise;
  const float q = x * d.r;
  return fmaf(fmaf(-q, d.s, x), d.r, q);
}

// scale of a block whose largest magnitude has these bits
__device__ __forceinline__ float block_scale(uint32_t most) {
  const float s = __uint_as_float(most) / kE4m3Max;
  return most == 0 ? 1.0f : s < kMinScale ? kMinScale : s;
}

// four nearest e4m3 values, ties to even, as the bytes of a word
__device__ __forceinline__ uint32_t pack_e4m3(float a, float b, float c, float d) {
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false), true);
}

// nearest e4m3 value, ties to even (|x| <= 448 but for a rounding; NaN stays)
__device__ __forceinline__ uint8_t to_e4m3(float x) {
  return (uint8_t)(__builtin_amdgcn_cvt_pk_fp8_f32(x, x, 0, false) & 0xff);
}

}  // namespace wam
