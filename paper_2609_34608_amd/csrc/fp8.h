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

// scale of a block whose largest magnitude has these bits
__device__ __forceinline__ float block_scale(uint32_t most) {
  const float s = __uint_as_float(most) / kE4m3Max;
  return most == 0 ? 1.0f : s < kMinScale ? kMinScale : s;
}

// nearest e4m3 value, ties to even (|x| <= 448 but for a rounding; NaN stays)
__device__ __forceinline__ uint8_t to_e4m3(float x) {
  return (uint8_t)(__builtin_amdgcn_cvt_pk_fp8_f32(x, x, 0, false) & 0xff);
}

}  // namespace wam
