// 4-bit blocks (gfx950): 32 codes of 1 sign, 2 exponent and 1 mantissa bit (0, 0.5, 1,
// 1.5, 2, 3, 4, 6) and a byte s for the power of two 2^(s - 127), or for NaN where it
// is 255.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "fp8.h"
#include "wam_internal.h"

namespace wam {

constexpr int kFp4Block = WAM_FP4_BLOCK;
constexpr uint32_t kFp4NaN = 255;

// Scale byte of a block whose largest magnitude has these bits: the exponent field
// less two, so that codes reach 4 to 6 of it (subnormals, like zero, have the field 0).
__device__ __forceinline__ uint32_t fp4_scale(uint32_t most) {
  const uint32_t e = most >> 23;
  return e == 255 ? kFp4NaN : e < 2 ? 0 : e - 2;
}
// A scale byte as the operand of the conversions, which read the exponent field alone
// (0 stands for 2^-127 there too; measured at every byte).
__device__ __forceinline__ float fp4_scale_operand(uint32_t byte) { return __uint_as_float(byte << 23); }

// Codes of eight values / 2^(byte - 127): nearest, ties to the even code, magnitudes
// above 6 to 6.  A block that stands for NaN has codes of zero.
__device__ __forceinline__ uint32_t pack_fp4(const float (&x)[8], uint32_t byte) {
  const float s = fp4_scale_operand(byte);
  uint32_t w = 0;
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[0], x[1], s, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[2], x[3], s, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[4], x[5], s, 2);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[6], x[7], s, 3);
  return byte == kFp4NaN ? 0 : w;
}

typedef __bf16 bf16x2v __attribute__((ext_vector_type(2)));
typedef float f32x2v __attribute__((ext_vector_type(2)));

// Eight values of a word of codes: exact in bf16 (two significant bits) but past its range
__device__ __forceinline__ bf16x8 fp4_to_bf16(uint32_t w, float s) {
  const bf16x2v a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 0), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 1),
                c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 2), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 3);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}
__device__ __forceinline__ void fp4_to_f32(float (&x)[8], uint32_t w, float s) {
  const f32x2v a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, s, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, s, 1),
               c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, s, 2), d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, s, 3);
  x[0] = a[0], x[1] = a[1], x[2] = b[0], x[3] = b[1], x[4] = c[0], x[5] = c[1], x[6] = d[0], x[7] = d[1];
}

// The first n of the eight codes of w into ceil(n / 2) bytes at q (codes past n are zero).
__device__ __forceinline__ void store_fp4(uint8_t* q, uint32_t w, int n) {
  if (n >= 8) {
    struct __attribute__((packed, aligned(1))) Word {
      uint32_t v;
    };
    reinterpret_cast<Word*>(q)->v = w;
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (2 * i < n) q[i] = (uint8_t)(w >> (8 * i));
  }
}

// Maximum over aligned groups of 4 lanes
__device__ __forceinline__ uint32_t quad_max(uint32_t v) {
  v = max(v, dpp<0xb1>(v));
  return max(v, dpp<0x4e>(v));
}

}  // namespace wam
