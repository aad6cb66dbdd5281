// What a byte of the 8-bit cache stands for (kv_q8.hip has the format).
#pragma once

#include "common.h"

namespace ipdv {

// The scale of a scale byte: 2^(byte - 127); 255 marks a row of NaN.
__device__ __forceinline__ float scale_value(unsigned byte) {
  return __uint_as_float(byte == 255u ? 0x7fc00000u : byte << 23);
}

// Eight e4m3 values times their row's scale.
__device__ __forceinline__ void values8(unsigned lo, unsigned hi, float f, float (&x)[8]) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const unsigned w = i ? hi : lo;
    const auto a = __builtin_amdgcn_cvt_pk_f32_fp8(w, false);
    const auto b = __builtin_amdgcn_cvt_pk_f32_fp8(w, true);
    x[4 * i + 0] = a[0] * f;
    x[4 * i + 1] = a[1] * f;
    x[4 * i + 2] = b[0] * f;
    x[4 * i + 3] = b[1] * f;
  }
}

}  // namespace ipdv
