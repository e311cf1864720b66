// Microscaled 8-bit integers: blocks of 32 consecutive values of a row, each an
// int8 -127..127 under one scale 2^(s - 127), s = floor(log2 m) - 6 + 127 for the
// block's largest absolute value m (at least 0), so that m is 64 to 128 steps.
// s = 255: the block holds no numbers.
#pragma once

#include "luffy_common.h"

namespace luffy {

// A matrix of them: q [rows, cols] int8, s [ceil(cols / 256)][rows][8].
struct Kept8 {
  uint8_t* q;
  uint8_t* s;
  int rows;
};

// s from the float32 bits of the largest absolute value.
__device__ __forceinline__ uint32_t mx8_exponent(uint32_t most) {
  const uint32_t ex = most >> 23;
  return ex == 255u ? 255u : (ex > 6u ? ex - 6u : 0u);
}
// 2^(127 - s), s <= 248.
__device__ __forceinline__ float mx8_inverse(uint32_t s) { return __uint_as_float((254u - s) << 23); }
// 2^(s - 127), NaN for 255.
__device__ __forceinline__ float mx8_scale(uint32_t s) {
  return s == 255u ? __uint_as_float(0x7FC00000u) : s == 0u ? __uint_as_float(0x00400000u) : __uint_as_float(s << 23);
}
// Four values as int8, the first in the low byte: adding 1.5 2^23 leaves the
// integer nearest to v / scale (halfway to even: the product is exact) in the low
// bits; 128, which values above 127.5 steps would round to, becomes 127.
__device__ __forceinline__ uint32_t mx8_pack(float a, float b, float c, float d, float inverse) {
  constexpr float kMagic = 12582912.0f;
  auto code = [&](float v) {
    return __float_as_uint(__builtin_amdgcn_fmed3f(fmaf(v, inverse, kMagic), kMagic - 127.0f, kMagic + 127.0f));
  };
  const uint32_t lo = __builtin_amdgcn_perm(code(b), code(a), 0x0C0C0400u);
  const uint32_t hi = __builtin_amdgcn_perm(code(d), code(c), 0x04000C0Cu);
  return lo | hi;
}
// Their values (exact in float32 and in bf16).
__device__ __forceinline__ void mx8_unpack(uint32_t w, float scale, float (&v)[4]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = static_cast<float>(static_cast<int8_t>(w >> (8 * i))) * scale;
}

}  // namespace luffy
