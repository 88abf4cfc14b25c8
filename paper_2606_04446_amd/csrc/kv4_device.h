// Device helpers of the 4-bit cache: E2M1 elements in blocks of 32 that share
// a power of two (layout and rounding: d2sd_kv4_cache in d2sd.h).
#pragma once

#include "common.h"

namespace d2sd {

namespace {

constexpr int kKv4Dim = D2SD_HEAD_DIM;
constexpr int kKv4RowBytes = kKv4Dim / 2;          // codes of a (token, KV head) row
constexpr int kKv4Blocks = kKv4Dim / 32;           // scale bytes of a row
constexpr int kKv4PageBytes = D2SD_PAGE_SIZE * kKv4RowBytes;
constexpr int kScaleMin = 3, kScaleMax = 252, kScaleNan = 255;   // bytes the quantiser writes

// Scale byte of a block whose largest magnitude has these bits: the smallest
// 2^e >= top / 7. With top = m 2^x, m in [0.5, 1): 7 = 0.875 * 2^3, so e is
// x - 3 for m <= 0.875 and x - 2 above, and 0.875 is mantissa field 0x600000.
// Subnormal tops have field 0 and end at the lower bound, infinities and NaN
// have field 255.
__device__ __forceinline__ int kv4_scale_byte(uint32_t top_bits) {
  const int field = (int)(top_bits >> 23);
  if (field == 255) return kScaleNan;
  const int e = field - ((top_bits & 0x7fffffu) <= 0x600000u ? 2 : 1);   // x = field - 126
  return clampi(e, kScaleMin, kScaleMax);
}

// Scale operand of the conversions for a scale byte: they read its exponent
// field only, 255 (an infinity here) as NaN.
__device__ __forceinline__ float kv4_scale(uint32_t byte) { return __uint_as_float(byte << 23); }

// Codes of eight values, the first in the lowest bits: x / scale rounded to
// the nearest E2M1 value, ties to even, saturating at 6.
__device__ __forceinline__ uint32_t kv4_encode8(const float (&x)[8], float scale) {
  uint32_t r = 0;
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[0], x[1], scale, 0);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[2], x[3], scale, 1);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[4], x[5], scale, 2);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[6], x[7], scale, 3);
  return r;
}

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

// Eight codes to bf16 (exact) and to fp32.
__device__ __forceinline__ uint4 kv4_decode8_bf16(uint32_t c, float scale) {
  uint4 r;
  r.x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 0));
  r.y = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 1));
  r.z = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 2));
  r.w = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 3));
  return r;
}
__device__ __forceinline__ void kv4_decode8(uint32_t c, float scale, float (&v)[8]) {
  const f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, scale, 0);
  const f32x2 b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, scale, 1);
  const f32x2 d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, scale, 2);
  const f32x2 e = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, scale, 3);
  v[0] = a[0]; v[1] = a[1]; v[2] = b[0]; v[3] = b[1]; v[4] = d[0]; v[5] = d[1]; v[6] = e[0]; v[7] = e[1];
}

}  // namespace

}  // namespace d2sd
