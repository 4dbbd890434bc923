// Device building blocks of the bounded cache (include/compresskv_cache.h):
// the kernels' view of a cache and the 4-bit rows.
#pragma once

#include "ckv_device.h"

namespace ckv {

enum CacheType : int { kCacheF32 = 0, kCacheBf16 = 1, kCacheFp4 = 2 };   // CKV_F32, CKV_BF16, CKV_FP4

// A cache as the kernels see it.  Group bg = b * Hkv + g.
struct CacheView {
  char *k, *v;                   // rows [groups][capacity][row bytes]
  uint8_t *k_scale, *v_scale;    // 4-bit rows: [groups][capacity][D / 32]
  int32_t *pos;
  float *weight;
  int32_t *len, *seen;
  int32_t groups, Hkv, capacity;
};

// Live slots of a group, whatever the caller left in len.
__device__ __forceinline__ int live_slots(const CacheView &c, int bg) {
  return min(max(c.len[bg], 0), c.capacity);
}

// 2^(byte - 127), and NaN-making infinity for the byte 255 (the conversion
// instructions read the exponent alone and give NaN for 255).
__device__ __forceinline__ float fp4_scale(uint32_t byte) { return __uint_as_float(byte << 23); }

// The scale byte of a block whose largest magnitude has the fp32 bits `top`:
// the smallest e with top <= 7 * 2^e, which keeps the rounding of the largest
// value within half of the last step (6 stands for up to 7).
__device__ __forceinline__ uint32_t fp4_scale_byte(uint32_t top) {
  if (top >= 0x7F800000u) return 255u;   // an infinity or a NaN in the block
  const int e = (int)(top >> 23) - 2 + ((top & 0x7FFFFFu) > 0x600000u ? 1 : 0);
  return (uint32_t)min(max(e, 27), 252);
}

// Four values pairs -> the eight codes of a dword (code 2i of pair i lowest).
__device__ __forceinline__ uint32_t fp4_codes(const float (&x)[8], uint32_t byte) {
  const float s = fp4_scale(byte);
  uint32_t w = 0;
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[0], x[1], s, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[2], x[3], s, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[4], x[5], s, 2);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[6], x[7], s, 3);
  return byte == 255u ? 0u : w;
}

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// Eight codes -> eight bf16 values, exact (two bits of mantissa, an exponent).
__device__ __forceinline__ uint4 fp4_values(uint32_t w, float scale) {
  uint4 r;
  r.x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0));
  r.y = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1));
  r.z = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2));
  r.w = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3));
  return r;
}

}  // namespace ckv
