// Rows held in 8 bits: groups of 32 values in E4M3 with one power of two (octo_mx8_rows).
#pragma once
#include "mfma_common.h"

namespace octo {

// Exponent byte of a group whose largest magnitude has these bits: the smallest power of two that brings it within 448 = 1.75 * 2^8 (the sum carries into the
// exponent exactly where the mantissa is above 1.75).  Infinities and NaN have larger bits than all numbers.
__device__ __forceinline__ int mx8_exp(unsigned most) { return max((int)((most + 0x1FFFFFu) >> 23) - 8, 1); }
// 2^(127 - e) for that byte, and 2^(e - 127)
__device__ __forceinline__ float mx8_inverse(int e) { return __uint_as_float((unsigned)(254 - e) << 23); }
__device__ __forceinline__ float mx8_scale(int e) { return __uint_as_float((unsigned)e << 23); }
// Four codes: values within 448 once scaled, so the conversion needs no clamp (it rounds to nearest, ties to even).
__device__ __forceinline__ unsigned mx8_pack4(floatx4 v, float inverse) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(v[0] * inverse, v[1] * inverse, 0, false);
  return (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(v[2] * inverse, v[3] * inverse, w, true);
}
constexpr unsigned MX8_NAN4 = 0x7F7F7F7Fu;      // codes of a group that holds a NaN or an infinity; its exponent byte is 255

inline bool mx8_ok(const octo_mx8_rows& r) {
  return r.d_codes && r.d_exps && !((uintptr_t)r.d_codes & 15) && r.code_row >= 0 && r.exp_row >= 0 && !(r.code_row & 15);
}

}  // namespace octo
