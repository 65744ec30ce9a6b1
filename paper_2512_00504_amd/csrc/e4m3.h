// Rows held in 8 bits: e4m3 codes times a power of two per row.
//
// A row's exponent is the smallest e >= -126 with max |x| <= 448 * 2^e, over its finite elements (e = 0 for a row of
// zeros); an element is code * 2^e with code = x * 2^-e rounded to e4m3 (1-4-3 bits, to the nearest, ties to even), at most
// 2^-4 of its value off, or 2^-10 * 2^e where it is below 2^-6 * 2^e.  e4m3 has no infinity: what is not finite is held as
// NaN.  A power of two makes the multiplications exact, so a row has the same codes however it is formed, and costs no
// precision: the codes are floating-point numbers, whose relative step does not depend on where the row's largest lies.
// The scales of a row of K and V are one 32-bit word, K's bfloat16 in the lower half and V's in the upper.
#pragma once

#include "gkv_internal.h"

#ifdef __HIPCC__
typedef float q8_f32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t q8_u32x4 __attribute__((ext_vector_type(4)));

// The scale of a row whose largest finite magnitude is amax, as the exponent field of a float: 448 = 1.75 * 2^8.
__device__ __forceinline__ uint32_t q8_scale_field(float amax) {
  const uint32_t u = __float_as_uint(amax);
  if (u == 0u) return 127u;
  const int f = (int)(u >> 23) - 8 + ((u & 0x7fffffu) > 0x600000u);
  return f < 1 ? 1u : (uint32_t)f;
}
__device__ __forceinline__ float q8_scale(uint32_t field) { return __uint_as_float(field << 23); }
__device__ __forceinline__ float q8_inverse(uint32_t field) { return __uint_as_float((254u - field) << 23); }
__device__ __forceinline__ uint32_t q8_scale_word(uint32_t k_field, uint32_t v_field) { return k_field << 7 | v_field << 23; }
__device__ __forceinline__ float q8_k_scale(uint32_t word) { return __uint_as_float(word << 16); }
__device__ __forceinline__ float q8_v_scale(uint32_t word) { return __uint_as_float(word & 0xffff0000u); }

// |x|, 0 if it is not finite.
__device__ __forceinline__ float q8_finite_magnitude(float x) {
  const uint32_t u = __float_as_uint(x) & 0x7fffffffu;
  return __uint_as_float(u >= 0x7f800000u ? 0u : u);
}
__device__ __forceinline__ float q8_scaled(float x, float inverse) {
  return (__float_as_uint(x) & 0x7fffffffu) >= 0x7f800000u ? __uint_as_float(0x7fc00000u) : x * inverse;
}
// Four codes of four elements.
__device__ __forceinline__ uint32_t q8_codes(float a, float b, float c, float d, float inverse) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(q8_scaled(a, inverse), q8_scaled(b, inverse), 0, false);
  w = __builtin_amdgcn_cvt_pk_fp8_f32(q8_scaled(c, inverse), q8_scaled(d, inverse), w, true);
  return (uint32_t)w;
}
// Codes of K meet queries as code * 2^-7 (3.5 at most, exact in bf16 too), and the 2^7 goes to the logit behind the row's scale: a query of up to 2^125
// times a code of 448 would be infinite where the logit is not.
constexpr float Q8_K_SHRUNK = 0x1p-7f, Q8_K_GROWN = 0x1p7f;
// The codes' values.
__device__ __forceinline__ void q8_values(uint32_t w, float (&x)[4]) {
  const q8_f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
  x[0] = a[0]; x[1] = a[1]; x[2] = b[0]; x[3] = b[1];
}
// The maximum of numbers that are not negative over groups of 2^log lanes (up to 32), in each of them; through registers, an exchange
// through LDS takes 60 ns.
template <int LOG>
__device__ __forceinline__ float q8_group_max(float v) {
#define GKV_Q8_DPP(ctrl) v = fmaxf(v, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), ctrl, 0xF, 0xF, false)))
  if constexpr (LOG > 0) GKV_Q8_DPP(0xB1);                   // quad_perm [1,0,3,2]
  if constexpr (LOG > 1) GKV_Q8_DPP(0x4E);                   // quad_perm [2,3,0,1]
  if constexpr (LOG > 2) GKV_Q8_DPP(LOG > 3 ? 0x124 : 0x141);   // row_ror:4, or the other quad of eight lanes (row_half_mirror)
  if constexpr (LOG > 3) GKV_Q8_DPP(0x128);                  // row_ror:8
#undef GKV_Q8_DPP
  if constexpr (LOG > 4) {
    const uint32_t u = __float_as_uint(v);
    const auto y = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    v = fmaxf(__uint_as_float(y[0]), __uint_as_float(y[1]));
  }
  return v;
}
// Byte offset of (row, 16-byte piece) in one KV head's K block whose first n_tiled rows are in tiled format.
__device__ __forceinline__ size_t q8_k_offset(int row, int piece, int d, int n_tiled) {
  return row < n_tiled ? (size_t)(row >> 4) * 16 * d + piece * 256 + (row & 15) * 16 : (size_t)row * d + piece * 16;
}
#endif  // __HIPCC__
