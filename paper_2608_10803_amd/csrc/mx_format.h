// The microscaled 4-bit format on gfx950: blocks of 32 values along a row, a
// scale byte s (the power of two 2^(s - 127), 255: the block is NaN) and 4-bit
// elements (sign, two bits of exponent, one of mantissa: 0, 0.5, 1, 1.5, 2, 3,
// 4, 6), two a byte, the first in the low half. Included INSIDE an unnamed
// namespace, after hip_runtime.h.

constexpr int MX_BLOCK = 32, MX_BYTES = 16;  // elements of a block, bytes of its codes

// 2^(s - 127) as fp32 (s = 0: the subnormal 2^-127; 255: NaN). The conversions
// between fp32 and 4 bits take it in this form and are exact for every s: the
// quotient by it is rounded once, to nearest even, and saturates.
__device__ __forceinline__ float mx_unit(uint32_t s) {
  return __uint_as_float(s == 0 ? 0x00400000u : s == 255 ? 0x7FC00000u : s << 23);
}
// The scale byte of a block whose largest magnitude has these bits: its
// exponent less 2, the exponent of the largest element 4 = 2^2 of full
// precision, so that the block's largest value comes to lie in [4, 8); what is
// above 6 saturates. At least 2^-127; a block with an infinity or a NaN has
// none of its values left.
__device__ __forceinline__ uint32_t mx_scale_byte(uint32_t top) {
  const uint32_t e = top >> 23;
  return e == 255 ? 255u : e > 2 ? e - 2 : 0u;
}
// Eight values to their codes.
__device__ __forceinline__ uint32_t mx_codes8(const float (&f)[8], uint32_t s) {
  const float unit = mx_unit(s);
  uint32_t c = 0;
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, f[0], f[1], unit, 0);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, f[2], f[3], unit, 1);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, f[4], f[5], unit, 2);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, f[6], f[7], unit, 3);
  return s == 255 ? 0u : c;
}
// The largest magnitude (as bits: they order as the magnitudes do, NaN above
// all) of eight values, then of the four lanes of a quad, which hold a block.
__device__ __forceinline__ uint32_t mx_top8(const float (&f)[8]) {
  uint32_t t = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) t = max(t, __float_as_uint(f[e]) & 0x7FFFFFFFu);
  return t;
}
__device__ __forceinline__ uint32_t mx_top_quad(uint32_t t) {
  t = max(t, (uint32_t)__builtin_amdgcn_mov_dpp((int)t, 0xB1, 0xF, 0xF, true));  // lanes 1 0 3 2
  return max(t, (uint32_t)__builtin_amdgcn_mov_dpp((int)t, 0x4E, 0xF, 0xF, true));  // lanes 2 3 0 1
}
// Eight codes to their values.
__device__ __forceinline__ void mx_values8(uint32_t c, uint32_t s, float (&f)[8]) {
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  const float unit = mx_unit(s);
  const f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, unit, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, unit, 1);
  const f32x2 d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, unit, 2), e = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, unit, 3);
  f[0] = a[0]; f[1] = a[1]; f[2] = b[0]; f[3] = b[1];
  f[4] = d[0]; f[5] = d[1]; f[6] = e[0]; f[7] = e[1];
}
