// Block-scaled 8-bit tensors: e4m3 codes and, for every block of 128 consecutive values (matrices: 128 x 128), the exponent of a power
// of two.
//
// Why powers of two: a value times one is exact, so quantising rounds once and dequantising not at all; the
// matrix instruction (v_mfma_scale_f32_16x16x128_f8f6f4: 128 values of K, which is why blocks have 128) takes the exponents of both
// operands itself, so the K loop accumulates across blocks without a multiplication; and nothing is lost against any
// other scale, since codes are floating-point numbers: their relative step is 2^-4 to 2^-3 wherever their block's maximum lies in (224, 448].
#pragma once

#include "moe_common.h"

namespace moe {

constexpr int kQuantBlock = 128;
inline int64_t quant_blocks(int64_t n) { return (n + kQuantBlock - 1) / kQuantBlock; }
inline int64_t quant_row(int64_t n) { return quant_blocks(n) * kQuantBlock; }  // bytes of a row of codes

// |x| as bits, 0 for infinities and NaN (they are no part of a block's maximum)
__device__ __forceinline__ uint32_t finite_bits(float x) {
  const uint32_t a = __float_as_uint(x) & 0x7fffffffu;
  return a < 0x7f800000u ? a : 0u;
}
// Exponent byte of a block whose largest finite magnitude has these bits: e + 127 for the smallest e with maximum <= 448 * 2^e
// (448 = 1.75 * 2^8), e at least -126 (2^-e is then a normal number, too); e = 0 for a block of zeros.
__device__ __forceinline__ int quant_exponent(uint32_t maximum) {
  if (maximum == 0) return 127;
  return max((int)((maximum + 0x1fffffu) >> 23) - 8, 1);  // (a mantissa above 0.75 carries into the exponent)
}
__device__ __forceinline__ float quant_factor(int byte) { return __uint_as_float((uint32_t)(254 - byte) << 23); }  // 2^-e
// Four codes: nearest, ties to even, subnormal codes included; the scaled values are at most 448, so none saturates.  The conversion makes NaN codes of
// infinities and NaN.
__device__ __forceinline__ uint32_t quant_codes(const float (&x)[4], float f) {
  const int w = __builtin_amdgcn_cvt_pk_fp8_f32(x[0] * f, x[1] * f, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x[2] * f, x[3] * f, w, true);
}
// maxima over the sixteen lanes of a row, in all of them (in-register rotations: a launch of 124 us took 170 with exchanges through LDS once its
// epilogue quantised its two outputs, 145 with these; several at a time, because a rotation may read what was written only two instructions later)
template <int ROTATE, int N>
__device__ __forceinline__ void rotate_max(int (&v)[N]) {
#pragma unroll
  for (int n = 0; n < N; n++) v[n] = max(v[n], __builtin_amdgcn_update_dpp(0, v[n], 0x120 + ROTATE, 0xf, 0xf, false));
}
template <int N>
__device__ __forceinline__ void row_max16(int (&v)[N]) {
  rotate_max<8>(v);
  rotate_max<4>(v);
  rotate_max<2>(v);
  rotate_max<1>(v);
}
// Blocks of 128 bf16 values, eight of each in each of sixteen lanes: the lane's codes and the blocks' exponent bytes.  With 0x80 added to their magnitudes
// infinities and NaN are negative 16-bit numbers and lose against every finite value.  `there`: 0xffffffff, or 0 in lanes whose values are not part of
// the blocks (codes of zero).
template <int N>
__device__ __forceinline__ void quant_blocks_bf16(const uint32_t (&v)[N][4], uint32_t there, uint2 (&codes)[N], int (&e)[N]) {
  typedef __attribute__((ext_vector_type(2))) int16_t i16x2_t;
  typedef __attribute__((ext_vector_type(2))) uint16_t u16x2_t;
  typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2_t;
  i16x2_t m[N];
  const uint32_t magnitude = 0x7fff7fffu & there;
#pragma unroll
  for (int n = 0; n < N; n++) m[n] = i16x2_t{0x80, 0x80};
#pragma unroll
  for (int i = 0; i < 4; i++)
#pragma unroll
    for (int n = 0; n < N; n++) {
      const u16x2_t t = __builtin_bit_cast(u16x2_t, v[n][i] & magnitude) + u16x2_t{0x80, 0x80};
      m[n] = __builtin_elementwise_max(m[n], __builtin_bit_cast(i16x2_t, t));
    }
  int a[N];
#pragma unroll
  for (int n = 0; n < N; n++) a[n] = max((int)m[n][0], (int)m[n][1]);
  row_max16(a);
#pragma unroll
  for (int n = 0; n < N; n++) {
    e[n] = quant_exponent((uint32_t)(a[n] - 0x80) << 16);
    const float scale = __uint_as_float((uint32_t)e[n] << 23);  // 2^e: the conversion divides by it
    i16x2_t c[2] = {};
#pragma unroll
    for (int i = 0; i < 2; i++) {
      c[i] = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(c[i], __builtin_bit_cast(bf16x2_t, v[n][2 * i]), scale, false);
      c[i] = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(c[i], __builtin_bit_cast(bf16x2_t, v[n][2 * i + 1]), scale, true);
    }
    codes[n] = make_uint2(__builtin_bit_cast(uint32_t, c[0]) & there, __builtin_bit_cast(uint32_t, c[1]) & there);
  }
}

}  // namespace moe
