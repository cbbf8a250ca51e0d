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
  return max((int)(maximum >> 23) - 8 + ((maximum & 0x7fffffu) > 0x600000u), 1);
}
__device__ __forceinline__ float quant_factor(int byte) { return __uint_as_float((uint32_t)(254 - byte) << 23); }  // 2^-e
// Four codes: nearest, ties to even, subnormal codes included; the scaled values are at most 448, so nothing saturates.  Infinities and
// NaN become the NaN code.
__device__ __forceinline__ uint32_t quant_codes(const float (&x)[4], float f) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(x[0] * f, x[1] * f, 0, false);
  w = __builtin_amdgcn_cvt_pk_fp8_f32(x[2] * f, x[3] * f, w, true);
  uint32_t r = (uint32_t)w;
#pragma unroll
  for (int i = 0; i < 4; i++)
    if ((__float_as_uint(x[i]) & 0x7fffffffu) >= 0x7f800000u) r |= 0x7fu << (8 * i);
  return r;
}

// quantises rows of bf16 values into rows of `ldq` codes and `lds` exponents (see moe_quant_rows)
void launch_quant_rows_bf16(const void* X, int n_rows, int cols, uint8_t* Q, uint8_t* S, int64_t ldq, int64_t lds, hipStream_t st);

}  // namespace moe
