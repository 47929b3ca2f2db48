// Quantised cache rows: a row of d values is d codes of e4m3 (sign, four
// exponent and three mantissa bits, no infinities, largest value 448) and one
// exponent byte 127 + e; code c stands for c * 2^e.  e is the smallest with
// the row's largest magnitude at most 448 * 2^e, so a value down to 2^-15 of
// the largest keeps four significant bits.  A power of two rounds nothing by
// itself, the type being relative already (another factor would round once
// more, and no value nearer), and every value is exact in bf16.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "dkv_device.hpp"

namespace dkv {

typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));

// e stays within [-117, 120]: the smallest code, 2^-9, is then a normal bf16
// and 2^(127 - e) a normal fp32.
constexpr int kF8MinExp = -117, kF8MaxExp = 120;

// Exponent of a row whose largest finite magnitude has these fp32 bits.
__device__ __forceinline__ int f8_exponent(uint32_t amax) {
  // amax = f 2^k, 1 <= f < 2, and 448 = 1.75 * 2^8
  const int e = (int)(amax >> 23) - 127 - 8 + ((amax & 0x7FFFFFu) > 0x600000u ? 1 : 0);
  return e < kF8MinExp ? kF8MinExp : (e > kF8MaxExp ? kF8MaxExp : e);
}

__device__ __forceinline__ uint32_t f8_pack4(float a, float b, float c, float d) {
  const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, lo, true);
}

// 2^e of an exponent byte.
__device__ __forceinline__ float f8_power(uint32_t byte) { return __uint_as_float(byte << 23); }

// Codes 2 HALF and 2 HALF + 1 of a word times `power`, exactly, as a bf16 pair.
template <bool HALF>
__device__ __forceinline__ uint32_t f8_pair(uint32_t codes, float power) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, power, HALF));
}

}  // namespace dkv
