// Quantised cache rows: a row of d values is d codes of e4m3 (sign, four
// exponent and three mantissa bits, no infinities, largest value 448) and one
// exponent byte 127 + e; code c stands for c * 2^e.  e is the smallest with
// the row's largest magnitude at most 448 * 2^e, so that lies in (224, 448] codes
// and a value keeps four significant bits down to the least normal code, 2^-6:
// 2^-13.8 of the largest (2^-14.8 at best; rows below 448 * 2^-60, whose e would
// have to be smaller, keep fewer).  A power of two rounds nothing by itself, the
// type being relative already (another factor would round once more, and no value
// nearer), and every value is exact in bf16.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "dkv_device.hpp"

namespace dkv {

typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));

// e stays within [-60, 120].  The lower end is for attention, whose weights carry
// 2^e of V's rows (below): a row of zeros would otherwise have e = -117, and
// beside rows of 2^7 the weight of a key that counts 2^-17 of another would
// leave fp32's range, and that share of the sum with it.
constexpr int kF8MinExp = -60, kF8MaxExp = 120;
constexpr uint32_t kF8MinByte = 127 + kF8MinExp;

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

// The same codes without a power, exact in fp16.
typedef __fp16 f16x2_t __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8_t __attribute__((ext_vector_type(8)));

template <bool HALF>
__device__ __forceinline__ uint32_t f8_pair_f16(uint32_t codes) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(codes, 1.f, HALF));
}

// Attention over quantised V.  The weight of key j's codes is 2^(s_j + e_j), s_j
// its score in log2 units: the running maximum M is that of s_j + e_j in place of
// the scores', and whole (rounded up), so that the exponent byte less M is exact
// and a weight's exponent is rounded once, where it is small (a sum with the byte
// first would be rounded near 2^7: outputs off by 2.4e-6 of their norm).  The
// largest weights of a row are then near one whatever the rows of V measure, and
// two fp16 parts, cut to 11 bits each, hold 22 bits of a weight (kF8Up raises
// them by 2^7: the smaller ones then stay clear of fp16's subnormals, and 2^(7 + 8)
// of a lazy maximum below its largest), for which codes, exact in fp16, need one
// product less than bf16 parts do.  The sum of the probabilities takes 2^-e_j back, in
// fp32 (at most 2^(16 + 60) a key).  A key's share of it is lost where one factor of it
// leaves fp32's exponential, at 2^-127: its weight in its tile, below 2^-132 of the
// largest, or, sooner, a step of M, when a tile's maximum or a fold's other side
// (key waves and halves, records) raises it by 127 or more.  A key lies at most kLazy = 8
// above the M that it was summed with, and M less than one above the largest, so
// no key within 2^-118 of the largest weight is lost; with |V| below 2^25
// throughout (e_j from -60 to 17) that is a probability of 2^-41 of the largest.
// A row that has seen no key has M = kF8None.
//
// s_j + e_j - M is exact in its whole part below 2^24.  Scores beyond that are off
// by units anyway; kF8Top then keeps the exponents finite.
constexpr float kF8Up = 7.f;
constexpr float kF8Top = 16.f;  // above kF8Up and a lazy maximum's 8
constexpr float kF8None = -0x1p127f;

typedef uint16_t u16x2_t __attribute__((ext_vector_type(2)));

struct F8Keys {
  float byte[8], back[8];  // exponent byte of the lane's key, and 2^(127 - byte)
};

// From the words of the lane's keys 4kg .. 4kg + 3 of two 16-key blocks
// (exponent bytes K V K V).  A byte of V below those of the store counts as its
// least: rows of zeros may come with any (one instruction for two keys, V's
// bytes being the upper ones).
__device__ __forceinline__ F8Keys f8_keys(const uint2 (&w)[2]) {
  F8Keys k;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const u16x2_t x = __builtin_elementwise_max(__builtin_bit_cast(u16x2_t, (j & 2) ? w[j >> 2].y : w[j >> 2].x),
                                                u16x2_t(kF8MinByte << 8));
    const uint32_t b = (__builtin_bit_cast(uint32_t, x) >> ((j & 1) ? 24 : 8)) & 0xFFu;
    k.byte[j] = (float)b;
    k.back[j] = __builtin_amdgcn_ldexpf(1.f, 127 - (int)b);
  }
  return k;
}

// Two weights as two fp16 pairs: rounded towards zero, and what that left out
// (exact, in one mixed-precision instruction each; conversions and differences,
// as the compiler forms them, take two).
__device__ __forceinline__ void f16_parts(float x0, float x1, uint32_t& a, uint32_t& b) {
  a = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_pkrtz(x0, x1));
  float r0, r1;
  asm("v_fma_mix_f32 %0, %1, -1.0, %2 op_sel_hi:[1,0,0]" : "=v"(r0) : "v"(a), "v"(x0));
  asm("v_fma_mix_f32 %0, %1, -1.0, %2 op_sel:[1,0,0] op_sel_hi:[1,0,0]" : "=v"(r1) : "v"(a), "v"(x1));
  b = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_pkrtz(r0, r1));
}

}  // namespace dkv
