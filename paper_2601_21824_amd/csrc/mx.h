// mx.h -- microscaled rows: 32 components of a row share a power of two 2^e, kept
// as the byte 127 + e (255: NaN), and are stored as value / 2^e, rounded to nearest even
// in e4m3 (DASH_CACHE_MXFP8) or e2m1 (DASH_CACHE_MXFP4, the lower half of a byte first).
//
// e is the least exponent with which the block's largest value is in range, largest <= 448 2^e
// (6 2^e): rounding the exponent down instead would cut up to an eighth (a quarter) off it.
// It is at least -117, with which every e4m3 value is a normal number of bf16: every
// stored value is one of bf16's, and reading a row rounds nothing.  Values from 1.5 2^127
// on count as that for e, and saturate; a block that holds a NaN or an infinity reads as NaN.
#pragma once
#include <stdint.h>

#if defined(__HIPCC__)
#define DASH_MX_HD __host__ __device__ inline
#else
#define DASH_MX_HD inline
#endif

namespace dash {

constexpr int kMxBlock = 32;
constexpr int kMxNaN = 255, kMxLeast = 10;

// The scale byte of a block whose largest |value| has the fp32 bits `most` (NaN and infinity
// have the largest of all).  448 = 1.75 2^8 and 6 = 1.5 2^2: a larger fraction takes one more.
template <bool FP4>
DASH_MX_HD int mx_byte(uint32_t most) {
  if (most >= 0x7f800000u) return kMxNaN;
  if (most > 0x7f400000u) most = 0x7f400000u;
  const int e = (int)((most + (0x7fffffu - (FP4 ? 0x400000u : 0x600000u))) >> 23) - (FP4 ? 2 : 8);
  return e < kMxLeast ? kMxLeast : e;
}

}  // namespace dash

#if defined(__HIPCC__)
#include "common.h"
namespace dash {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// The scale of a byte, as the conversions below take it: they make NaN of every element for 255.
__device__ inline float mx_scale(unsigned byte) { return __builtin_bit_cast(float, byte << 23); }

// elements 2p, 2p + 1 of a word, times the scale, as two bf16 (exact)
template <bool FP4>
__device__ inline unsigned mx_pair(unsigned word, int p, float scale);
template <>
__device__ inline unsigned mx_pair<true>(unsigned word, int p, float scale) {
  switch (p) {  // (an immediate: p is known where this is inlined)
    case 0: return __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, scale, 0));
    case 1: return __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, scale, 1));
    case 2: return __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, scale, 2));
    default: return __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, scale, 3));
  }
}
template <>
__device__ inline unsigned mx_pair<false>(unsigned word, int p, float scale) {
  return p == 0 ? __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(word, scale, false))
                : __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(word, scale, true));
}

// largest |value| of eight, as bits
__device__ inline unsigned mx_most(const float (&y)[8]) {
  unsigned m = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const unsigned b = __builtin_bit_cast(unsigned, y[i]) & 0x7fffffffu;
    m = m > b ? m : b;
  }
  return m;
}

// eight values of a block with this scale byte -> their elements: two words of e4m3, one of e2m1
template <bool FP4>
__device__ inline u32x2 mx_pack(const float (&y)[8], int byte) {
  const bool nan = byte == kMxNaN;
  const float down = __builtin_bit_cast(float, (unsigned)(254 - (nan ? 127 : byte)) << 23);  // 2^-e
  float z[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) z[i] = nan ? 0.f : y[i] * down;
  unsigned a = 0, b = 0;
  if constexpr (FP4) {
    a = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(a, z[0], z[1], 1.f, 0);  // (saturates at 6)
    a = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(a, z[2], z[3], 1.f, 1);
    a = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(a, z[4], z[5], 1.f, 2);
    a = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(a, z[6], z[7], 1.f, 3);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) z[i] = __builtin_amdgcn_fmed3f(z[i], -448.f, 448.f);
    a = __builtin_amdgcn_cvt_pk_fp8_f32(z[0], z[1], 0, false);
    a = __builtin_amdgcn_cvt_pk_fp8_f32(z[2], z[3], a, true);
    b = __builtin_amdgcn_cvt_pk_fp8_f32(z[4], z[5], 0, false);
    b = __builtin_amdgcn_cvt_pk_fp8_f32(z[6], z[7], b, true);
  }
  return u32x2{a, b};
}

}  // namespace dash
#endif
