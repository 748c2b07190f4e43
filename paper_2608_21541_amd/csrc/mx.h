// Microscaled rows: helpers shared by the kernels that write and read them.
//
// A row of d dims is d/32 blocks of 32 consecutive dims; a block is held as 32
// codes c_i and a byte x, the values c_i 2^(x - 127).  mxfp8: a byte a code, e4m3
// (four exponent bits of bias 7, three of significand, largest 448); mxfp4: four
// bits a code, e2m1 (two exponent bits of bias 1, one of significand, largest 6),
// the even dim in the low half of a byte.  The block's exponent e = x - 127 is the
// smallest under which its largest magnitude is at most the largest code, within
// [-100, 119] (mxfp8) or [-100, 125] (mxfp4): every value is then a normal bf16
// number, so a row is read exactly whatever precision it is read in.  Only
// magnitudes beyond 2^127 times 1.75 or 1.5 saturate.  A block that held a
// non-finite value is x = 255 with codes 0, and reads as NaN.
#pragma once

#include "common.h"

namespace certkv {

template <int F>
struct MxFormat;
template <>
struct MxFormat<CERTKV_CACHE_MXFP8> {
  static constexpr int kBits = 8, kTopExp = 8, kLastExp = 119;
  static constexpr uint32_t kTopFrac = 0x600000u;  // of 448 = 1.75 x 2^8
  static constexpr float kMost = 448.f;
};
template <>
struct MxFormat<CERTKV_CACHE_MXFP4> {
  static constexpr int kBits = 4, kTopExp = 2, kLastExp = 125;
  static constexpr uint32_t kTopFrac = 0x400000u;  // of 6 = 1.5 x 2^2
  static constexpr float kMost = 6.f;
};
constexpr int kMxBlock = 32, kMxMinExp = -100;

// Bytes of a row's codes.
__host__ __device__ constexpr int mx_row_bytes(int format, int d) {
  return format == CERTKV_CACHE_BF16 ? 2 * d : format == CERTKV_CACHE_MXFP8 ? d : d / 2;
}

// The block exponent for the largest magnitude whose bits are m (finite).
template <int F>
__device__ __forceinline__ int mx_exponent(uint32_t m) {
  const int e = (int)(m >> 23) - 127 - MxFormat<F>::kTopExp +
                ((m & 0x7fffffu) > MxFormat<F>::kTopFrac ? 1 : 0);
  return min(max(e, kMxMinExp), MxFormat<F>::kLastExp);
}
// 2^e for a normal exponent.
__device__ __forceinline__ float mx_pow2(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }
// The scale of byte x (NaN for 255).
__device__ __forceinline__ float mx_scale(uint32_t x) {
  return __uint_as_float(x == 255u ? 0x7fc00000u : x << 23);
}

// Eight values, already divided by the block's scale, to codes: ties to even, larger
// magnitudes to the largest code.  mxfp8: eight bytes; mxfp4: the low word.
template <int F>
__device__ __forceinline__ uint2 mx_encode8(const float y[8]) {
  float c[8];
#pragma unroll
  for (int i = 0; i < 8; ++i)
    c[i] = __builtin_amdgcn_fmed3f(y[i], -MxFormat<F>::kMost, MxFormat<F>::kMost);
  if constexpr (F == CERTKV_CACHE_MXFP8) {
    int lo = 0, hi = 0;
    lo = __builtin_amdgcn_cvt_pk_fp8_f32(c[0], c[1], lo, false);
    lo = __builtin_amdgcn_cvt_pk_fp8_f32(c[2], c[3], lo, true);
    hi = __builtin_amdgcn_cvt_pk_fp8_f32(c[4], c[5], hi, false);
    hi = __builtin_amdgcn_cvt_pk_fp8_f32(c[6], c[7], hi, true);
    return make_uint2((uint32_t)lo, (uint32_t)hi);
  } else {
    uint32_t w = 0;
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, c[0], c[1], 1.f, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, c[2], c[3], 1.f, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, c[4], c[5], 1.f, 2);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, c[6], c[7], 1.f, 3);
    return make_uint2(w, 0u);
  }
}

typedef __bf16 mx_bf16x2 __attribute__((ext_vector_type(2)));

// Two codes to two bf16 values (the first dim in the low half): the codes of
// 16-bit half I of w (mxfp8) or of byte I (mxfp4), times scale, a power of two.
template <int F, int I>
__device__ __forceinline__ uint32_t mx_decode2(uint32_t w, float scale) {
  if constexpr (F == CERTKV_CACHE_MXFP8)
    return __builtin_bit_cast(uint32_t, (mx_bf16x2)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(
                                            w, scale, I == 1));
  else
    return __builtin_bit_cast(uint32_t,
                              (mx_bf16x2)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, I));
}

// Eight codes (mxfp8: both words; mxfp4: x) to eight bf16 values.
template <int F>
__device__ __forceinline__ uint4 mx_decode8(uint2 c, float scale) {
  if constexpr (F == CERTKV_CACHE_MXFP8)
    return make_uint4(mx_decode2<F, 0>(c.x, scale), mx_decode2<F, 1>(c.x, scale),
                      mx_decode2<F, 0>(c.y, scale), mx_decode2<F, 1>(c.y, scale));
  else
    return make_uint4(mx_decode2<F, 0>(c.x, scale), mx_decode2<F, 1>(c.x, scale),
                      mx_decode2<F, 2>(c.x, scale), mx_decode2<F, 3>(c.x, scale));
}

}  // namespace certkv
