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

// The block maximum over its four lanes (bits of magnitudes order as numbers do).
__device__ __forceinline__ uint32_t mx_max4(uint32_t x) {
  x = max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0xB1, 0xf, 0xf, true));  // lanes 1 0 3 2
  x = max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x4E, 0xf, 0xf, true));  // lanes 2 3 0 1
  return x;
}

// A lane's eight dims of a row to codes and, from the first of the block's four
// lanes, the scale byte.
template <int F>
__device__ __forceinline__ void mx_store8(const Geo& g, const float x[8], int64_t at,
                                          uint8_t* __restrict__ codes,
                                          uint8_t* __restrict__ scales) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(x[i]) & 0x7fffffffu);
  m = mx_max4(m);
  const bool bad = m >= 0x7f800000u;
  const int e = bad ? 0 : mx_exponent<F>(m);
  const float inv = mx_pow2(-e);
  float y[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) y[i] = bad ? 0.f : x[i] * inv;  // (exact, or far below a code)
  const uint2 c = mx_encode8<F>(y);
  if constexpr (F == CERTKV_CACHE_MXFP8)
    *reinterpret_cast<uint2*>(codes + at) = c;
  else
    *reinterpret_cast<uint32_t*>(codes + at / 2) = c.x;
  if ((threadIdx.x & 3) == 0) scales[at / kMxBlock] = bad ? 255u : (uint8_t)(e + 127);
  if (bad) report_nonfinite(g);
}

typedef uint32_t MxU4 __attribute__((ext_vector_type(4)));
typedef float MxF4 __attribute__((ext_vector_type(4)));
template <typename T>
struct MxRaw;  // eight values as they are loaded
template <>
struct MxRaw<uint16_t> {
  uint4 a;
  __device__ __forceinline__ void load(const uint16_t* p) {
    const MxU4 v = __builtin_nontemporal_load(reinterpret_cast<const MxU4*>(p));
    a = make_uint4(v[0], v[1], v[2], v[3]);
  }
  __device__ __forceinline__ void values(float x[8]) const {
    const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = bf16_lo(w[i]);
      x[2 * i + 1] = bf16_hi(w[i]);
    }
  }
};
template <>
struct MxRaw<float> {
  float4 a, b;
  __device__ __forceinline__ void load(const float* p) {
    const MxF4 v = __builtin_nontemporal_load(reinterpret_cast<const MxF4*>(p));
    const MxF4 w = __builtin_nontemporal_load(reinterpret_cast<const MxF4*>(p) + 1);
    a = make_float4(v[0], v[1], v[2], v[3]);
    b = make_float4(w[0], w[1], w[2], w[3]);
  }
  __device__ __forceinline__ void values(float x[8]) const {
    x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w;
    x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
  }
};

}  // namespace certkv
