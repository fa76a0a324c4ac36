// Quantising a row: sixteen lanes hold it, eight channels each, so a block of 32 channels is four neighbouring lanes.
#pragma once

#include "common.h"

namespace rkv {

constexpr int kBf16 = -1;  // in the place of a format: a bf16 cache

// Bytes of a row of codes, and of a lane's eight channels of it.
template <int FMT>
struct CodeRow {
  static constexpr int kBytes = FMT == ROCKETKV_Q_E4M3 ? kHeadDim : kHeadDim / 2;
  static constexpr int kLane = kBytes / 16;
};

struct Codes8 {
  uint2 codes;     // eight bytes, or four in .x
  uint32_t scale;  // of the lane's block
};

// Largest of the block's four lanes; all four get it.
__device__ __forceinline__ uint32_t block_max_u32(uint32_t x) {
  x = max(x, (uint32_t)__builtin_amdgcn_update_dpp((int)x, (int)x, 0xb1, 0xf, 0xf, false));  // quad_perm [1, 0, 3, 2]
  return max(x, (uint32_t)__builtin_amdgcn_update_dpp((int)x, (int)x, 0x4e, 0xf, 0xf, false));  // quad_perm [2, 3, 0, 1]
}

// The block's power of two is the smallest that brings its largest magnitude m to the largest code at most, 1.75 x 2^8 or
// 1.5 x 2^2: m's exponent less 8 or 2, one more where m's mantissa is above 1.75 or 1.5, which is where adding what is
// missing to the next binade carries.  Magnitudes are compared by their bits; those of inf and NaN are the largest.
// Each value is rounded once, from fp32 to its code: to the nearest, half way to the even one.
template <int FMT>
__device__ __forceinline__ Codes8 quantise8(const float (&x)[8]) {
  [[maybe_unused]] constexpr bool kEight = FMT == ROCKETKV_Q_E4M3;
  Codes8 r = {make_uint2(0u, 0u), 0u};
#ifdef __HIP_DEVICE_COMPILE__
  uint32_t m = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) m = max(m, __float_as_uint(x[e]) & 0x7fffffffu);
  m = block_max_u32(m);
  const int scale = min(max((int)((m + (kEight ? 0x1fffffu : 0x3fffffu)) >> 23) - (kEight ? 8 : 2), 27), kEight ? 246 : 252);
  const float inv = __uint_as_float((uint32_t)(254 - scale) << 23);
  float y[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) y[e] = __builtin_amdgcn_fmed3f(x[e] * inv, kEight ? -448.f : -6.f, kEight ? 448.f : 6.f);
  if constexpr (kEight) {
    int lo = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
    lo = __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], lo, true);
    int hi = __builtin_amdgcn_cvt_pk_fp8_f32(y[4], y[5], 0, false);
    hi = __builtin_amdgcn_cvt_pk_fp8_f32(y[6], y[7], hi, true);
    r.codes = make_uint2((uint32_t)lo, (uint32_t)hi);
  } else {
    uint32_t w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, y[0], y[1], 1.f, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[2], y[3], 1.f, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[4], y[5], 1.f, 2);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[6], y[7], 1.f, 3);
    r.codes.x = w;
  }
  r.scale = (uint32_t)scale;
  if (m >= 0x7f800000u) r = {make_uint2(0u, 0u), 255u};
#endif
  return r;
}

// The same from bf16, whose conversions divide by the scale and round once as well.  What exceeds the largest code, which only
// the highest power of two for E4M3 leaves (above 1.75 x 2^127), they would make NaN.
template <int FMT>
__device__ __forceinline__ Codes8 quantise8(const uint4& v) {
  [[maybe_unused]] constexpr bool kEight = FMT == ROCKETKV_Q_E4M3;
  Codes8 r = {make_uint2(0u, 0u), 0u};
#ifdef __HIP_DEVICE_COMPILE__
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
  typedef short s16x2 __attribute__((ext_vector_type(2)));
  uint32_t w[4] = {v.x, v.y, v.z, v.w};
  const auto size = [](uint32_t pair) { return __builtin_bit_cast(u16x2, pair & 0x7fff7fffu); };
  const u16x2 most = __builtin_elementwise_max(__builtin_elementwise_max(size(w[0]), size(w[1])), __builtin_elementwise_max(size(w[2]), size(w[3])));
  const uint32_t m = block_max_u32(max((uint32_t)most.x, (uint32_t)most.y)) << 16;
  const int scale = min(max((int)((m + (kEight ? 0x1fffffu : 0x3fffffu)) >> 23) - (kEight ? 8 : 2), 27), kEight ? 246 : 252);
  const float by = __uint_as_float((uint32_t)scale << 23);
  if (kEight && __any(m > 0x7f600000u)) {
    const u16x2 limit = {0x7f60, 0x7f60};
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = (w[i] & 0x80008000u) | __builtin_bit_cast(uint32_t, __builtin_elementwise_min(size(w[i]), limit));
  }
  const auto pair = [&](int i) { return __builtin_bit_cast(bf16x2, w[i]); };
  if constexpr (kEight) {
    s16x2 lo = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(s16x2{0, 0}, pair(0), by, false);
    lo = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(lo, pair(1), by, true);
    s16x2 hi = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(s16x2{0, 0}, pair(2), by, false);
    hi = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(hi, pair(3), by, true);
    r.codes = make_uint2(__builtin_bit_cast(uint32_t, lo), __builtin_bit_cast(uint32_t, hi));
  } else {
    uint32_t x = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(0u, pair(0), by, 0);
    x = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(x, pair(1), by, 1);
    x = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(x, pair(2), by, 2);
    x = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(x, pair(3), by, 3);
    r.codes.x = x;
  }
  r.scale = (uint32_t)scale;
  if (m >= 0x7f800000u) r = {make_uint2(0u, 0u), 255u};
#endif
  return r;
}

// What eight codes stand for, in bf16, exactly.  (The conversion takes the scale's exponent alone; the highest gives NaN.)
template <int FMT>
__device__ __forceinline__ uint4 restore8(uint2 codes, uint32_t scale) {
  uint4 v = make_uint4(0u, 0u, 0u, 0u);
#ifdef __HIP_DEVICE_COMPILE__
  const float s = __uint_as_float(scale << 23);
  const auto bits = [](auto x) { return __builtin_bit_cast(uint32_t, x); };
  if constexpr (FMT == ROCKETKV_Q_E4M3) {
    v.x = bits(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)codes.x, s, false));
    v.y = bits(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)codes.x, s, true));
    v.z = bits(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)codes.y, s, false));
    v.w = bits(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)codes.y, s, true));
  } else {
    v.x = bits(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes.x, s, 0));
    v.y = bits(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes.x, s, 1));
    v.z = bits(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes.x, s, 2));
    v.w = bits(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes.x, s, 3));
  }
#endif
  return v;
}

// A lane's eight channels of the row of token `tok` (counted over the pool), `lane16` of sixteen.
template <int FMT>
__device__ __forceinline__ void store_codes(void* codes, uint8_t* scales, int64_t tok, int lane16, const Codes8& x) {
  char* at = static_cast<char*>(codes) + tok * CodeRow<FMT>::kBytes + lane16 * CodeRow<FMT>::kLane;
  if constexpr (FMT == ROCKETKV_Q_E4M3) *reinterpret_cast<uint2*>(at) = x.codes;
  else *reinterpret_cast<uint32_t*>(at) = x.codes.x;
  if (lane16 % 4 == 0) scales[tok * 4 + lane16 / 4] = (uint8_t)x.scale;
}
template <int FMT>
__device__ __forceinline__ Codes8 load_codes(const void* codes, const uint8_t* scales, int64_t tok, int lane16) {
  const char* at = static_cast<const char*>(codes) + tok * CodeRow<FMT>::kBytes + lane16 * CodeRow<FMT>::kLane;
  Codes8 x;
  if constexpr (FMT == ROCKETKV_Q_E4M3) x.codes = *reinterpret_cast<const uint2*>(at);
  else x.codes = make_uint2(*reinterpret_cast<const uint32_t*>(at), 0u);
  x.scale = scales[tok * 4 + lane16 / 4];
  return x;
}

}  // namespace rkv
