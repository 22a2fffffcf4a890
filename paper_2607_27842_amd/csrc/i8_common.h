// 8-bit integers with an fp32 scale: what the kernels that write or read them share.
//   s = max(largest |v|, 2^-100) (1 / 127),   q = the integer nearest v (1 / s), ties to even
// in fp32.  The floor keeps 1 / s finite, so that zeros give zeros; |v| (1 / s) <= 127 (1 + 2^-21), which
// rounds to 127.  A NaN or an infinity has no integer: it makes the scale NaN, and so every value
// that goes by that scale.
#pragma once
#include "dev_common.h"

namespace ff {

constexpr float kI8Floor = 0x1p-100f, kI8Step = 1.0f / 127.0f;
constexpr uint32_t kInfBits = 0x7f800000u;

// Magnitudes are compared as bit patterns: those of infinities and NaN are above all others, so that a
// maximum does not pass over a NaN.
template <int N>
__device__ __forceinline__ uint32_t top_bits(const float* v, uint32_t m = 0) {
#pragma unroll
  for (int e = 0; e < N; ++e) m = max(m, __float_as_uint(v[e]) & 0x7fffffffu);
  return m;
}
template <int CTL>
__device__ __forceinline__ uint32_t dpp_max(uint32_t x) {
  return max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, CTL, 0xf, 0xf, false));
}
// over 16 neighbouring lanes, over the wavefront; every lane receives it
__device__ __forceinline__ uint32_t top16(uint32_t x) {
  x = dpp_max<0xB1>(x);      // quad_perm [1, 0, 3, 2]
  x = dpp_max<0x4E>(x);      // quad_perm [2, 3, 0, 1]
  x = dpp_max<0x141>(x);     // row_half_mirror
  return dpp_max<0x140>(x);  // row_mirror
}
__device__ __forceinline__ uint32_t top64(uint32_t x) {
  x = top16(x);
  const auto r16 = __builtin_amdgcn_permlane16_swap(x, x, false, false);
  x = max((uint32_t)r16[0], (uint32_t)r16[1]);
  const auto r32 = __builtin_amdgcn_permlane32_swap(x, x, false, false);
  return max((uint32_t)r32[0], (uint32_t)r32[1]);
}

struct I8Scale {
  float s, inv;
  bool bad;
  __device__ __forceinline__ explicit I8Scale(uint32_t top) {
    bad = top >= kInfBits;
    s = fmaxf(__uint_as_float(bad ? 0u : top), kI8Floor) * kI8Step;
    inv = 1.0f / s;
    if (bad) s = __uint_as_float(0x7fc00000u);
  }
};
// 4 values as bytes.  x + 1.5 * 2^23 has no fraction bits left: the addition rounds x to the nearest
// integer, ties to even, and that integer's low byte is the sum's.
__device__ __forceinline__ uint32_t i8_pack4(const float* v, const I8Scale& k) {
#pragma clang fp contract(off)   // the product is rounded before the addition
  uint32_t b[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const float p = v[e] * k.inv;
    b[e] = __float_as_uint(p + 12582912.0f);
  }
  const uint32_t lo = __builtin_amdgcn_perm(b[1], b[0], 0x0c0c0400u), hi = __builtin_amdgcn_perm(b[3], b[2], 0x04000c0cu);
  return k.bad ? 0u : lo | hi;
}
__device__ __forceinline__ u32x2_t i8_pack8(const float* v, const I8Scale& k) { return u32x2_t{i8_pack4(v, k), i8_pack4(v + 4, k)}; }
__device__ __forceinline__ void i8_unpack4(uint32_t w, float* v) {
#pragma unroll
  for (int e = 0; e < 4; ++e) v[e] = (float)(int8_t)(w >> (8 * e));
}

}  // namespace ff
