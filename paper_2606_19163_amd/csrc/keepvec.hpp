// Eight channels to and from kept rows (keep.hip, kgrad.hip).  A group's byte b
// of exponents stands for 2^(b - 126), whose bits are (b + 1) << 23; 255 for NaN.
#pragma once

#include "rowvec.hpp"

namespace pulse {

__device__ __forceinline__ uint32_t abs_bits(float v) { return __float_as_uint(v) & 0x7fffffffu; }

// the byte of the group whose largest |value| has the bits m: 64 <= |value|
// 2^-e < 127.5, which rounds to at most 127 (127.5 itself rounds to 128).  At
// 2^121, where 128 of them are past fp32, it stops.
__device__ __forceinline__ uint32_t keep_exp(uint32_t m) {
  if (m >= 0x7f800000u) return 255;
  const int e = (int)(m >> 23) - 7 + ((m & 0x7fffffu) >= 0x7f0000u);
  return (uint32_t)min(max(e, 0), 247);
}

// bits of a largest value over the four lanes of a group (NaN is above inf)
__device__ __forceinline__ uint32_t group_max(uint32_t m) {
  m = max(m, __float_as_uint(dpp<DPP_XOR1>(__uint_as_float(m))));
  return max(m, __float_as_uint(dpp<DPP_XOR2>(__uint_as_float(m))));
}

// round(v[0..4) inv) as four signed bytes, cut to [-127, 127]: the sum with 1.5
// 2^23 rounds to a whole number, to nearest even, whose low byte is at the bottom
__device__ __forceinline__ uint32_t bytes4(const float* v, float inv) {
  constexpr float MAGIC = 12582912.f;
  uint32_t b[4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
    b[i] = __float_as_uint(
        __builtin_amdgcn_fmed3f(fmaf(v[i], inv, MAGIC), MAGIC - 127.f, MAGIC + 127.f));
  return __builtin_amdgcn_perm(__builtin_amdgcn_perm(b[3], b[2], 0x0c0c0400u),
                               __builtin_amdgcn_perm(b[1], b[0], 0x0c0c0400u), 0x05040100u);
}

__device__ __forceinline__ void keep8(const float (&v)[8], uint8_t* q, uint8_t* e, bool first) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) m = max(m, abs_bits(v[i]));
  const uint32_t b = keep_exp(group_max(m));
  const float inv = b == 255 ? 0.f : __uint_as_float((253u - b) << 23);
  *reinterpret_cast<uint2*>(q) = uint2{bytes4(v, inv), bytes4(v + 4, inv)};
  if (first) *e = (uint8_t)b;
}

__device__ __forceinline__ float keep_step(uint32_t b) {
  return b == 255 ? __uint_as_float(0x7fc00000u) : __uint_as_float((b + 1) << 23);
}

__device__ __forceinline__ void unkeep4(float* v, uint32_t w, float step) {
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = (float)(int8_t)(w >> (8 * i)) * step;
}

__device__ __forceinline__ void load8(float (&v)[8], const uint8_t* q, uint32_t b) {
  const uint2 w = *reinterpret_cast<const uint2*>(q);
  const float step = keep_step(b);
  unkeep4(v, w.x, step);
  unkeep4(v + 4, w.y, step);
}

}  // namespace pulse
