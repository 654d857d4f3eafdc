// Device helpers of the row operators (bnorm.hip, keep.hip, lin8.hip): 8
// channels as fp32, sums over the lanes that share a row, activations.
#pragma once

#include "common.hpp"
#include "okernels.hpp"

namespace pulse {

// 8 channels in memory, and as fp32
template <typename T>
struct Vec8;
template <>
struct Vec8<uint16_t> {
  uint4 w;
  __device__ __forceinline__ void load(const uint16_t* p) {
    w = *reinterpret_cast<const uint4*>(p);
  }
  __device__ __forceinline__ void zero() { w = uint4{0, 0, 0, 0}; }
  __device__ __forceinline__ float get(int i) const {
    const uint32_t x = i < 2 ? w.x : i < 4 ? w.y : i < 6 ? w.z : w.w;
    return __uint_as_float(i & 1 ? x & 0xffff0000u : x << 16);
  }
};
template <>
struct Vec8<float> {
  float4 a, b;
  __device__ __forceinline__ void load(const float* p) {
    a = reinterpret_cast<const float4*>(p)[0];
    b = reinterpret_cast<const float4*>(p)[1];
  }
  __device__ __forceinline__ void zero() { a = b = make_float4(0.f, 0.f, 0.f, 0.f); }
  __device__ __forceinline__ float get(int i) const {
    const float4& x = i < 4 ? a : b;
    return (i & 3) == 0 ? x.x : (i & 3) == 1 ? x.y : (i & 3) == 2 ? x.z : x.w;
  }
};

__device__ __forceinline__ void put8(uint16_t* p, const float (&v)[8]) {
  *reinterpret_cast<uint4*>(p) =
      uint4{pack2(v[0], v[1]), pack2(v[2], v[3]), pack2(v[4], v[5]), pack2(v[6], v[7])};
}
__device__ __forceinline__ void put8(float* p, const float (&v)[8]) {
  reinterpret_cast<float4*>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
  reinterpret_cast<float4*>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
}

// v of lane ^ 1, 2 (quad permutes), of the mirrored lane of 8 and of 16
template <int CTRL>
__device__ __forceinline__ float dpp(float v) {
  return __int_as_float(
      __builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, true));
}
constexpr int DPP_XOR1 = 0xb1, DPP_XOR2 = 0x4e, DPP_HALF_MIRROR = 0x141, DPP_MIRROR = 0x140;

struct Add {
  __device__ __forceinline__ float operator()(float a, float b) const { return a + b; }
};

// op over the 16 (32, 64) lanes that hold a row, the same on each: vector
// instructions alone, where a shuffle would go through LDS
template <int L, class Op>
__device__ __forceinline__ float lanes_op(float v, Op op) {
  v = op(v, dpp<DPP_XOR1>(v));
  v = op(v, dpp<DPP_XOR2>(v));
  v = op(v, dpp<DPP_HALF_MIRROR>(v));
  v = op(v, dpp<DPP_MIRROR>(v));
  if constexpr (L >= 32) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false,
                                                    false);
    v = op(__uint_as_float(r[0]), __uint_as_float(r[1]));
  }
  if constexpr (L >= 64) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false,
                                                    false);
    v = op(__uint_as_float(r[0]), __uint_as_float(r[1]));
  }
  return v;
}

// Threads of a block whose rows take L lanes each: rows of up to a wave share
// a block of four waves, longer ones have a block of their own.
template <int L>
constexpr int ROW_THREADS = L > 64 ? L : 256;

// sums of a and b over the L lanes of a row.  L > 64 takes the whole block and
// L / 32 floats of LDS, which alternate between two such sets.
template <int L>
__device__ __forceinline__ void row_sums(float& a, float& b, float* sm, int& turn) {
  a = lanes_op<(L > 64 ? 64 : L)>(a, Add());
  b = lanes_op<(L > 64 ? 64 : L)>(b, Add());
  if constexpr (L > 64) {
    constexpr int W = L / 64;
    float2* s = reinterpret_cast<float2*>(sm) + W * turn;
    turn ^= 1;
    if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = make_float2(a, b);
    __syncthreads();
    a = b = 0.f;
#pragma unroll
    for (int w = 0; w < W; ++w) {
      const float2 v = s[w];
      a += v.x;
      b += v.y;
    }
  }
}

// Activations of fp32 values, to the accuracy of the type T that the result is stored
// in: for bf16 by the hardware's exponential and reciprocal, for fp32 by the library's
// functions.

// GELU(z) = z Phi(z) = max(z, 0) - |z| Q(|z|) with Q = 1 - Phi: nothing cancels on
// either side.  For bf16 Abramowitz and Stegun 7.1.26 gives Q as P(t) e^(-z^2 / 2) / 2, t =
// 1 / (1 + p |z| / sqrt 2), to 7.5e-8, which takes three operations less than by way of
// erf: 5e-5 of the value at z = -3, and more than bf16's half step only below z = -6,
// where the value is above -6e-9.  For fp32 that would be 900 units at z = -3; erfc costs
// 16 us of 100 at 8192 x 5632, and its gradient 34 of 115.
template <typename T>
__device__ __forceinline__ float gelu_q(float z) {
  float q;
  if constexpr (sizeof(T) == 4) {
    q = 0.5f * erfcf(fabsf(z) * 0.70710678118654752f);
  } else {
    const float t = __builtin_amdgcn_rcpf(fmaf(fabsf(z), 0.3275911f * 0.70710678118654752f, 1.0f));
    q = t * fmaf(t, fmaf(t, fmaf(t, fmaf(t, 0.5f * 1.061405429f, 0.5f * -1.453152027f),
                                 0.5f * 1.421413741f),
                         0.5f * -0.284496736f),
                 0.5f * 0.254829592f);
    q *= __expf(-0.5f * z * z);
  }
  // a finite |z|: 0 for -inf, inf for inf; q carries a NaN
  return fmaf(-fminf(fabsf(z), 1e38f), q, fmaxf(z, 0.0f));
}
// GELU'(z) = Phi(z) + z phi(z)
template <typename T>
__device__ __forceinline__ float gelu_qd(float z) {
  if constexpr (sizeof(T) == 4) {
    const float q = 0.5f * erfcf(fabsf(z) * 0.70710678118654752f);
    return fmaf(z * 0.39894228040143268f, expf(-0.5f * z * z), z > 0.f ? 1.0f - q : q);
  }
  return gelu_d(z);
}

// SiLU(z) = z s with s = 1 / (1 + e^-z), and SiLU'(z) = s (1 + z (1 - s))
template <typename T>
__device__ __forceinline__ float silu_q(float z) {
  if constexpr (sizeof(T) == 4) return z / (1.0f + expf(-z));
  return silu_f(z);
}
template <typename T>
__device__ __forceinline__ float silu_qd(float z) {
  if constexpr (sizeof(T) == 4) {
    const float e = expf(-z), s = 1.0f / (1.0f + e);
    return s * fmaf(z, z > 0.f ? e * s : 1.0f - s, 1.0f);
  }
  return dsilu_f(z);
}

// act(z) and act'(z), `act` a pulse_act
template <int ACT, typename T>
__device__ __forceinline__ float act_f(float z) {
  if constexpr (ACT == PULSE_ACT_GELU) return gelu_q<T>(z);
  if constexpr (ACT == PULSE_ACT_SILU) return silu_q<T>(z);
  return z;
}
template <int ACT, typename T>
__device__ __forceinline__ float act_d(float z) {
  static_assert(ACT == PULSE_ACT_GELU || ACT == PULSE_ACT_SILU, "there is an act");
  if constexpr (ACT == PULSE_ACT_GELU) return gelu_qd<T>(z);
  return silu_qd<T>(z);
}

}  // namespace pulse
