// Activations kept in 8 bits (gfx950): groups of 32 channels share a power of
// two.  Four lanes hold a group, 8 channels each, and find its largest value
// by two quad permutes.  A power of two keeps values exact in bf16, so that the
// products of a weight gradient are exact; it costs up to one of the eight bits.
// Bound by memory, every tensor read and written once: 8192 x 5632 with GELU 42 to
// 50 us (232 MB, 4.7 to 5.5 TB/s), read back 22 (139 MB), the gradient 45 (232 MB).
#include "keepvec.hpp"

namespace pulse {
namespace {

struct Place {
  int row, vec;
};
// vector e of a block's rows of V vectors each, M = ceil(2^32 / V); exact for
// e V < 2^32
__device__ __forceinline__ Place place(uint32_t e, uint32_t V, uint32_t M) {
  const uint32_t r = V == 1 ? e : __umulhi(e, M);
  return Place{(int)r, (int)(e - r * V)};
}

constexpr int UN = 2;  // vectors in flight per thread

// rows of a block: about this many vectors
constexpr int BLOCK_VECS = 256 * UN;

// f(row, vec) for the block's vectors; a group's four lanes go together,
// since a row has a multiple of four vectors
template <class F>
__device__ __forceinline__ void walk(int tokens, int rows, uint32_t V, uint32_t M, F f) {
  const long t0 = (long)blockIdx.x * rows;
  const int n = (int)min((long)rows, tokens - t0);
#pragma unroll UN
  for (uint32_t e = threadIdx.x; e < (uint32_t)n * V; e += 256) {
    const Place p = place(e, V, M);
    f(t0 + p.row, p.vec);
  }
}

template <typename T, int ACT, bool PUT>
__global__ __launch_bounds__(256) void k_keep_save(KeepArgs a, int rows, uint32_t V, uint32_t M,
                                                   uint8_t* q, uint8_t* e) {
  walk(a.tokens, rows, V, M, [&](long t, int k) {
    const bool in = 8 * k < a.C;
    float v[8];
    Vec8<T> x;
    x.zero();
    if (in) x.load(static_cast<const T*>(a.x) + t * a.xt + 8 * k);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = x.get(i);
    keep8(v, q + (t * V + k) * 8, e + t * keep_exp_pitch(a.C) + (k >> 2), (k & 3) == 0);
    if (PUT && in) {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = act_f<ACT, T>(v[i]);
      put8(static_cast<T*>(a.y) + t * a.yt + 8 * k, v);
    }
  });
}

template <typename T>
__global__ __launch_bounds__(256) void k_keep_load(KeepArgs a, int rows, uint32_t V, uint32_t M,
                                                   const uint8_t* q, const uint8_t* e) {
  walk(a.tokens, rows, V, M, [&](long t, int k) {
    if (8 * k >= a.C) return;
    float v[8];
    load8(v, q + (t * V + k) * 8, e[t * keep_exp_pitch(a.C) + (k >> 2)]);
    put8(static_cast<T*>(a.y) + t * a.yt + 8 * k, v);
  });
}

template <typename T, int ACT, bool PUT>
__global__ __launch_bounds__(256) void k_keep_back(KeepArgs a, int rows, uint32_t V, uint32_t M,
                                                   const uint8_t* q, const uint8_t* e, uint8_t* q2,
                                                   uint8_t* e2) {
  walk(a.tokens, rows, V, M, [&](long t, int k) {
    const bool in = 8 * k < a.C;
    float z[8], v[8];
    load8(z, q + (t * V + k) * 8, e[t * keep_exp_pitch(a.C) + (k >> 2)]);
    if (in) {
      Vec8<T> g;
      g.load(static_cast<const T*>(a.x) + t * a.xt + 8 * k);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = g.get(i) * act_d<ACT, T>(z[i]);
      put8(static_cast<T*>(a.y) + t * a.yt + 8 * k, v);
    }
    if (PUT) {
#pragma unroll
      for (int i = 0; i < 8; ++i) z[i] = in ? act_f<ACT, T>(z[i]) : 0.f;
      keep8(z, q2 + (t * V + k) * 8, e2 + t * keep_exp_pitch(a.C) + (k >> 2), (k & 3) == 0);
    }
  });
}

struct Grid {
  int rows, blocks;
  uint32_t V, M;
};
Grid grid_of(const KeepArgs& a) {
  Grid g;
  g.V = (uint32_t)(keep_pitch(a.C) / 8);
  g.M = (uint32_t)(((UINT64_C(1) << 32) + g.V - 1) / g.V);
  g.rows = g.V >= BLOCK_VECS ? 1 : BLOCK_VECS / (int)g.V;
  g.blocks = (a.tokens + g.rows - 1) / g.rows;
  return g;
}

// f(T, ACT)
template <class F>
hipError_t by_kind(const KeepArgs& a, F f) {
  using std::integral_constant;
#define PULSE_ACTS(T)                                                                             \
  (a.act == PULSE_ACT_GELU   ? f(T(), integral_constant<int, PULSE_ACT_GELU>())                    \
   : a.act == PULSE_ACT_SILU ? f(T(), integral_constant<int, PULSE_ACT_SILU>())                    \
                             : f(T(), integral_constant<int, PULSE_ACT_NONE>()))
  return a.dtype == PULSE_BF16 ? PULSE_ACTS(uint16_t) : PULSE_ACTS(float);
#undef PULSE_ACTS
}

uint8_t* exps(const KeepArgs& a, void* kept) {
  return static_cast<uint8_t*>(kept) + keep_exps_at(a.C, a.tokens);
}

}  // namespace

hipError_t launch_keep_save(const KeepArgs& a, hipStream_t st) {
  if (a.tokens == 0) return hipSuccess;
  const Grid g = grid_of(a);
  return by_kind(a, [&](auto t, auto act) {
    using T = decltype(t);
    constexpr int ACT = decltype(act)::value;
    auto kern = k_keep_save<T, PULSE_ACT_NONE, false>;
    if constexpr (ACT != PULSE_ACT_NONE)
      if (a.y) kern = k_keep_save<T, ACT, true>;
    hipLaunchKernelGGL(kern, dim3(g.blocks), dim3(256), 0, st, a, g.rows, g.V, g.M,
                       static_cast<uint8_t*>(a.kept), exps(a, a.kept));
    return hipGetLastError();
  });
}

hipError_t launch_keep_load(const KeepArgs& a, hipStream_t st) {
  if (a.tokens == 0) return hipSuccess;
  const Grid g = grid_of(a);
  auto kern = a.dtype == PULSE_BF16 ? k_keep_load<uint16_t> : k_keep_load<float>;
  hipLaunchKernelGGL(kern, dim3(g.blocks), dim3(256), 0, st, a, g.rows, g.V, g.M,
                     static_cast<const uint8_t*>(a.kept), exps(a, a.kept));
  return hipGetLastError();
}

hipError_t launch_keep_back(const KeepArgs& a, hipStream_t st) {
  if (a.tokens == 0) return hipSuccess;
  const Grid g = grid_of(a);
  return by_kind(a, [&](auto t, auto act) {
    using T = decltype(t);
    constexpr int ACT = decltype(act)::value;
    if constexpr (ACT == PULSE_ACT_NONE) {
      return hipErrorInvalidValue;
    } else {
      auto kern = a.a_kept ? k_keep_back<T, ACT, true> : k_keep_back<T, ACT, false>;
      hipLaunchKernelGGL(kern, dim3(g.blocks), dim3(256), 0, st, a, g.rows, g.V, g.M,
                         static_cast<const uint8_t*>(a.kept), exps(a, a.kept),
                         static_cast<uint8_t*>(a.a_kept), a.a_kept ? exps(a, a.a_kept) : nullptr);
      return hipGetLastError();
    }
  });
}

}  // namespace pulse
