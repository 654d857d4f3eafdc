// Rotary positions with several axes (gfx950): the pair (x0, x1) of pair p of
// token t turns by pos[t][axis(p)] * freq[p].  A block forms the cosines and
// sines of its tokens once, in LDS, and turns all their heads with them.
// Bound by memory: x is read and y written once.  15795 tokens of 16 heads of
// 64 in fp32, forward and backward: 56 us, 95 % of a copy's rate; 8192 tokens
// of 32 heads of 88 in bf16: 45 us, 85 %; 512 tokens of 24 heads of 64, forward:
// 3.5 us in the kernel, a chain of load, angle, sine and store.
#include "common.hpp"
#include "okernels.hpp"

namespace pulse {
namespace {

// Tokens per block: few heads want several, short calls want many blocks.  The
// short call, the bf16 one and the fp32 one, in a graph: 3.8, 34.1, 46.8 us
// with 1, 3.9, 32.5, 46.5 with 2, 4.0, 32.7, 47.1 with 4, 5.1, 34.0, 53.0
// with 8.
constexpr int RT = 2;
constexpr int MAXP = 128;  // pairs per head

struct RopeGeo {
  int tokens, heads, hd, R, axes;
  int end[4];  // first pair after each axis
  long xt, xh, yt, yh;
};

__device__ __forceinline__ void ldv(const uint16_t* p, float (&v)[4]) {
  const uint2 q = *reinterpret_cast<const uint2*>(p);
  v[0] = __uint_as_float(q.x << 16);
  v[1] = __uint_as_float(q.x & 0xffff0000u);
  v[2] = __uint_as_float(q.y << 16);
  v[3] = __uint_as_float(q.y & 0xffff0000u);
}
__device__ __forceinline__ void ldv(const float* p, float (&v)[4]) {
  const float4 q = *reinterpret_cast<const float4*>(p);
  v[0] = q.x, v[1] = q.y, v[2] = q.z, v[3] = q.w;
}
__device__ __forceinline__ void stv(uint16_t* p, const float (&v)[4]) {
  *reinterpret_cast<uint2*>(p) = uint2{pack2(v[0], v[1]), pack2(v[2], v[3])};
}
__device__ __forceinline__ void stv(float* p, const float (&v)[4]) {
  *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
}

// A unit is 8 channels: 4 + 4 of the two halves (HALVES), 8 in a row
// (adjacent pairs), or 8 in a row that are copied (beyond R).
template <typename T, bool HALVES>
__global__ __launch_bounds__(256) void k_rope(RopeGeo a, const T* x, const float* pos,
                                              const float* freq, T* y, float sign) {
  __shared__ float2 cs[RT][MAXP];
  const int t0 = blockIdx.x * RT, nt = min(RT, a.tokens - t0);
  const int np = a.R >> 1;
  for (int e = threadIdx.x; e < nt * np; e += 256) {
    const int t = e / np, p = e - t * np;
    int ax = 0;
    while (ax < a.axes - 1 && p >= a.end[ax]) ++ax;
    // the angle in turns, exact to 64 bits however far the position is
    double r = (double)pos[(long)(t0 + t) * a.axes + ax] * (double)freq[p] *
               0.15915494309189533577;
    r -= rint(r);
    float s, c;
    sincospif(2.f * (float)r, &s, &c);
    cs[t][p] = make_float2(c, s * sign);
  }
  __syncthreads();
  const int upt = a.heads * (a.hd >> 3);  // units per token
  for (int e = threadIdx.x; e < nt * upt; e += 256) {
    const int t = e / upt, u = e - t * upt;
    const int h = u / (a.hd >> 3), k = u - h * (a.hd >> 3);
    const T* px = x + (t0 + t) * a.xt + h * a.xh;
    T* py = y + (t0 + t) * a.yt + h * a.yh;
    float v0[4], v1[4];
    if (HALVES && 8 * k < a.R) {
      const int c0 = 4 * k, c1 = c0 + np;
      ldv(px + c0, v0);
      ldv(px + c1, v1);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float2 w = cs[t][c0 + i];
        const float p0 = v0[i], p1 = v1[i];
        v0[i] = p0 * w.x - p1 * w.y;
        v1[i] = p0 * w.y + p1 * w.x;
      }
      stv(py + c0, v0);
      stv(py + c1, v1);
    } else {
      const int c0 = 8 * k;
      ldv(px + c0, v0);
      ldv(px + c0 + 4, v1);
      if (c0 < a.R) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const float2 w = cs[t][4 * k + i], z = cs[t][4 * k + 2 + i];
          const float p0 = v0[2 * i], p1 = v0[2 * i + 1], r0 = v1[2 * i], r1 = v1[2 * i + 1];
          v0[2 * i] = p0 * w.x - p1 * w.y;
          v0[2 * i + 1] = p0 * w.y + p1 * w.x;
          v1[2 * i] = r0 * z.x - r1 * z.y;
          v1[2 * i + 1] = r0 * z.y + r1 * z.x;
        }
      }
      stv(py + c0, v0);
      stv(py + c0 + 4, v1);
    }
  }
}

template <typename T>
hipError_t run(const pulse_rope_desc& d, const RopeGeo& a, bool backward, const void* x,
               const float* pos, const float* freq, void* y, hipStream_t st) {
  const dim3 grid((a.tokens + RT - 1) / RT);
  const float sign = backward ? -1.f : 1.f;
  if (d.pairs == PULSE_ROPE_HALVES)
    hipLaunchKernelGGL((k_rope<T, true>), grid, dim3(256), 0, st, a, static_cast<const T*>(x), pos,
                       freq, static_cast<T*>(y), sign);
  else
    hipLaunchKernelGGL((k_rope<T, false>), grid, dim3(256), 0, st, a, static_cast<const T*>(x),
                       pos, freq, static_cast<T*>(y), sign);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_rope(const pulse_rope_desc& d, int tokens, bool backward, const pulse_heads& x,
                       const float* pos, const float* freq, const pulse_heads& y, hipStream_t st) {
  if (tokens == 0) return hipSuccess;
  RopeGeo a{};
  a.tokens = tokens;
  a.heads = d.heads;
  a.hd = d.head_dim;
  a.axes = d.axes;
  for (int i = 0; i < d.axes; ++i) {
    a.R += d.axis_dim[i];
    a.end[i] = a.R / 2;
  }
  a.xt = x.token_stride, a.xh = x.head_stride;
  a.yt = y.token_stride, a.yh = y.head_stride;
  return d.dtype == PULSE_BF16 ? run<uint16_t>(d, a, backward, x.ptr, pos, freq, y.ptr, st)
                               : run<float>(d, a, backward, x.ptr, pos, freq, y.ptr, st);
}

}  // namespace pulse
