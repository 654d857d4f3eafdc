// The joint between two halves of a transformer block (gfx950): gate and
// residual, the norms on both sides, the documents' scales and shifts.  A row
// lies in the registers of the lanes that share it, so that every tensor is
// read and written once; bound by memory.
#include "rowvec.hpp"

namespace pulse {
namespace {

// 1 / standard deviation, and the rows' values turned to n
template <int L, int NV>
__device__ __forceinline__ float norm_row(float (&v)[NV][8], int nv, int lr, int kind, float inv_c,
                                          float eps, float* sm, int& turn) {
  float s = 0.f, q = 0.f;
  if (kind == PULSE_NORM_LAYER) {
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int i = 0; i < 8; ++i) s += v[j][i];
    row_sums<L>(s, q, sm, turn);
    const float mean = s * inv_c;
    // lanes past the row hold 0 and stay at 0
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int i = 0; i < 8; ++i) v[j][i] = lr + L * j < nv ? v[j][i] - mean : 0.f;
  }
  s = q = 0.f;
  // shares of the mean, which overflow only where it does
#pragma unroll
  for (int j = 0; j < NV; ++j)
#pragma unroll
    for (int i = 0; i < 8; ++i) s = fmaf(v[j][i] * inv_c, v[j][i], s);
  row_sums<L>(s, q, sm, turn);
  const float r = rsqrtf(s + eps);
#pragma unroll
  for (int j = 0; j < NV; ++j)
#pragma unroll
    for (int i = 0; i < 8; ++i) v[j][i] *= r;
  return r;
}

// the gradient g of n turned to that of the values: r (g - mean g - n mean(g n))
template <int L, int NV>
__device__ __forceinline__ void norm_back(float (&g)[NV][8], const float (&n)[NV][8], float r,
                                          int kind, float inv_c, float* sm, int& turn) {
  float a = 0.f, b = 0.f;
#pragma unroll
  for (int j = 0; j < NV; ++j)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      a += g[j][i];
      b = fmaf(g[j][i], n[j][i], b);
    }
  row_sums<L>(a, b, sm, turn);
  a = kind == PULSE_NORM_LAYER ? a * inv_c : 0.f;
  b *= inv_c;
#pragma unroll
  for (int j = 0; j < NV; ++j)
#pragma unroll
    for (int i = 0; i < 8; ++i) g[j][i] = r * (g[j][i] - a - n[j][i] * b);
}

// document of row t: docs or -1 for none
__device__ __forceinline__ int doc_of(const int32_t* off, int docs, int t) {
  if (!off) return 0;
  int a = 0, b = docs + 1;
  while (a < b) {
    const int m = (a + b) >> 1;
    if (off[m] <= t)
      a = m + 1;
    else
      b = m;
  }
  return a - 1;
}

template <int L, int NV, class F>
__device__ __forceinline__ void each(int nv, int lr, F f) {
#pragma unroll
  for (int j = 0; j < NV; ++j)
    if (lr + L * j < nv) f(j, 8 * (lr + L * j));
}

__device__ __forceinline__ void ldf8(float (&v)[8], const float* p) {
  Vec8<float> x;
  x.load(p);
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = x.get(i);
}

// L lanes per row, NV vectors of 8 channels per lane, `rows` rows in order
template <typename TS, typename TB, int L, int NV>
__global__ __launch_bounds__(256) void k_norm_fwd(NormArgs a, int rows) {
  __shared__ float sm[16];
  int turn = 0;
  const int lr = threadIdx.x % L, nv = a.C >> 3;
  const long t0 = ((long)blockIdx.x * (256 / L) + threadIdx.x / L) * rows;
  const float inv_c = 1.f / a.C;
  float A[NV][8], B[NV][8], G[NV][8];  // of the norm, its shift, of the branch
  int cur = -2;
  for (long t = t0; t < t0 + rows && t < a.tokens; ++t) {
    const TS* px = static_cast<const TS*>(a.x) + t * a.xt;
    Vec8<TS> x[NV];
    Vec8<TB> y[NV];
    each<L, NV>(nv, lr, [&](int j, int c) {
      x[j].load(px + c);
      if (a.branch) y[j].load(static_cast<const TB*>(a.y) + t * a.yt + c);
    });
    const int d = doc_of(a.off, a.docs, (int)t);
    const bool inside = d >= 0 && d < a.docs;
    if (d != cur && inside) {
      cur = d;
      each<L, NV>(nv, lr, [&](int j, int c) {
        float w[8], s[8], b[8], f[8], g[8], p[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = g[i] = p[i] = 1.f, s[i] = b[i] = f[i] = 0.f;
        if (a.weight) ldf8(w, a.weight + c);
        if (a.bias) ldf8(b, a.bias + c);
        if (a.scale) ldf8(s, a.scale + (long)d * a.scale_t + c);
        if (a.shift) ldf8(f, a.shift + (long)d * a.shift_t + c);
        if (a.gate) ldf8(g, a.gate + (long)d * a.gate_t + c);
        if (a.post_weight) ldf8(p, a.post_weight + c);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          A[j][i] = w[i] * (1.f + s[i]);
          B[j][i] = fmaf(b[i], 1.f + s[i], f[i]);
          G[j][i] = a.r * g[i] * p[i];
        }
      });
    }
    float h[NV][8];
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int i = 0; i < 8; ++i) h[j][i] = lr + L * j < nv ? x[j].get(i) : 0.f;
    if (a.branch) {
      if (inside) {
        float v[NV][8];
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
          for (int i = 0; i < 8; ++i) v[j][i] = lr + L * j < nv ? y[j].get(i) : 0.f;
        if (a.post) norm_row<L, NV>(v, nv, lr, a.post, inv_c, a.eps, sm, turn);
        each<L, NV>(nv, lr, [&](int j, int) {
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            h[j][i] = fmaf(G[j][i], v[j][i], h[j][i]);
            // the norm is that of the stream as it is stored
            if (sizeof(TS) == 2) h[j][i] = bf2f(f2bf(h[j][i]));
          }
        });
      }
      TS* ph = static_cast<TS*>(a.h) + t * a.ht;
      each<L, NV>(nv, lr, [&](int j, int c) { put8(ph + c, h[j]); });
    }
    if (a.pre) {
      TB* pu = static_cast<TB*>(a.u) + t * a.ut;
      if (inside) norm_row<L, NV>(h, nv, lr, a.pre, inv_c, a.eps, sm, turn);
      each<L, NV>(nv, lr, [&](int j, int c) {
#pragma unroll
        for (int i = 0; i < 8; ++i) h[j][i] = inside ? fmaf(h[j][i], A[j][i], B[j][i]) : 0.f;
        put8(pu + c, h[j]);
      });
    }
  }
}

// Block b takes rows [b R, b R + R), one document after another, and leaves
// the sums over its rows of document d, of du, du n and dH ny, in slot b + d:
// from one pair (b, d) with rows to the next one of the two grows and neither
// sinks, so that no two pairs share a slot.
template <typename TS, typename TB, int L, int NV>
__global__ __launch_bounds__(256, 2) void k_norm_bwd(NormArgs a, int R, float* part) {
  extern __shared__ float comb[];  // [256 / L][C]
  __shared__ float sm[16];
  int turn = 0;
  constexpr int GR = 256 / L;
  const int lr = threadIdx.x % L, gr = threadIdx.x / L, nv = a.C >> 3;
  const float inv_c = 1.f / a.C;
  const long end = min((long)(blockIdx.x + 1) * R, (long)a.tokens);
  for (long seg = (long)blockIdx.x * R; seg < end;) {
    const int d = doc_of(a.off, a.docs, (int)seg);
    const bool inside = d >= 0 && d < a.docs;
    long stop = end;
    if (a.off && d < a.docs) stop = max(seg + 1, min(end, (long)a.off[d + 1]));
    float A[NV][8], G[NV][8];
    float P1[NV][8], P2[NV][8], P3[NV][8];
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int i = 0; i < 8; ++i) P1[j][i] = P2[j][i] = P3[j][i] = 0.f;
    if (inside)
      each<L, NV>(nv, lr, [&](int j, int c) {
        float w[8], s[8], g[8], p[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = g[i] = p[i] = 1.f, s[i] = 0.f;
        if (a.weight) ldf8(w, a.weight + c);
        if (a.scale) ldf8(s, a.scale + (long)d * a.scale_t + c);
        if (a.gate) ldf8(g, a.gate + (long)d * a.gate_t + c);
        if (a.post_weight) ldf8(p, a.post_weight + c);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          A[j][i] = w[i] * (1.f + s[i]);
          G[j][i] = a.r * g[i] * p[i];
        }
      });
    for (long t = seg + gr; t < stop; t += GR) {
      Vec8<TS> dh[NV], h[NV];
      Vec8<TB> du[NV], y[NV];
      each<L, NV>(nv, lr, [&](int j, int c) {
        if (a.dh) dh[j].load(static_cast<const TS*>(a.dh) + t * a.dht + c);
        else dh[j].zero();
        if (inside && a.pre) {
          h[j].load(static_cast<const TS*>(a.h) + t * a.ht + c);
          du[j].load(static_cast<const TB*>(a.du) + t * a.dut + c);
        }
        if (inside && a.branch) y[j].load(static_cast<const TB*>(a.y) + t * a.yt + c);
      });
      float g[NV][8], n[NV][8];
      if (inside && a.pre) {
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const bool in = lr + L * j < nv;
            n[j][i] = in ? h[j].get(i) : 0.f;
          }
        const float r = norm_row<L, NV>(n, nv, lr, a.pre, inv_c, a.eps, sm, turn);
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const bool in = lr + L * j < nv;
            const float u = in ? du[j].get(i) : 0.f;
            P1[j][i] += u;
            P2[j][i] = fmaf(u, n[j][i], P2[j][i]);
            g[j][i] = in ? u * A[j][i] : 0.f;
          }
        norm_back<L, NV>(g, n, r, a.pre, inv_c, sm, turn);
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
          for (int i = 0; i < 8; ++i) g[j][i] = lr + L * j < nv ? g[j][i] + dh[j].get(i) : 0.f;
      } else {
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
          for (int i = 0; i < 8; ++i) g[j][i] = lr + L * j < nv ? dh[j].get(i) : 0.f;
      }
      if (a.dx) {
        TS* pd = static_cast<TS*>(a.dx) + t * a.dxt;
        each<L, NV>(nv, lr, [&](int j, int c) { put8(pd + c, g[j]); });
      }
      if (a.branch) {
        if (inside) {
          float r = 0.f;
#pragma unroll
          for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int i = 0; i < 8; ++i) n[j][i] = lr + L * j < nv ? y[j].get(i) : 0.f;
          if (a.post) r = norm_row<L, NV>(n, nv, lr, a.post, inv_c, a.eps, sm, turn);
#pragma unroll
          for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              P3[j][i] = fmaf(g[j][i], n[j][i], P3[j][i]);
              g[j][i] = lr + L * j < nv ? g[j][i] * G[j][i] : 0.f;
            }
          if (a.post) norm_back<L, NV>(g, n, r, a.post, inv_c, sm, turn);
        }
        TB* pd = static_cast<TB*>(a.dy) + t * a.dyt;
        each<L, NV>(nv, lr, [&](int j, int c) {
          if (!inside)
#pragma unroll
            for (int i = 0; i < 8; ++i) g[j][i] = 0.f;
          put8(pd + c, g[j]);
        });
      }
    }
    if (inside && part) {
      float* dst = part + ((long)blockIdx.x + d) * 3 * a.C;
      auto join = [&](float (&P)[NV][8], int k) __attribute__((always_inline)) {
        if constexpr (GR == 1) {
          each<L, NV>(nv, lr, [&](int j, int c) { put8(dst + (long)k * a.C + c, P[j]); });
        } else {
          __syncthreads();  // the last sums were read
          each<L, NV>(nv, lr, [&](int j, int c) { put8(comb + gr * a.C + c, P[j]); });
          __syncthreads();
          for (int c = 4 * threadIdx.x; c < a.C; c += 1024) {
            float4 s = *reinterpret_cast<const float4*>(comb + c);
#pragma unroll
            for (int w = 1; w < GR; ++w) {
              const float4 v = *reinterpret_cast<const float4*>(comb + w * a.C + c);
              s.x += v.x, s.y += v.y, s.z += v.z, s.w += v.w;
            }
            *reinterpret_cast<float4*>(dst + (long)k * a.C + c) = s;
          }
        }
      };
      if (a.pre) {
        join(P1, 0);
        join(P2, 1);
      }
      if (a.branch) join(P3, 2);
    }
    seg = stop;
  }
}

// Sums over a document's slots: 64 channels x 4 lanes of slots, which meet in
// a fixed order.  `docsum` [docs][3][C] receives what the weights' gradients
// sum over documents.
__global__ __launch_bounds__(256) void k_norm_docs(NormArgs a, pulse_norm_grads o, int R, int nb,
                                                   const float* part, float* docsum) {
  __shared__ float sm[3][4][64];
  const int lane = threadIdx.x & 63, k = threadIdx.x >> 6;
  const int c = blockIdx.x * 64 + lane;
  for (int d = blockIdx.y; d < a.docs; d += gridDim.y) {
    const int r0 = a.off ? max(a.off[d], 0) : 0;
    const int r1 = a.off ? min(a.off[d + 1], a.tokens) : a.tokens;
    float p[3] = {0.f, 0.f, 0.f};
    if (r1 > r0 && c < a.C)
      for (int b = r0 / R + k; b <= (r1 - 1) / R; b += 4) {
        const float* src = part + ((long)b + d) * 3 * a.C + c;
        if (a.pre) {
          p[0] += src[0];
          p[1] += src[a.C];
        }
        if (a.branch) p[2] += src[2 * a.C];
      }
#pragma unroll
    for (int i = 0; i < 3; ++i) sm[i][k][lane] = p[i];
    __syncthreads();
    if (k == 0 && c < a.C) {
#pragma unroll
      for (int i = 0; i < 3; ++i)
        p[i] = (sm[i][0][lane] + sm[i][1][lane]) + (sm[i][2][lane] + sm[i][3][lane]);
      const float w = a.weight ? a.weight[c] : 1.f, b = a.bias ? a.bias[c] : 0.f;
      const float s = 1.f + (a.scale ? a.scale[(long)d * a.scale_t + c] : 0.f);
      const float g = a.r * (a.gate ? a.gate[(long)d * a.gate_t + c] : 1.f);
      const float wp = a.post_weight ? a.post_weight[c] : 1.f;
      const long at = (long)d * a.C + c;
      if (o.dshift) o.dshift[at] = p[0];
      if (o.dscale) o.dscale[at] = w * p[1] + b * p[0];
      if (o.dgate) o.dgate[at] = a.r * wp * p[2];
      if (docsum) {
        docsum[(long)d * 3 * a.C + c] = s * p[1];
        docsum[(long)d * 3 * a.C + a.C + c] = s * p[0];
        docsum[(long)d * 3 * a.C + 2 * a.C + c] = g * p[2];
      }
    }
    __syncthreads();
  }
}

__global__ __launch_bounds__(1024) void k_norm_weights(NormArgs a, pulse_norm_grads o,
                                                       const float* docsum) {
  __shared__ float sm[3][16][64];
  const int lane = threadIdx.x & 63, k = threadIdx.x >> 6;
  const int c = blockIdx.x * 64 + lane;
  float p[3] = {0.f, 0.f, 0.f};
  if (c < a.C)
    for (int d = k; d < a.docs; d += 16) {
      const float* src = docsum + (long)d * 3 * a.C + c;
#pragma unroll
      for (int i = 0; i < 3; ++i) p[i] += src[(long)i * a.C];
    }
#pragma unroll
  for (int i = 0; i < 3; ++i) sm[i][k][lane] = p[i];
  __syncthreads();
  if (k < 3 && c < a.C) {
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) s += sm[k][i][lane];
    float* dst = k == 0 ? o.dweight : k == 1 ? o.dbias : o.dpost_weight;
    if (dst) dst[c] = s;
  }
}

// Rows per block of the backward pass: whole rounds of two blocks per CU,
// and at least one row per group of lanes.
int back_rows(int tokens, int groups) {
  int r = (tokens + 511) / 512;
  r = (r + groups - 1) / groups * groups;
  return r < groups ? groups : r;
}

int groups_of(int C) { return C <= 256 ? 16 : C <= 2048 ? 4 : 1; }

template <typename TS, typename TB, int L, int NV>
hipError_t fwd(const NormArgs& a, hipStream_t st) {
  const int rows = 1;
  const int per = 256 / L * rows;
  hipLaunchKernelGGL((k_norm_fwd<TS, TB, L, NV>), dim3((a.tokens + per - 1) / per), dim3(256), 0,
                     st, a, rows);
  return hipGetLastError();
}

template <typename TS, typename TB, int L, int NV>
hipError_t bwd(const NormArgs& a, int R, int nb, float* part, hipStream_t st) {
  constexpr int GR = 256 / L;
  const size_t shared = GR > 1 ? (size_t)GR * a.C * 4 : 0;
  hipLaunchKernelGGL((k_norm_bwd<TS, TB, L, NV>), dim3(nb), dim3(256), shared, st, a, R, part);
  return hipGetLastError();
}

// f(L, NV) for a row of C channels
template <class F>
hipError_t by_size(int C, F f) {
  const int v = C / 8;
  using std::integral_constant;
#define PULSE_ROW(L, NV) f(integral_constant<int, L>(), integral_constant<int, NV>())
  if (v <= 16) return PULSE_ROW(16, 1);
  if (v <= 32) return PULSE_ROW(16, 2);
  if (v <= 64) return PULSE_ROW(64, 1);
  if (v <= 128) return PULSE_ROW(64, 2);
  if (v <= 192) return PULSE_ROW(64, 3);
  if (v <= 256) return PULSE_ROW(64, 4);
  if (v <= 512) return PULSE_ROW(256, 2);
  return PULSE_ROW(256, 4);
#undef PULSE_ROW
}

template <class F>
hipError_t by_type(const NormArgs& a, F f) {
  if (a.dtype == PULSE_F32) return f(float(), float());
  if (a.stream_dtype == PULSE_F32) return f(float(), uint16_t());
  return f(uint16_t(), uint16_t());
}

struct BackPlan {
  int R, nb;
  size_t slots;  // floats of the slots, then of the documents' sums
  size_t floats;
};
BackPlan back_plan(int C, int docs, int tokens) {
  BackPlan p;
  p.R = back_rows(tokens, groups_of(C));
  p.nb = (tokens + p.R - 1) / p.R;
  p.slots = ((size_t)p.nb + docs) * 3 * C;
  p.floats = p.slots + (size_t)docs * 3 * C;
  return p;
}

}  // namespace

size_t norm_bwd_bytes(const pulse_norm_desc& d, int tokens) {
  return back_plan(d.channels, d.docs, tokens).floats * 4;
}

hipError_t launch_norm_fwd(const NormArgs& a, hipStream_t st) {
  if (a.tokens == 0) return hipSuccess;
  return by_type(a, [&](auto ts, auto tb) {
    return by_size(a.C, [&](auto l, auto nv) {
      return fwd<decltype(ts), decltype(tb), decltype(l)::value, decltype(nv)::value>(a, st);
    });
  });
}

hipError_t launch_norm_bwd(const NormArgs& a, const pulse_norm_grads& o, float* ws,
                           hipStream_t st) {
  const bool conds = o.dgate || o.dscale || o.dshift;
  const bool weights = o.dweight || o.dbias || o.dpost_weight;
  const BackPlan p = back_plan(a.C, a.docs, a.tokens);
  float* part = conds || weights ? ws : nullptr;
  if (a.tokens) {
    const hipError_t e = by_type(a, [&](auto ts, auto tb) {
      return by_size(a.C, [&](auto l, auto nv) {
        return bwd<decltype(ts), decltype(tb), decltype(l)::value, decltype(nv)::value>(
            a, p.R, p.nb, part, st);
      });
    });
    if (e != hipSuccess) return e;
  }
  if (!part) return hipSuccess;
  float* docsum = weights ? ws + p.slots : nullptr;
  hipLaunchKernelGGL(k_norm_docs, dim3((a.C + 63) / 64, a.docs < 32768 ? a.docs : 32768),
                     dim3(256), 0, st, a, o, p.R, p.nb, part, docsum);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || !weights) return e;
  hipLaunchKernelGGL(k_norm_weights, dim3((a.C + 63) / 64), dim3(1024), 0, st, a, o, docsum);
  return hipGetLastError();
}

}  // namespace pulse
