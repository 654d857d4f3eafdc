// The joint between two halves of a transformer block (gfx950): gate and
// residual, the norms on both sides, the documents' scales and shifts.
//
// A row lies in the registers of the lanes that share it, 8 channels each, so
// that every tensor is read and written once; as many waves take a row as that
// needs, since with 24 or 32 channels a lane the sums over rows that the backward
// pass keeps beside the row spilled (83 us instead of 43 at 8192 x 1408 then).  Only
// the backward pass of an fp32 stream of more than 4096 channels does spill, 52 to 88
// bytes a lane: its 16 waves have 128 registers each (1408 x 8192 70 us, where 2816 x
// 4096 takes 47).  Bound
// by memory: 8192 x 1408 in bf16 forward 19.6 us in the kernel (92 MB, 4.7 TB/s),
// backward 32 (139 MB, 4.3) and 4.3 for the sums over blocks; 15795 x 1280 with an
// fp32 stream and a norm on both sides 80 (365 MB, 4.6) + 5.1 + 4.7; a copy of 2
// GiB reaches 4.9 TB/s.  512 x 768 forward: 4.4 us, a chain of loads, two sums
// and a store.
#include "rowvec.hpp"

namespace pulse {
namespace {

// floats of LDS that the sums over a row take
template <int L>
constexpr int ROW_LDS = L > 64 ? L / 16 : 1;

// 1 / standard deviation, and the row's values turned to n.  Lanes past the
// row (`in` false) hold 0 and stay at 0.
template <int L>
__device__ __forceinline__ float norm_row(float (&v)[8], bool in, int kind, float inv_c, float eps,
                                          float* sm, int& turn) {
  float s = 0.f, q = 0.f;
  if (kind == PULSE_NORM_LAYER) {
#pragma unroll
    for (int i = 0; i < 8; ++i) s += v[i];
    row_sums<L>(s, q, sm, turn);
    const float mean = in ? s * inv_c : 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] -= mean;
  }
  s = q = 0.f;
  // shares of the mean, which overflow only where it does
#pragma unroll
  for (int i = 0; i < 8; ++i) s = fmaf(v[i] * inv_c, v[i], s);
  row_sums<L>(s, q, sm, turn);
  const float r = rsqrtf(s + eps);
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] *= r;
  return r;
}

// the gradient g of n turned to that of the values: r (g - mean g - n mean(g n))
template <int L>
__device__ __forceinline__ void norm_back(float (&g)[8], const float (&n)[8], float r, int kind,
                                          float inv_c, float* sm, int& turn) {
  float a = 0.f, b = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    a += g[i];
    b = fmaf(g[i], n[i], b);
  }
  row_sums<L>(a, b, sm, turn);
  a = kind == PULSE_NORM_LAYER ? a * inv_c : 0.f;
  b *= inv_c;
#pragma unroll
  for (int i = 0; i < 8; ++i) g[i] = r * (g[i] - a - n[i] * b);
}

// Document of row t: docs or -1 for none.  A wave whose lanes ask for one row
// looks at 64 offsets at a time; bisection where they ask for several.
template <bool WAVE>
__device__ __forceinline__ int doc_of(const int32_t* off, int docs, int t) {
  if (!off) return 0;
  int a = 0, n = docs + 1;  // the first offset above t is in [a, a + n]
  if (WAVE) {
    const int lane = threadIdx.x & 63;
    while (n > 64) {
      const int step = (n + 63) >> 6;
      const int i = a + lane * step;
      const uint64_t m = __ballot(i < a + n && off[min(i, docs)] <= t);
      if (!m) return a - 1;
      const int first = a + (__popcll(m) - 1) * step;
      n = min(step, a + n - first);
      a = first;
    }
    return a + __popcll(__ballot(lane < n && off[min(a + lane, docs)] <= t)) - 1;
  }
  int b = n;
  while (a < b) {
    const int m = (a + b) >> 1;
    if (off[m] <= t)
      a = m + 1;
    else
      b = m;
  }
  return a - 1;
}

__device__ __forceinline__ void ldf8(float (&v)[8], const float* p) {
  Vec8<float> x;
  x.load(p);
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = x.get(i);
}

// What a document's rows share, for a lane's channels: the norm's factor A and
// shift B, the branch's factor G.
struct Cond {
  float A[8], B[8], G[8];
  __device__ __forceinline__ void load(const NormArgs& a, int d, int c) {
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
      A[i] = w[i] * (1.f + s[i]);
      B[i] = fmaf(b[i], 1.f + s[i], f[i]);
      G[i] = a.r * g[i] * p[i];
    }
  }
};

template <typename T>
__device__ __forceinline__ void get8(float (&v)[8], const Vec8<T>& x, bool in) {
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = in ? x.get(i) : 0.f;
}

// L lanes per row, 8 channels per lane; `rows` rows in order, the next one on
// its way while one is worked on
template <typename TS, typename TB, int L>
__global__ __launch_bounds__(ROW_THREADS<L>) void k_norm_fwd(NormArgs a, int rows) {
  __shared__ float sm[ROW_LDS<L>];
  int turn = 0;
  const int c = 8 * (threadIdx.x % L);
  const bool in = c < a.C;
  const float inv_c = 1.f / a.C;
  const long t0 = ((long)blockIdx.x * (ROW_THREADS<L> / L) + threadIdx.x / L) * rows;
  const long t1 = min(t0 + rows, (long)a.tokens);
  Vec8<TS> x;
  Vec8<TB> y;
  x.zero();
  y.zero();
  auto fetch = [&](long t) __attribute__((always_inline)) {
    if (in && t < t1) {
      x.load(static_cast<const TS*>(a.x) + t * a.xt + c);
      if (a.branch) y.load(static_cast<const TB*>(a.y) + t * a.yt + c);
    }
  };
  fetch(t0);
  Cond k;
  bool inside = false;
  long stop = t0;  // the first row past this document
  for (long t = t0; t < t1; ++t) {
    float h[8], v[8];
    if (t >= stop) {
      const int d = doc_of<(L >= 64)>(a.off, a.docs, (int)t);
      inside = d >= 0 && d < a.docs;
      stop = a.off && d < a.docs ? a.off[d + 1] : a.tokens;
      if (inside && in) k.load(a, d, c);
    }
    get8(h, x, in);
    get8(v, y, in);
    fetch(t + 1);
    if (a.branch) {
      if (inside) {
        if (a.post) norm_row<L>(v, in, a.post, inv_c, a.eps, sm, turn);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          h[i] = in ? fmaf(k.G[i], v[i], h[i]) : 0.f;
          // the norm is that of the stream as it is stored
          if (sizeof(TS) == 2) h[i] = bf2f(f2bf(h[i]));
        }
      }
      if (in) put8(static_cast<TS*>(a.h) + t * a.ht + c, h);
    }
    if (a.pre) {
      if (inside) norm_row<L>(h, in, a.pre, inv_c, a.eps, sm, turn);
#pragma unroll
      for (int i = 0; i < 8; ++i) h[i] = inside ? fmaf(h[i], k.A[i], k.B[i]) : 0.f;
      if (in) put8(static_cast<TB*>(a.u) + t * a.ut + c, h);
    }
  }
}

// Block b takes rows [b R, b R + R), one document after another, and leaves
// the sums over its rows of document d, of du, du n and dH ny, in slot b + d:
// from one pair (b, d) with rows to the next one of the two grows and neither
// sinks, so that no two pairs share a slot.
template <typename TS, typename TB, int L>
__global__ __launch_bounds__(ROW_THREADS<L>) void k_norm_bwd(NormArgs a, int R, float* part) {
  constexpr int GR = ROW_THREADS<L> / L;
  __shared__ float sm[ROW_LDS<L>];
  __shared__ __attribute__((aligned(16))) float comb[GR > 1 ? GR * 8 * L : 4];
  int turn = 0;
  const int gr = threadIdx.x / L, c = 8 * (threadIdx.x % L);
  const bool in = c < a.C;
  const float inv_c = 1.f / a.C;
  const long end = min((long)(blockIdx.x + 1) * R, (long)a.tokens);
  for (long seg = (long)blockIdx.x * R; seg < end;) {
    const int d = doc_of<true>(a.off, a.docs, (int)seg);
    const bool inside = d >= 0 && d < a.docs;
    long stop = end;
    if (a.off && d < a.docs) stop = max(seg + 1, min(end, (long)a.off[d + 1]));
    Vec8<TS> dh, h;
    Vec8<TB> du, y;
    dh.zero(), h.zero(), du.zero(), y.zero();
    auto fetch = [&](long t) __attribute__((always_inline)) {
      if (!in || t >= stop) return;
      if (a.dh) dh.load(static_cast<const TS*>(a.dh) + t * a.dht + c);
      if (inside && a.pre) {
        h.load(static_cast<const TS*>(a.h) + t * a.ht + c);
        du.load(static_cast<const TB*>(a.du) + t * a.dut + c);
      }
      if (inside && a.branch) y.load(static_cast<const TB*>(a.y) + t * a.yt + c);
    };
    fetch(seg + gr);
    Cond k;
    if (inside && in) k.load(a, d, c);
    float P1[8], P2[8], P3[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) P1[i] = P2[i] = P3[i] = 0.f;
    for (long t = seg + gr; t < stop; t += GR) {
      float g[8], n[8], u[8], ny[8], e[8];
      get8(e, dh, in);
      get8(n, h, in);
      get8(u, du, in);
      get8(ny, y, in);
      fetch(t + GR);
#pragma unroll
      for (int i = 0; i < 8; ++i) g[i] = 0.f;
      if (inside && a.pre) {
        const float r = norm_row<L>(n, in, a.pre, inv_c, a.eps, sm, turn);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          P1[i] += u[i];
          P2[i] = fmaf(u[i], n[i], P2[i]);
          g[i] = in ? u[i] * k.A[i] : 0.f;
        }
        norm_back<L>(g, n, r, a.pre, inv_c, sm, turn);
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) g[i] = in ? g[i] + e[i] : 0.f;
      if (a.dx && in) put8(static_cast<TS*>(a.dx) + t * a.dxt + c, g);
      if (a.branch) {
        if (inside) {
          float r = 0.f;
          if (a.post) r = norm_row<L>(ny, in, a.post, inv_c, a.eps, sm, turn);
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            P3[i] = fmaf(g[i], ny[i], P3[i]);
            g[i] = in ? g[i] * k.G[i] : 0.f;
          }
          if (a.post) norm_back<L>(g, ny, r, a.post, inv_c, sm, turn);
        } else {
#pragma unroll
          for (int i = 0; i < 8; ++i) g[i] = 0.f;
        }
        if (in) put8(static_cast<TB*>(a.dy) + t * a.dyt + c, g);
      }
    }
    if (inside && part) {
      float* dst = part + ((long)blockIdx.x + d) * 3 * a.C + c;
      auto join = [&](float (&P)[8], int w) __attribute__((always_inline)) {
        if constexpr (GR > 1) {
          __syncthreads();  // the last sums were read
          put8(comb + gr * 8 * L + c, P);
          __syncthreads();
          if (gr == 0)
#pragma unroll
            for (int i = 1; i < GR; ++i) {
              float v[8];
              ldf8(v, comb + i * 8 * L + c);
#pragma unroll
              for (int j = 0; j < 8; ++j) P[j] += v[j];
            }
        }
        if (gr == 0 && in) put8(dst + (long)w * a.C, P);
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

// A block of the sums over slots and documents: 64 channels, four each of 16
// lanes, times K lanes of what is summed, which meet in a fixed order.
constexpr int SUM_C = 64, SUM_K = 16;
template <int K>
using Sums = float[3][K][SUM_C];

// p[i] += the sums over n rows of three vectors, the first at src, the others
// `step` floats apart, for the vectors i that are there.  Four rows at a time
// are on their way: in turn, each would wait for memory.
__device__ __forceinline__ void add_rows(float4 (&p)[3], const float* src, long step, int n, int C,
                                         bool first2, bool third) {
  constexpr int AHEAD = 4;
  for (int r0 = 0; r0 < n; r0 += AHEAD) {
    float4 v[AHEAD][3];
#pragma unroll
    for (int r = 0; r < AHEAD; ++r)
#pragma unroll
      for (int i = 0; i < 3; ++i) {
        v[r][i] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (r0 + r < n && (i < 2 ? first2 : third))
          v[r][i] = *reinterpret_cast<const float4*>(src + (r0 + r) * step + (long)i * C);
      }
#pragma unroll
    for (int r = 0; r < AHEAD; ++r)
#pragma unroll
      for (int i = 0; i < 3; ++i) {
        p[i].x += v[r][i].x, p[i].y += v[r][i].y;
        p[i].z += v[r][i].z, p[i].w += v[r][i].w;
      }
  }
}

// thread t < 192: the total of sum t / 64, channel t % 64
template <int K>
__device__ __forceinline__ float meet(Sums<K>& sm, const float4 (&p)[3]) {
  const int k = threadIdx.x >> 4, c = 4 * (threadIdx.x & 15);
#pragma unroll
  for (int i = 0; i < 3; ++i) *reinterpret_cast<float4*>(&sm[i][k][c]) = p[i];
  __syncthreads();
  float s = 0.f;
  if (threadIdx.x < 3 * SUM_C)
#pragma unroll
    for (int j = 0; j < K; ++j) s += sm[threadIdx.x >> 6][j][threadIdx.x & 63];
  return s;
}

// What a document's sums p0 of du, p1 of du n and p2 of dH ny, channel c, turn
// into.  `docsum` [docs][3][C] receives what the weights' gradients sum over
// documents.
struct DocOut {
  float w, b, s, g, wp;
  __device__ __forceinline__ void load(const NormArgs& a, int d, int c) {
    w = a.weight ? a.weight[c] : 1.f, b = a.bias ? a.bias[c] : 0.f;
    s = 1.f + (a.scale ? a.scale[(long)d * a.scale_t + c] : 0.f);
    g = a.r * (a.gate ? a.gate[(long)d * a.gate_t + c] : 1.f);
    wp = a.post_weight ? a.post_weight[c] : 1.f;
  }
  // a document without rows adds nothing, whatever its conditions hold
  __device__ __forceinline__ void none() { w = b = s = g = wp = 0.f; }
  __device__ __forceinline__ void put(const NormArgs& a, const pulse_norm_grads& o, float* docsum,
                                      int d, int c, float p0, float p1, float p2) const {
    const long at = (long)d * a.C + c;
    if (o.dshift) o.dshift[at] = p0;
    if (o.dscale) o.dscale[at] = w * p1 + b * p0;
    if (o.dgate) o.dgate[at] = a.r * wp * p2;
    if (docsum) {
      docsum[(long)d * 3 * a.C + c] = s * p1;
      docsum[(long)d * 3 * a.C + a.C + c] = s * p0;
      docsum[(long)d * 3 * a.C + 2 * a.C + c] = g * p2;
    }
    if (a.docs == 1) {  // nothing to sum over documents
      if (o.dweight) o.dweight[c] = s * p1;
      if (o.dbias) o.dbias[c] = s * p0;
      if (o.dpost_weight) o.dpost_weight[c] = g * p2;
    }
  }
};

// blocks that hold rows of document d: the first, and how many
__device__ __forceinline__ int2 blocks_of(const NormArgs& a, int R, int d) {
  const int r0 = a.off ? max(a.off[d], 0) : 0;
  const int r1 = a.off ? min(a.off[d + 1], a.tokens) : a.tokens;
  return r1 > r0 ? make_int2(r0 / R, (r1 - 1) / R - r0 / R + 1) : make_int2(0, 0);
}

// Many documents of few slots: 16 documents per block, 16 lanes of four
// channels each.
__global__ __launch_bounds__(256) void k_norm_many(NormArgs a, pulse_norm_grads o, int R,
                                                   const float* part, float* docsum) {
  const int d = blockIdx.x * SUM_K + (threadIdx.x >> 4);
  const int c = blockIdx.y * SUM_C + 4 * (threadIdx.x & 15);
  if (d >= a.docs || c >= a.C) return;
  DocOut out[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) out[i].load(a, d, c + i);
  float4 p[3];
  p[0] = p[1] = p[2] = make_float4(0.f, 0.f, 0.f, 0.f);
  const int2 b = blocks_of(a, R, d);
  if (b.y == 0)
#pragma unroll
    for (int i = 0; i < 4; ++i) out[i].none();
  add_rows(p, part + ((long)b.x + d) * 3 * a.C + c, 3L * a.C, b.y, a.C, a.pre != 0,
           a.branch != 0);
  out[0].put(a, o, docsum, d, c, p[0].x, p[1].x, p[2].x);
  out[1].put(a, o, docsum, d, c + 1, p[0].y, p[1].y, p[2].y);
  out[2].put(a, o, docsum, d, c + 2, p[0].z, p[1].z, p[2].z);
  out[3].put(a, o, docsum, d, c + 3, p[0].w, p[1].w, p[2].w);
}

// Few documents of many slots: a block per document and 64 channels.
template <int K>
__global__ __launch_bounds__(16 * K) void k_norm_docs(NormArgs a, pulse_norm_grads o, int R,
                                                      const float* part, float* docsum) {
  __shared__ __attribute__((aligned(16))) Sums<K> sm;
  __shared__ float tot[3][SUM_C];
  const int k = threadIdx.x >> 4, c4 = blockIdx.x * SUM_C + 4 * (threadIdx.x & 15);
  const int d = blockIdx.y;
  float4 p[3];
  p[0] = p[1] = p[2] = make_float4(0.f, 0.f, 0.f, 0.f);
  // what the totals are turned with, on its way beside them
  const int c = blockIdx.x * SUM_C + threadIdx.x;
  const bool mine = threadIdx.x < SUM_C && c < a.C;
  DocOut out{};
  if (mine) out.load(a, d, c);
  const int2 b = blocks_of(a, R, d);
  if (b.y == 0) out.none();
  if (k < b.y && c4 < a.C)
    add_rows(p, part + ((long)b.x + k + d) * 3 * a.C + c4, (long)K * 3 * a.C,
             (b.y - k + K - 1) / K, a.C, a.pre != 0, a.branch != 0);
  const float total = meet<K>(sm, p);
  if (threadIdx.x < 3 * SUM_C) tot[threadIdx.x >> 6][threadIdx.x & 63] = total;
  __syncthreads();
  if (mine)
    out.put(a, o, docsum, d, c, tot[0][threadIdx.x], tot[1][threadIdx.x], tot[2][threadIdx.x]);
}

__global__ __launch_bounds__(256) void k_norm_weights(NormArgs a, pulse_norm_grads o,
                                                      const float* docsum) {
  __shared__ __attribute__((aligned(16))) Sums<SUM_K> sm;
  const int k = threadIdx.x >> 4, c4 = blockIdx.x * SUM_C + 4 * (threadIdx.x & 15);
  float4 p[3];
  p[0] = p[1] = p[2] = make_float4(0.f, 0.f, 0.f, 0.f);
  if (c4 < a.C && k < a.docs)
    add_rows(p, docsum + (long)k * 3 * a.C + c4, (long)SUM_K * 3 * a.C,
             (a.docs - k + SUM_K - 1) / SUM_K, a.C, true, true);
  const float total = meet<SUM_K>(sm, p);
  const int i = threadIdx.x >> 6, c = blockIdx.x * SUM_C + (threadIdx.x & 63);
  float* dst = i == 0 ? o.dweight : i == 1 ? o.dbias : i == 2 ? o.dpost_weight : nullptr;
  if (dst && c < a.C) dst[c] = total;
}

template <typename TS, typename TB, int L>
hipError_t fwd(const NormArgs& a, hipStream_t st) {
  // rows in order share the loads of their document's vectors (8192 x 1408: 27.6
  // us with one, 23.5 with two, 22.8 with four, 21.5 with six); a block per row
  // while there are few
  const int rows = a.tokens >= 8192 ? 4 : a.tokens >= 4096 ? 2 : 1;
  const int per = ROW_THREADS<L> / L * rows;
  hipLaunchKernelGGL((k_norm_fwd<TS, TB, L>), dim3((a.tokens + per - 1) / per),
                     dim3(ROW_THREADS<L>), 0, st, a, rows);
  return hipGetLastError();
}

template <typename TS, typename TB, int L>
hipError_t bwd(const NormArgs& a, int R, int nb, float* part, hipStream_t st) {
  hipLaunchKernelGGL((k_norm_bwd<TS, TB, L>), dim3(nb), dim3(ROW_THREADS<L>), 0, st, a, R, part);
  return hipGetLastError();
}

// Lanes of a row: f(L).
template <class F>
auto by_size(int C, F f) {
  using std::integral_constant;
  if (C <= 128) return f(integral_constant<int, 16>());
  if (C <= 512) return f(integral_constant<int, 64>());
  if (C <= 1024) return f(integral_constant<int, 128>());
  if (C <= 1536) return f(integral_constant<int, 192>());
  if (C <= 2048) return f(integral_constant<int, 256>());
  if (C <= 4096) return f(integral_constant<int, 512>());
  return f(integral_constant<int, 1024>());
}

template <class F>
hipError_t by_type(const NormArgs& a, F f) {
  if (a.dtype == PULSE_F32) return f(float(), float());
  if (a.stream_dtype == PULSE_F32) return f(float(), uint16_t());
  return f(uint16_t(), uint16_t());
}

// Three blocks of three waves per CU: more blocks are more partial sums to
// write and read.  8192 x 1408: 42.7 us with 512, 43.2 with 768, 43.5 with 1024, 50.8
// with 1536; 15795 x 1280: 96.0, 96.6, 109 and 105 (with slower sums over them).
constexpr int BACK_BLOCKS = 768;

struct BackPlan {
  int R, nb;
  size_t slots;  // floats of the slots, then of the documents' sums
  size_t floats;
};
BackPlan back_plan(int C, int docs, int tokens) {
  BackPlan p;
  const int groups = by_size(C, [](auto l) {
    constexpr int L = decltype(l)::value;
    return ROW_THREADS<L> / L;
  });
  // rows per block: the blocks fill the GPU, and every group of lanes has one
  p.R = (tokens + BACK_BLOCKS - 1) / BACK_BLOCKS;
  p.R = (p.R + groups - 1) / groups * groups;
  if (p.R < groups) p.R = groups;
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
    return by_size(a.C, [&](auto l) {
      return fwd<decltype(ts), decltype(tb), decltype(l)::value>(a, st);
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
      return by_size(a.C, [&](auto l) {
        return bwd<decltype(ts), decltype(tb), decltype(l)::value>(a, p.R, p.nb, part, st);
      });
    });
    if (e != hipSuccess) return e;
  }
  if (!part) return hipSuccess;
  float* docsum = weights && a.docs > 1 ? ws + p.slots : nullptr;
  const int tiles = (a.C + SUM_C - 1) / SUM_C;
  // 16 documents to a block where they have eight slots or less on average (20000
  // x 2048 of 200 documents 129 us instead of 136), 64 lanes to a document's slots
  // where they are more than 64 (8192 x 1408 of one document 44 us instead of 47.7)
  if (a.docs * 8L >= p.nb)
    hipLaunchKernelGGL(k_norm_many, dim3((a.docs + SUM_K - 1) / SUM_K, tiles), dim3(256), 0, st, a,
                       o, p.R, part, docsum);
  else if (p.nb > 64L * a.docs)
    hipLaunchKernelGGL(k_norm_docs<64>, dim3(tiles, a.docs), dim3(1024), 0, st, a, o, p.R, part,
                       docsum);
  else
    hipLaunchKernelGGL(k_norm_docs<16>, dim3(tiles, a.docs), dim3(256), 0, st, a, o, p.R, part,
                       docsum);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || !docsum) return e;
  hipLaunchKernelGGL(k_norm_weights, dim3(tiles), dim3(256), 0, st, a, o, docsum);
  return hipGetLastError();
}

}  // namespace pulse
