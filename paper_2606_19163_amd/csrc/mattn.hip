// Attention under a row mask (gfx950, bf16 MFMA 16x16x32, fp32
// accumulation).  Query row i attends keys lo_i <= j < hi_i:
//   z = scale q k^T, capped: z = cap tanh(z / cap), then - slope |pos_i - j|
//   p = softmax over the attended keys, o = p v, lse = log sum exp z
// backward: p from z and lse; D = rowsum(do o), dp = do v^T,
//   ds = p (dp - D) (1 - tanh^2) scale, dq = ds k, dk = ds^T q, dv = p^T do.
// dq has a kernel per query tile, dk and dv one per key tile, each of which
// computes z again, so that nothing is accumulated across blocks.
// Scores are kept in the log2 domain (z log2 e).
//
// A key that a row does not attend must not reach it even when it holds a NaN
// or an infinity, which the products' zero weights do not ensure (0 NaN =
// NaN).  In a tile that some row attends only in part, an operand fragment
// that holds such a value is multiplied row by row, with the positions that
// the row does not attend cleared.
#include "common.hpp"
#include "okernels.hpp"

namespace pulse {
namespace {

typedef __attribute__((__vector_size__(8 * sizeof(__bf16)))) __bf16 bf16x8;
typedef __attribute__((__vector_size__(4 * sizeof(float)))) float f32x4;
typedef short v4s __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) v4s lds_v4s;

constexpr int BT = 64;  // rows and keys per tile
constexpr float LOG2E = 1.44269504088896341f;
constexpr float LN2 = 0.693147180559945309f;
constexpr float LOWEST = -3.0e38f;  // finite: below every finite score

struct Dev {  // device view of MattnArgs
  int Tq, Tk, H, rep, hd8;
  float c1, c2;  // no cap: scale log2e; cap: scale / cap and cap log2e
  float scale;
  const uint16_t *q, *k, *v, *dout, *o_in;
  uint16_t *o, *dq, *dk, *dv;
  long qt, qh, kt, kh, vt, vh, ot, oh, dot, doh, dqt, dqh, dkt, dkh, dvt, dvh;
  const pulse_mask_row* rows;
  const MaskTile* tiles;
  const float* slopes;
  float* lse;
  float* dsum;
};

__device__ __forceinline__ f32x4 mma(bf16x8 a, bf16x8 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ float ex2(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ f32x4 zero4() { return f32x4{0.f, 0.f, 0.f, 0.f}; }

// element offset of 16-byte chunk c of row r of a [rows][D] tile; the chunks
// of a row are permuted so that 16 rows of one chunk fall on distinct banks
template <int D>
__device__ __forceinline__ int toff(int r, int c) {
  const int x = D == 64 ? ((((r >> 1) & 1) << 1) | ((r >> 2) & 1) | (((r >> 3) & 1) << 2))
              : D == 96 ? ((r >> 2) & 3)
                        : (r & 15);
  return r * D + ((c ^ x) << 3);
}

// rows [0, BT) of a strided tensor into a tile; rows past `valid` and channels
// past the head dimension become 0
template <int D>
__device__ __forceinline__ void load_tile(uint16_t* t, const uint16_t* src, long stride, int valid,
                                          int hd8) {
  for (int e = threadIdx.x; e < BT * D / 8; e += 256) {
    const int r = e / (D / 8), c = e % (D / 8);
    uint4 v{0, 0, 0, 0};
    if (r < valid && c < hd8) v = *reinterpret_cast<const uint4*>(src + r * stride + c * 8);
    *reinterpret_cast<uint4*>(t + toff<D>(r, c)) = v;
  }
}

// operand of 8 consecutive channels straight from memory (0 where absent)
__device__ __forceinline__ bf16x8 row_frag(const uint16_t* p, int c, bool ok, int hd8) {
  uint4 v{0, 0, 0, 0};
  if (ok && c < hd8) v = *reinterpret_cast<const uint4*>(p + c * 8);
  return __builtin_bit_cast(bf16x8, v);
}

template <int D>
__device__ __forceinline__ bf16x8 frag_row(const uint16_t* t, int r, int kk, int g) {
  return *reinterpret_cast<const bf16x8*>(t + toff<D>(r, 4 * kk + g));
}

__device__ __forceinline__ v4s rd_tr(const uint16_t* p) {
  return __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s*)(p));
}

// operand whose k index runs down the tile: lane (g, j) receives rows
// r0 + 8 g .. + 7 of channel d0 + j
template <int D>
__device__ __forceinline__ bf16x8 frag_tr(const uint16_t* t, int r0, int d0, int lane) {
  const int g = lane >> 4, j = lane & 15;
  const int col = d0 + 4 * (j & 3);
  const int r = r0 + 8 * g + (j >> 2);
  const v4s lo = rd_tr(t + toff<D>(r, col >> 3) + (col & 7));
  const v4s hi = rd_tr(t + toff<D>(r + 4, col >> 3) + (col & 7));
  return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
}

// a wave's strip of 16 rows x 64 columns
__device__ __forceinline__ int soff(int r, int c) { return r * BT + ((c ^ (r & 7)) << 3); }
__device__ __forceinline__ void sput(uint16_t* s, int r, int col, float v) {
  s[soff(r, col >> 3) + (col & 7)] = f2bf(v);
}
__device__ __forceinline__ bf16x8 sfrag(const uint16_t* s, int m, int ks, int g) {
  return *reinterpret_cast<const bf16x8*>(s + soff(m, 4 * ks + g));
}

// any NaN or infinity among the wave's fragment
__device__ __forceinline__ bool nonfinite(bf16x8 v) {
  const uint4 w = __builtin_bit_cast(uint4, v);
  const uint32_t x[4] = {w.x, w.y, w.z, w.w};
  bool bad = false;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    bad |= ((x[i] & 0x7f80u) == 0x7f80u) | ((x[i] & 0x7f800000u) == 0x7f800000u);
  return __any(bad);
}

// c += a b where row r of a has zero weights at the positions k it does not
// attend and b holds a NaN or infinity: row r's product is formed with those
// positions of b cleared.  keep(r, k) says whether row r attends position k
// (0..31); rows and k as in the operands.
template <typename F>
__device__ __forceinline__ f32x4 mma_rows(bf16x8 a, bf16x8 b, f32x4 c, int lane, F keep) {
  const int g = lane >> 4;
  for (int r = 0; r < 16; ++r) {
    bf16x8 z = b;
#pragma unroll
    for (int t = 0; t < 8; ++t)
      if (!keep(r, 8 * g + t)) z[t] = (__bf16)0.f;
    const f32x4 y = mma(a, z, zero4());
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (4 * g + i == r) c[i] += y[i];
  }
  return c;
}

// log2-domain score and d z / d (scale q.k) of a raw product
template <bool CAP>
__device__ __forceinline__ float score(const Dev& a, float raw, float& slope) {
  if (!CAP) {
    slope = 1.f;
    return raw * a.c1;
  }
  // tanh(x) = 1 - 2 / (1 + e^(2x)); e^(2x) may overflow to inf: tanh = 1
  const float e = ex2(raw * a.c1 * (2.f * LOG2E));
  const float t = 1.f - 2.f * __builtin_amdgcn_rcpf(1.f + e);
  slope = 1.f - t * t;
  return t * a.c2;
}

__device__ __forceinline__ float dist(int pos, int j) { return fabsf((float)(pos - j)); }

struct Row {
  int lo, hi, pos;
};
__device__ __forceinline__ Row row_at(const Dev& a, int i) {
  if (i >= a.Tq) return Row{0, 0, 0};
  const pulse_mask_row r = a.rows[i];
  return Row{r.lo, r.hi, r.pos};
}

// ---------------------------------------------------------------------------
// forward: block (64-row tile, head), wave w rows 16 w .. + 15
// ---------------------------------------------------------------------------
template <int D, bool CAP>
__global__ __launch_bounds__(256) void k_mattn_fwd(Dev a) {
  __shared__ __attribute__((aligned(16))) uint16_t Ks[BT * D];
  __shared__ __attribute__((aligned(16))) uint16_t Vs[BT * D];
  __shared__ __attribute__((aligned(16))) uint16_t Ps[4][16 * BT];
  const int qt = blockIdx.x, h = blockIdx.y, kh = h / a.rep;
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, m = lane & 15, g = lane >> 4;
  const int q0 = qt * BT + 16 * w;
  const MaskTile mt = a.tiles[qt];
  const float sl = a.slopes ? a.slopes[h] * LOG2E : 0.f;
  bf16x8 qa[D / 32];
#pragma unroll
  for (int kk = 0; kk < D / 32; ++kk)
    qa[kk] = row_frag(a.q + (long)(q0 + m) * a.qt + h * a.qh, 4 * kk + g, q0 + m < a.Tq, a.hd8);
  Row rw[4];
  float mx[4], l[4];
  f32x4 acc[D / 16];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    rw[i] = row_at(a, q0 + 4 * g + i);
    mx[i] = LOWEST;
    l[i] = 0.f;
  }
#pragma unroll
  for (int jd = 0; jd < D / 16; ++jd) acc[jd] = zero4();
  for (int k0 = mt.lo; k0 < mt.hi; k0 += BT) {
    __syncthreads();
    load_tile<D>(Ks, a.k + (long)k0 * a.kt + kh * a.kh, a.kt, a.Tk - k0, a.hd8);
    load_tile<D>(Vs, a.v + (long)k0 * a.vt + kh * a.vh, a.vt, a.Tk - k0, a.hd8);
    __syncthreads();
    const bool part = mt.all_lo > k0 || mt.all_hi < k0 + BT;
    f32x4 s[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      s[j] = zero4();
#pragma unroll
      for (int kk = 0; kk < D / 32; ++kk)
        s[j] = mma(qa[kk], frag_row<D>(Ks, 16 * j + m, kk, g), s[j]);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float v = -INFINITY;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int key = k0 + 16 * j + m;
        float dz;
        float z = score<CAP>(a, s[j][i], dz) - sl * dist(rw[i].pos, key);
        if (key < rw[i].lo || key >= rw[i].hi) z = -INFINITY;
        s[j][i] = z;
        v = fmaxf(v, z);
      }
#pragma unroll
      for (int x = 1; x < 16; x <<= 1) v = fmaxf(v, __shfl_xor(v, x, 64));
      const float nm = fmaxf(mx[i], v);
      const float al = ex2(mx[i] - nm);
      mx[i] = nm;
      l[i] *= al;
#pragma unroll
      for (int jd = 0; jd < D / 16; ++jd) acc[jd][i] *= al;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float p = ex2(s[j][i] - nm);
        l[i] += p;
        sput(Ps[w], 4 * g + i, 16 * j + m, p);
      }
    }
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
      const bf16x8 p = sfrag(Ps[w], m, ks, g);
#pragma unroll
      for (int jd = 0; jd < D / 16; ++jd) {
        const bf16x8 v = frag_tr<D>(Vs, 32 * ks, 16 * jd, lane);
        if (part && nonfinite(v))
          acc[jd] = mma_rows(p, v, acc[jd], lane, [&](int r, int k) {
            const Row x = row_at(a, q0 + r);
            const int key = k0 + 32 * ks + k;
            return key >= x.lo && key < x.hi;
          });
        else
          acc[jd] = mma(p, v, acc[jd]);
      }
    }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
#pragma unroll
    for (int x = 1; x < 16; x <<= 1) l[i] += __shfl_xor(l[i], x, 64);
    const int r = q0 + 4 * g + i;
    if (r >= a.Tq) continue;
    const bool empty = rw[i].hi <= rw[i].lo;
    const float f = empty ? 0.f : 1.f / l[i];
    if (m == 0) a.lse[(long)h * a.Tq + r] = empty ? -INFINITY : (mx[i] + log2f(l[i])) * LN2;
#pragma unroll
    for (int jd = 0; jd < D / 16; ++jd)
      if (2 * jd + (m >> 3) < a.hd8)
        a.o[(long)r * a.ot + h * a.oh + 16 * jd + m] = f2bf(empty ? 0.f : acc[jd][i] * f);
  }
}

// ---------------------------------------------------------------------------
// backward, per 64-row tile: D = rowsum(do o), dq = ds k
// ---------------------------------------------------------------------------
template <int D, bool CAP>
__global__ __launch_bounds__(256) void k_mattn_bwd_q(Dev a) {
  __shared__ __attribute__((aligned(16))) uint16_t Ks[BT * D];
  __shared__ __attribute__((aligned(16))) uint16_t Vs[BT * D];
  __shared__ __attribute__((aligned(16))) uint16_t Ss[4][16 * BT];
  const int qt = blockIdx.x, h = blockIdx.y, kh = h / a.rep;
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, m = lane & 15, g = lane >> 4;
  const int q0 = qt * BT + 16 * w;
  const MaskTile mt = a.tiles[qt];
  const float sl = a.slopes ? a.slopes[h] * LOG2E : 0.f;
  const bool in = q0 + m < a.Tq;
  bf16x8 qa[D / 32], da[D / 32];
  float dpart = 0.f;
#pragma unroll
  for (int kk = 0; kk < D / 32; ++kk) {
    const long r = q0 + m;
    qa[kk] = row_frag(a.q + r * a.qt + h * a.qh, 4 * kk + g, in, a.hd8);
    da[kk] = row_frag(a.dout + r * a.dot + h * a.doh, 4 * kk + g, in, a.hd8);
    const bf16x8 ov = row_frag(a.o_in + r * a.ot + h * a.oh, 4 * kk + g, in, a.hd8);
#pragma unroll
    for (int t = 0; t < 8; ++t) dpart += (float)da[kk][t] * (float)ov[t];
  }
  dpart += __shfl_xor(dpart, 16, 64);
  dpart += __shfl_xor(dpart, 32, 64);
  if (g == 0 && in) a.dsum[(long)h * a.Tq + q0 + m] = dpart;
  Row rw[4];
  float Di[4], li[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int r = q0 + 4 * g + i;
    rw[i] = row_at(a, r);
    Di[i] = __shfl(dpart, 4 * g + i, 64);
    li[i] = r < a.Tq ? a.lse[(long)h * a.Tq + r] * LOG2E : 0.f;
  }
  f32x4 acc[D / 16];
#pragma unroll
  for (int jd = 0; jd < D / 16; ++jd) acc[jd] = zero4();
  for (int k0 = mt.lo; k0 < mt.hi; k0 += BT) {
    __syncthreads();
    load_tile<D>(Ks, a.k + (long)k0 * a.kt + kh * a.kh, a.kt, a.Tk - k0, a.hd8);
    load_tile<D>(Vs, a.v + (long)k0 * a.vt + kh * a.vh, a.vt, a.Tk - k0, a.hd8);
    __syncthreads();
    const bool part = mt.all_lo > k0 || mt.all_hi < k0 + BT;
    f32x4 s[4], dp[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      s[j] = zero4();
      dp[j] = zero4();
#pragma unroll
      for (int kk = 0; kk < D / 32; ++kk) {
        s[j] = mma(qa[kk], frag_row<D>(Ks, 16 * j + m, kk, g), s[j]);
        dp[j] = mma(da[kk], frag_row<D>(Vs, 16 * j + m, kk, g), dp[j]);
      }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int key = k0 + 16 * j + m;
        float dz;
        const float z = score<CAP>(a, s[j][i], dz) - sl * dist(rw[i].pos, key);
        float ds = ex2(z - li[i]) * (dp[j][i] - Di[i]) * dz;
        if (key < rw[i].lo || key >= rw[i].hi) ds = 0.f;
        sput(Ss[w], 4 * g + i, 16 * j + m, ds);
      }
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
      const bf16x8 p = sfrag(Ss[w], m, ks, g);
#pragma unroll
      for (int jd = 0; jd < D / 16; ++jd) {
        const bf16x8 v = frag_tr<D>(Ks, 32 * ks, 16 * jd, lane);
        if (part && nonfinite(v))
          acc[jd] = mma_rows(p, v, acc[jd], lane, [&](int r, int k) {
            const Row x = row_at(a, q0 + r);
            const int key = k0 + 32 * ks + k;
            return key >= x.lo && key < x.hi;
          });
        else
          acc[jd] = mma(p, v, acc[jd]);
      }
    }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int r = q0 + 4 * g + i;
    if (r >= a.Tq) continue;
#pragma unroll
    for (int jd = 0; jd < D / 16; ++jd)
      if (2 * jd + (m >> 3) < a.hd8)
        a.dq[(long)r * a.dqt + h * a.dqh + 16 * jd + m] = f2bf(acc[jd][i] * a.scale);
  }
}

// ---------------------------------------------------------------------------
// backward, per 64-key tile and key head: wave w owns keys 16 w .. + 15; the
// query tiles of every head of the group that attend any of its keys stream by
// ---------------------------------------------------------------------------
template <int D, bool CAP>
__global__ __launch_bounds__(256) void k_mattn_bwd_kv(Dev a) {
  __shared__ __attribute__((aligned(16))) uint16_t Qs[BT * D];
  __shared__ __attribute__((aligned(16))) uint16_t Os[BT * D];
  __shared__ __attribute__((aligned(16))) uint16_t Ws[4][16 * BT];
  const int kt0 = blockIdx.x * BT, kh = blockIdx.y;
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, m = lane & 15, g = lane >> 4;
  const int k0 = kt0 + 16 * w;
  const int nqt = mask_tiles(a.Tq);
  bf16x8 ka[D / 32], va[D / 32];
#pragma unroll
  for (int kk = 0; kk < D / 32; ++kk) {
    const bool in = k0 + m < a.Tk;
    ka[kk] = row_frag(a.k + (long)(k0 + m) * a.kt + kh * a.kh, 4 * kk + g, in, a.hd8);
    va[kk] = row_frag(a.v + (long)(k0 + m) * a.vt + kh * a.vh, 4 * kk + g, in, a.hd8);
  }
  f32x4 dk[D / 16], dv[D / 16];
#pragma unroll
  for (int jd = 0; jd < D / 16; ++jd) dk[jd] = dv[jd] = zero4();
  for (int h = kh * a.rep; h < (kh + 1) * a.rep; ++h) {
    const float sl = a.slopes ? a.slopes[h] * LOG2E : 0.f;
    for (int qt = 0; qt < nqt; ++qt) {
      const MaskTile mt = a.tiles[qt];
      if (mt.lo >= kt0 + BT || mt.hi <= kt0) continue;
      const bool part = mt.all_lo > kt0 || mt.all_hi < kt0 + BT;
      const int q0 = qt * BT;
      __syncthreads();
      load_tile<D>(Qs, a.q + (long)q0 * a.qt + h * a.qh, a.qt, a.Tq - q0, a.hd8);
      load_tile<D>(Os, a.dout + (long)q0 * a.dot + h * a.doh, a.dot, a.Tq - q0, a.hd8);
      __syncthreads();
      f32x4 s[4], dp[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        s[j] = zero4();
        dp[j] = zero4();
#pragma unroll
        for (int kk = 0; kk < D / 32; ++kk) {
          s[j] = mma(ka[kk], frag_row<D>(Qs, 16 * j + m, kk, g), s[j]);
          dp[j] = mma(va[kk], frag_row<D>(Os, 16 * j + m, kk, g), dp[j]);
        }
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int q = q0 + 16 * j + m;
        const Row x = row_at(a, q);
        const float lq = q < a.Tq ? a.lse[(long)h * a.Tq + q] * LOG2E : 0.f;
        const float Dq = q < a.Tq ? a.dsum[(long)h * a.Tq + q] : 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int key = k0 + 4 * g + i;
          float dz;
          const float z = score<CAP>(a, s[j][i], dz) - sl * dist(x.pos, key);
          float p = ex2(z - lq);
          float ds = p * (dp[j][i] - Dq) * dz;
          if (key < x.lo || key >= x.hi) p = ds = 0.f;
          dp[j][i] = ds;
          sput(Ws[w], 4 * g + i, 16 * j + m, p);
        }
      }
      const auto keep = [&](int ks) {
        return [&, ks](int r, int k) {
          const Row x = row_at(a, q0 + 32 * ks + k);
          return k0 + r >= x.lo && k0 + r < x.hi;
        };
      };
#pragma unroll
      for (int ks = 0; ks < 2; ++ks) {
        const bf16x8 p = sfrag(Ws[w], m, ks, g);
#pragma unroll
        for (int jd = 0; jd < D / 16; ++jd) {
          const bf16x8 v = frag_tr<D>(Os, 32 * ks, 16 * jd, lane);
          dv[jd] = part && nonfinite(v) ? mma_rows(p, v, dv[jd], lane, keep(ks))
                                        : mma(p, v, dv[jd]);
        }
      }
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) sput(Ws[w], 4 * g + i, 16 * j + m, dp[j][i]);
#pragma unroll
      for (int ks = 0; ks < 2; ++ks) {
        const bf16x8 p = sfrag(Ws[w], m, ks, g);
#pragma unroll
        for (int jd = 0; jd < D / 16; ++jd) {
          const bf16x8 v = frag_tr<D>(Qs, 32 * ks, 16 * jd, lane);
          dk[jd] = part && nonfinite(v) ? mma_rows(p, v, dk[jd], lane, keep(ks))
                                        : mma(p, v, dk[jd]);
        }
      }
    }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int r = k0 + 4 * g + i;
    if (r >= a.Tk) continue;
#pragma unroll
    for (int jd = 0; jd < D / 16; ++jd)
      if (2 * jd + (m >> 3) < a.hd8) {
        const int c = 16 * jd + m;
        a.dk[(long)r * a.dkt + kh * a.dkh + c] = f2bf(dk[jd][i] * a.scale);
        a.dv[(long)r * a.dvt + kh * a.dvh + c] = f2bf(dv[jd][i]);
      }
  }
}

Dev view(const MattnArgs& a) {
  Dev d{};
  d.Tq = a.Tq, d.Tk = a.Tk, d.H = a.H, d.rep = a.H / a.KV, d.hd8 = a.hd / 8;
  d.scale = a.scale;
  d.c1 = a.cap > 0.f ? a.scale / a.cap : a.scale * LOG2E;
  d.c2 = a.cap * LOG2E;
  const auto in = [](const pulse_heads& x) { return static_cast<const uint16_t*>(x.ptr); };
  const auto out = [](const pulse_heads& x) { return static_cast<uint16_t*>(x.ptr); };
  d.q = in(a.q), d.k = in(a.k), d.v = in(a.v), d.dout = in(a.dout), d.o_in = in(a.o);
  d.o = out(a.o), d.dq = out(a.dq), d.dk = out(a.dk), d.dv = out(a.dv);
  d.qt = a.q.token_stride, d.qh = a.q.head_stride;
  d.kt = a.k.token_stride, d.kh = a.k.head_stride;
  d.vt = a.v.token_stride, d.vh = a.v.head_stride;
  d.ot = a.o.token_stride, d.oh = a.o.head_stride;
  d.dot = a.dout.token_stride, d.doh = a.dout.head_stride;
  d.dqt = a.dq.token_stride, d.dqh = a.dq.head_stride;
  d.dkt = a.dk.token_stride, d.dkh = a.dk.head_stride;
  d.dvt = a.dv.token_stride, d.dvh = a.dv.head_stride;
  d.rows = static_cast<const pulse_mask_row*>(a.mask);
  d.tiles = reinterpret_cast<const MaskTile*>(d.rows + a.Tq);
  d.slopes = a.slopes;
  d.lse = a.lse;
  d.dsum = static_cast<float*>(a.ws);
  return d;
}

template <int D, bool CAP>
hipError_t fwd(const Dev& d, hipStream_t st) {
  hipLaunchKernelGGL((k_mattn_fwd<D, CAP>), dim3(mask_tiles(d.Tq), d.H), dim3(256), 0, st, d);
  return hipGetLastError();
}

template <int D, bool CAP>
hipError_t bwd(const Dev& d, hipStream_t st) {
  if (d.Tq) {
    hipLaunchKernelGGL((k_mattn_bwd_q<D, CAP>), dim3(mask_tiles(d.Tq), d.H), dim3(256), 0, st, d);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (d.Tk)
    hipLaunchKernelGGL((k_mattn_bwd_kv<D, CAP>), dim3((d.Tk + BT - 1) / BT, d.H / d.rep),
                       dim3(256), 0, st, d);
  return hipGetLastError();
}

}  // namespace

size_t mattn_fwd_bytes(const pulse_attn_desc&) { return 0; }
size_t mattn_bwd_bytes(const pulse_attn_desc& d) {
  return (size_t)d.heads * d.queries * sizeof(float);
}

hipError_t launch_mattn_fwd(const MattnArgs& a, hipStream_t st) {
  if (a.Tq == 0) return hipSuccess;
  const Dev d = view(a);
  const bool cap = a.cap > 0.f;
  if (a.hd <= 64) return cap ? fwd<64, true>(d, st) : fwd<64, false>(d, st);
  if (a.hd <= 96) return cap ? fwd<96, true>(d, st) : fwd<96, false>(d, st);
  return cap ? fwd<128, true>(d, st) : fwd<128, false>(d, st);
}

hipError_t launch_mattn_bwd(const MattnArgs& a, hipStream_t st) {
  const Dev d = view(a);
  const bool cap = a.cap > 0.f;
  if (a.hd <= 64) return cap ? bwd<64, true>(d, st) : bwd<64, false>(d, st);
  if (a.hd <= 96) return cap ? bwd<96, true>(d, st) : bwd<96, false>(d, st);
  return cap ? bwd<128, true>(d, st) : bwd<128, false>(d, st);
}

}  // namespace pulse
