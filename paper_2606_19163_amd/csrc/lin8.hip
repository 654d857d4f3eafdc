// Linear layers in 8-bit integers (gfx950): y = s_x s_w (q_x q_w^T) + bias.
// Both operands are laid out as the matrix instructions take them: a fragment
// is 16 rows of 64 values, 1 KB, lane l's 16 bytes being row l % 16, values 16
// (l / 16) to + 15.  A tile in LDS is a list of fragments, which LDS-DMA copies
// as they are and which reads without bank conflicts.
//
// 8192 x 1408 x 5632: laying out x 11 us (35 MB, bound by memory), the product 84
// (1.55 POP/s) and with GELU 103, traced (the least 76 and 92; a pass in a loop of such
// takes 88 and 102 in all); K of 5632 at 2.1 POP/s, where torch's int8 product reaches
// 2.4 at 16384^3.  Bound by the LDS-DMA, 48 KB per 2 x 128 x 256 x 64 and
// CU, and the outputs' vector work (two dozen instructions each with GELU), which two
// blocks per CU overlap.  Tried: 256 x 256 tiles of eight waves (117 us instead of
// 107 in all then), fragments read a step ahead behind the MFMAs (even), and in
// flight unknown to the compiler (even, and no compiler promises their registers).  1 x 1408
// x 8448: 4.2 us, 12 MB of weights at 2.8 TB/s, a launch's length.
#include "ldscopy.hpp"
#include "rowvec.hpp"

namespace pulse {
namespace {

typedef int i32x4_t __attribute__((ext_vector_type(4)));

constexpr int FRAG = 1024;
constexpr int ROWS = 256;  // rows of both operands are padded to whole tiles

__host__ __device__ inline long pad_to(long v, long m) { return (v + m - 1) / m * m; }
// fragments along K: steps of the kernels take one or two, so there are whole
// pairs
__host__ __device__ inline int k_frags(int K) { return (int)(pad_to(K, 128) / 64); }

// a laid-out operand: fp32 scales of its padded rows, then [rows / 16][k / 64]
// fragments
struct Laid {
  const float* scale;
  const char* frag;
};
__host__ __device__ inline Laid laid(const void* p, int rows) {
  const char* c = static_cast<const char*>(p);
  return Laid{reinterpret_cast<const float*>(c), c + pad_to(rows, ROWS) * 4};
}
size_t laid_bytes(int rows, int K) {
  return (size_t)pad_to(rows, ROWS) * 4 + (size_t)pad_to(rows, ROWS) * k_frags(K) * 64;
}

// What a row's largest value gives: the factor of its values, and its scale.
struct Turn {
  float r, s;
};
__device__ __forceinline__ Turn turn_of(uint32_t m) {
  const float top = fmaxf(__uint_as_float(m), 0x1p-100f);
  const bool bad = m >= 0x7f800000u;
  return Turn{bad ? 0.f : 127.f / top, bad ? __uint_as_float(0x7fc00000u) : top / 127.f};
}

template <typename T>
__device__ __forceinline__ uint32_t bits_max(uint32_t m, const Vec8<T>& v) {
#pragma unroll
  for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(v.get(i)) & 0x7fffffffu);
  return m;
}
struct MaxBits {
  __device__ __forceinline__ float operator()(float a, float b) const {
    return __uint_as_float(max(__float_as_uint(a), __float_as_uint(b)));
  }
};
// over a wave's lanes; NaN is above infinity
__device__ __forceinline__ uint32_t wave_max(uint32_t m) {
  return __float_as_uint(lanes_op<64>(__uint_as_float(m), MaxBits()));
}

// eight values as bytes: the product is rounded, then its sum with 1.5 2^23,
// to a whole number, to nearest even, whose low byte is at the bottom
template <typename T>
__device__ __forceinline__ uint2 bytes8(const Vec8<T>& v, float r) {
#pragma clang fp contract(off)
  uint32_t b[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float t = r == 0.f ? 0.f : v.get(i) * r;
    b[i] = __float_as_uint(t + 12582912.f);
  }
  const auto four = [](const uint32_t* b) __attribute__((always_inline)) {
    return __builtin_amdgcn_perm(__builtin_amdgcn_perm(b[3], b[2], 0x0c0c0400u),
                                 __builtin_amdgcn_perm(b[1], b[0], 0x0c0c0400u), 0x05040100u);
  };
  return uint2{four(b), four(b + 4)};
}

// A wave per row, the 16 rows of a fragment per block, so that whole lines
// meet in one L2.  Rows of up to 512 NV values stay in registers between the
// search for the largest and the bytes.
template <typename T, int NV>
__global__ __launch_bounds__(1024) void k_rows8(int rows, int K, const T* x, long xt, float* scale,
                                                char* frag) {
  const int row = blockIdx.x * 16 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int KS = k_frags(K);
  const bool in = row < rows;
  const T* px = x + (long)row * xt;
  Vec8<T> v[NV];
  uint32_t m = 0;
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    v[j].zero();
    if (in && 8 * lane + 512 * j < K) v[j].load(px + 8 * lane + 512 * j);
  }
#pragma unroll
  for (int j = 0; j < NV; ++j) m = bits_max(m, v[j]);
  if (in)
    for (int k = 8 * lane + 512 * NV; k < K; k += 512) {
      Vec8<T> w;
      w.load(px + k);
      m = bits_max(m, w);
    }
  const Turn t = turn_of(wave_max(m));
  if (lane == 0) scale[row] = t.s;
  char* pf = frag + (long)blockIdx.x * KS * FRAG + (row & 15) * 16;
  const auto put = [&](int k, const Vec8<T>& w) __attribute__((always_inline)) {
    *reinterpret_cast<uint2*>(pf + (long)(k >> 6) * FRAG + ((k >> 4) & 3) * 256 + (k & 8)) =
        bytes8(w, t.r);
  };
#pragma unroll
  for (int j = 0; j < NV; ++j)
    if (8 * lane + 512 * j < KS * 64) put(8 * lane + 512 * j, v[j]);
  for (int k = 8 * lane + 512 * NV; k < KS * 64; k += 512) {
    Vec8<T> w;
    w.zero();
    if (in && k < K) w.load(px + k);
    put(k, w);
  }
}

// What four outputs share: their scales and biases.
struct Outs {
  float s[4], b[4];
  __device__ __forceinline__ void load(const Lin8Args& a, const float* sw, int n) {
    const float4 w = *reinterpret_cast<const float4*>(sw + n);
    s[0] = w.x, s[1] = w.y, s[2] = w.z, s[3] = w.w;
    const float4 v = a.bias ? *reinterpret_cast<const float4*>(a.bias + n)
                            : make_float4(0.f, 0.f, 0.f, 0.f);
    b[0] = v.x, b[1] = v.y, b[2] = v.z, b[3] = v.w;
  }
};
// a sum of less than 2^31 times two such scales stays within fp32's range
__device__ __forceinline__ bool plain(float s) { return s >= 0x1p-40f && s <= 0x1p40f; }
__device__ __forceinline__ bool plain(const Outs& o) {
  return plain(o.s[0]) && plain(o.s[1]) && plain(o.s[2]) && plain(o.s[3]);
}

// Four outputs of a row.  Scales that are not plain are multiplied apart from
// their powers of two, so that a product passes fp32's range only where the
// result does; the roundings, and so the bits, are the same.
template <int ACT, bool PLAIN>
__device__ __forceinline__ uint2 out4(i32x4_t acc, float sx, const Outs& o) {
#pragma clang fp contract(off)
  float v[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float z = (float)acc[i];
    if constexpr (PLAIN)
      z = z * sx * o.s[i];
    else
      z = ldexpf(z * __builtin_amdgcn_frexp_mantf(sx) * __builtin_amdgcn_frexp_mantf(o.s[i]),
                 __builtin_amdgcn_frexp_expf(sx) + __builtin_amdgcn_frexp_expf(o.s[i]));
    v[i] = act_f<ACT, uint16_t>(z + o.b[i]);
  }
  return uint2{pack2(v[0], v[1]), pack2(v[2], v[3])};
}

// Few rows: a block of 4 waves takes 16 outputs and TT x 16 rows, its waves a
// quarter of K each, the weights straight from memory; their sums meet in LDS.
// FUSED: up to 16 rows, which every block lays out for itself, in LDS, while its
// first weights are on their way: one launch, where the rows are few enough.
template <int ACT, int TT, bool FUSED>
__global__ __launch_bounds__(256) void k_lin8_few(Lin8Args a, Laid x, Laid w) {
  extern __shared__ __attribute__((aligned(16))) char rows[];  // FUSED: [tokens][pitch]
  __shared__ i32x4_t part[4][TT][64];
  __shared__ float scales[16];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int KS = k_frags(a.K);
  const int tn = blockIdx.x, tt = blockIdx.y * TT;
  const char* pw = w.frag + ((long)tn * KS + wave) * FRAG + lane * 16;
  constexpr int AHEAD = 8;
  i32x4_t fw[AHEAD];
  const auto fetch = [&](int k0) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < AHEAD; ++i)
      if (k0 + 4 * i + wave < KS)
        fw[i] = *reinterpret_cast<const i32x4_t*>(pw + (long)(k0 + 4 * i) * FRAG);
  };
  fetch(0);
  const int pitch = FUSED ? KS * 64 + 16 : 0;
  const char* px[TT];
  if constexpr (FUSED) {
    for (int t = wave; t < a.tokens; t += 4) {
      const uint16_t* src = static_cast<const uint16_t*>(a.x) + t * a.xt;
      uint32_t m = 0;
      for (int k = 8 * lane; k < a.K; k += 512) {
        Vec8<uint16_t> v;
        v.load(src + k);
        m = bits_max(m, v);
      }
      const Turn q = turn_of(wave_max(m));
      if (lane == 0) scales[t] = q.s;
      for (int k = 8 * lane; k < KS * 64; k += 512) {
        Vec8<uint16_t> v;
        v.zero();
        if (k < a.K) v.load(src + k);
        *reinterpret_cast<uint2*>(rows + t * pitch + k) = bytes8(v, q.r);
      }
    }
    __syncthreads();
    // rows past the last give sums that are not stored
    px[0] = rows + min(lane & 15, a.tokens - 1) * pitch + (lane >> 4) * 16 + wave * 64;
  } else {
#pragma unroll
    for (int i = 0; i < TT; ++i)
      px[i] = x.frag + ((long)(tt + i) * KS + wave) * FRAG + lane * 16;
  }
  i32x4_t acc[TT];
#pragma unroll
  for (int i = 0; i < TT; ++i) acc[i] = i32x4_t{0, 0, 0, 0};
  for (int k0 = 0; k0 < KS; k0 += 4 * AHEAD) {
    if (k0) fetch(k0);
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) {
      const int k = k0 + 4 * j;
      if (k + wave < KS)
#pragma unroll
        for (int i = 0; i < TT; ++i) {
          const i32x4_t fx =
              *reinterpret_cast<const i32x4_t*>(px[i] + (long)k * (FUSED ? 64 : FRAG));
          acc[i] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fw[j], fx, acc[i], 0, 0, 0);
        }
    }
  }
#pragma unroll
  for (int i = 0; i < TT; ++i) part[wave][i][lane] = acc[i];
  __syncthreads();
  for (int i = wave; i < TT; i += 4) {
    const i32x4_t s = part[0][i][lane] + part[1][i][lane] + part[2][i][lane] + part[3][i][lane];
    const long t = (tt + i) * 16 + (lane & 15);
    const int n = tn * 16 + 4 * (lane >> 4);
    if (t < a.tokens && n < a.N) {
      Outs o;
      o.load(a, w.scale, n);
      *reinterpret_cast<uint2*>(static_cast<uint16_t*>(a.y) + t * a.yt + n) =
          out4<ACT, false>(s, FUSED ? scales[t] : x.scale[t], o);
    }
  }
}

// BT rows x BN outputs per block, WT x WN per wave
template <int BT_, int BN_, int WT_, int WN_, int STAGES_, int KB_>
struct Tile {
  static constexpr int KB = KB_;  // fragments along K per step
  static constexpr int BT = BT_, BN = BN_, WT = WT_, WN = WN_, STAGES = STAGES_;
  static constexpr int WAVES_T = BT / WT, NW = WAVES_T * (BN / WN), NT = NW * 64;
  static constexpr int TT = WT / 16, TN = WN / 16;
  static constexpr int FT = BT / 16, FN = BN / 16, STAGE = (FT + FN) * KB * FRAG;
  static constexpr int NU = (FT + FN) * KB / NW;  // fragments per wave and step
  static constexpr int LDS = STAGES * STAGE;
  // outputs on their way out: WT rows of each wave, which start 16 bytes apart
  // modulo the banks
  static constexpr int PY = WN * 2 + 16, OUT = WT * PY, CPR = WN / 8;
  static_assert(NU * NW == (FT + FN) * KB && (KB == 1 || KB == 2), "loads");
  static_assert(NW * OUT <= LDS, "outputs");
  static_assert(LDS <= 160 * 1024 && (STAGES - 2) * NU < 64, "LDS, vmcnt");
};

template <class C, int ACT>
__global__ __launch_bounds__(C::NT, 2) void k_lin8(Lin8Args a, Laid x, Laid w, int tilesN,
                                                   int GT) {
#if defined(__HIP_DEVICE_COMPILE__)
  __shared__ __attribute__((aligned(1024))) char smem[C::LDS];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wt = wave % C::WAVES_T, wn = wave / C::WAVES_T;
  // a contiguous range of tiles per XCD, groups of GT row tiles swept column by
  // column: what runs together on an XCD shares its rows and its weights in L2
  const int lb = xcd_order(blockIdx.x, gridDim.x), tilesT = gridDim.x / tilesN;
  const int group = lb / (GT * tilesN), at = lb - group * GT * tilesN;
  const int gt = min(GT, tilesT - group * GT);
  const int tn = at / gt, tt = group * GT + at - tn * gt;
  const int KS = k_frags(a.K), KT = KS / C::KB;
  // fragment f of a stage: part f % KB along K of rows f / KB.  Rows are padded
  // to whole tiles: every fragment of a tile exists.
  const char* src[C::NU];
#pragma unroll
  for (int u = 0; u < C::NU; ++u) {
    const int f = u * C::NW + wave, r = f / C::KB;
    src[u] = (r < C::FT ? x.frag + ((long)tt * C::FT + r) * KS * FRAG
                        : w.frag + ((long)tn * C::FN + r - C::FT) * KS * FRAG) +
             f % C::KB * FRAG + lane * 16;
  }
  const uint32_t sbase = lds_at(smem);
  auto issue = [&](int kt, int stage) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < C::NU; ++u)
      lds_copy16(src[u] + (long)kt * C::KB * FRAG,
                 sbase + stage * C::STAGE + (u * C::NW + wave) * FRAG);
  };
  i32x4_t acc[C::TN][C::TT];
#pragma unroll
  for (int j = 0; j < C::TN; ++j)
#pragma unroll
    for (int i = 0; i < C::TT; ++i) acc[j][i] = i32x4_t{0, 0, 0, 0};
  i32x4_t fx[C::KB][C::TT], fw[C::KB][C::TN];
  auto read = [&](int stage, int P) __attribute__((always_inline)) {
    const char* sb = smem + stage * C::STAGE + P * FRAG + lane * 16;
#pragma unroll
    for (int i = 0; i < C::TT; ++i)
      fx[P][i] = *reinterpret_cast<const i32x4_t*>(sb + (wt * C::TT + i) * C::KB * FRAG);
#pragma unroll
    for (int j = 0; j < C::TN; ++j)
      fw[P][j] = *reinterpret_cast<const i32x4_t*>(sb + (C::FT + wn * C::TN + j) * C::KB * FRAG);
  };
  auto mul = [&](int P) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < C::TN; ++j)
#pragma unroll
      for (int i = 0; i < C::TT; ++i)
        acc[j][i] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fw[P][j], fx[P][i], acc[j][i], 0, 0, 0);
  };
#pragma unroll
  for (int i = 0; i < C::STAGES - 1; ++i)
    if (i < KT) issue(i, i);
  int stage = 0;
  for (int kt = 0; kt < KT; ++kt) {
    // this step's fragments are there: at most the later stages' copies are not
    if (kt + C::STAGES - 2 < KT)
      lds_meet<(C::STAGES - 2) * C::NU>();
    else
      lds_meet<0>();
    if (kt + C::STAGES - 1 < KT)
      issue(kt + C::STAGES - 1, stage == 0 ? C::STAGES - 1 : stage - 1);
#pragma unroll
    for (int P = 0; P < C::KB; ++P) read(stage, P);
    // all reads are on their way before the first product: taken in turn by the
    // compiler, 8192 x 5632 x 1408 takes 113 us instead of 109
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int P = 0; P < C::KB; ++P) mul(P);
    stage = stage + 1 == C::STAGES ? 0 : stage + 1;
  }
  // lane: outputs 4 (lane / 16) .. + 3 of row lane % 16 of each 16 x 16.  They
  // go through LDS, so that whole rows of a wave's outputs leave together: 8
  // bytes a lane straight to memory took 90 us more at 8192 x 1408 x 5632.
  __syncthreads();  // all waves are done with the stages
  char* out = smem + wave * C::OUT;
  const long t0 = (long)tt * C::BT + wt * C::WT;
  const int n0 = tn * C::BN + wn * C::WN;
  float sx[C::TT];
  bool ok = true;
#pragma unroll
  for (int i = 0; i < C::TT; ++i) {
    sx[i] = x.scale[t0 + i * 16 + (lane & 15)];
    ok = ok && (plain(sx[i]) || t0 + i * 16 + (lane & 15) >= a.tokens);
  }
  ok = __all(ok);
#pragma unroll
  for (int j = 0; j < C::TN; ++j) {
    const int n = j * 16 + 4 * (lane >> 4);
    if (n0 + n >= a.N) continue;
    Outs o;
    o.load(a, w.scale, n0 + n);
    const auto put = [&](auto tag) __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < C::TT; ++i)
        *reinterpret_cast<uint2*>(out + (i * 16 + (lane & 15)) * C::PY + n * 2) =
            out4<ACT, decltype(tag)::value>(acc[j][i], sx[i], o);
    };
    if (ok && __all(plain(o)))
      put(std::true_type());
    else
      put(std::false_type());
  }
  // a wave reads what it wrote itself
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll 4
  for (int e = lane; e < C::WT * C::CPR; e += 64) {
    const int r = e / C::CPR, c = e % C::CPR;
    if (t0 + r < a.tokens && n0 + 8 * c < a.N)
      *reinterpret_cast<uint4*>(static_cast<uint16_t*>(a.y) + (t0 + r) * a.yt + n0 + 8 * c) =
          *reinterpret_cast<const uint4*>(out + r * C::PY + 16 * c);
  }
#endif
}

template <class C, int ACT>
hipError_t tiles(const Lin8Args& a, Laid x, Laid w, hipStream_t st) {
  const int tilesN = (a.N + C::BN - 1) / C::BN, tilesT = (a.tokens + C::BT - 1) / C::BT;
  // Row by row while an XCD's L2 of 4 MB holds all weights, four rows at a time
  // past that: 8192 x 1408 x 5632 112 -> 107.5 us, 512 x 1408 x 5632 18.1 -> 15.9, K and
  // N of 5632 270 -> 265 (512 x 5632 x 1408 24 -> 25.2); 1232 x 1408 x 2816 with
  // four 16.5 instead of 16.1.
  const int group = (long)a.N * a.K > 4 << 20 ? 4 : 1;
  hipLaunchKernelGGL((k_lin8<C, ACT>), dim3(tilesN * tilesT), dim3(C::NT), 0, st, a, x, w, tilesN,
                     group);
  return hipGetLastError();
}

template <typename T>
hipError_t rows8(int rows, int K, const void* x, long xt, Laid to, hipStream_t st) {
  auto kern = K <= 512    ? k_rows8<T, 1>
              : K <= 1024 ? k_rows8<T, 2>
              : K <= 1536 ? k_rows8<T, 3>
              : K <= 2048 ? k_rows8<T, 4>
                          : k_rows8<T, 6>;
  hipLaunchKernelGGL(kern, dim3(pad_to(rows, 16) / 16), dim3(1024), 0, st, rows, K,
                     static_cast<const T*>(x), xt, const_cast<float*>(to.scale),
                     const_cast<char*>(to.frag));
  return hipGetLastError();
}

// Bytes of LDS that up to 16 rows take, if every block is to lay them out.
bool fused(int tokens, int K) { return tokens <= 16 && tokens * (k_frags(K) * 64 + 16) <= 32768; }

template <int ACT>
hipError_t run(const Lin8Args& a, Laid x, Laid w, hipStream_t st) {
  const int tn = (a.N + 15) / 16;
  if (fused(a.tokens, a.K)) {
    hipLaunchKernelGGL((k_lin8_few<ACT, 1, true>), dim3(tn, 1), dim3(256),
                       a.tokens * (k_frags(a.K) * 64 + 16), st, a, x, w);
    return hipGetLastError();
  }
  const hipError_t e = rows8<uint16_t>(a.tokens, a.K, a.x, a.xt, x, st);
  if (e != hipSuccess) return e;
  if (a.tokens <= 64) {
    if (a.tokens <= 16)
      hipLaunchKernelGGL((k_lin8_few<ACT, 1, false>), dim3(tn, 1), dim3(256), 0, st, a, x, w);
    else
      hipLaunchKernelGGL((k_lin8_few<ACT, 2, false>), dim3(tn, (a.tokens + 31) / 32), dim3(256), 0,
                         st, a, x, w);
    return hipGetLastError();
  }
  const auto count = [&](int bt, int bn) {
    return (long)((a.tokens + bt - 1) / bt) * ((a.N + bn - 1) / bn);
  };
  if (count(128, 256) >= 256) return tiles<Tile<128, 256, 64, 128, 3, 1>, ACT>(a, x, w, st);
  // 64 x 64 while all of them run at once, three on a CU: 512 x 5632 x 1408 24 us
  // against 33 with 64 x 128, 512 x 1408 x 5632 18.0 against 19.7; past that 64 x
  // 128: 1232 x 1408 x 2816 16 against 19.6.  Two fragments along K per step: one
  // takes 28 us instead of 24 for K of 5632, the same for K of 768 and 1408.
  // Eight stages where one tile is on a CU: even (128 x 5632 x 1408 24.4 and 24.8).
  return count(64, 64) <= 768 ? tiles<Tile<64, 64, 32, 32, 3, 2>, ACT>(a, x, w, st)
                              : tiles<Tile<64, 128, 32, 64, 3, 2>, ACT>(a, x, w, st);
}

}  // namespace

size_t lin8_weight_bytes(int K, int N) { return laid_bytes(N, K); }
size_t lin8_ws_bytes(int tokens, int K, int) { return fused(tokens, K) ? 0 : laid_bytes(tokens, K); }

hipError_t launch_lin8_pack(int K, int N, const void* w, int w_dtype, void* weights,
                            hipStream_t st) {
  const Laid to = laid(weights, N);
  return w_dtype == PULSE_BF16 ? rows8<uint16_t>(N, K, w, K, to, st)
                               : rows8<float>(N, K, w, K, to, st);
}

hipError_t launch_lin8(const Lin8Args& a, hipStream_t st) {
  if (a.tokens == 0) return hipSuccess;
  const Laid x = laid(a.ws, a.tokens), w = laid(a.weights, a.N);
  switch (a.act) {
    case PULSE_ACT_GELU: return run<PULSE_ACT_GELU>(a, x, w, st);
    case PULSE_ACT_SILU: return run<PULSE_ACT_SILU>(a, x, w, st);
    default: return run<PULSE_ACT_NONE>(a, x, w, st);
  }
}

}  // namespace pulse
