// Linear layers in 8-bit integers (gfx950): y = s_x s_w (q_x q_w^T) + bias.
// Both operands are laid out as the matrix instructions take them: a fragment
// is 16 rows of 64 values, 1 KB, lane l's 16 bytes being row l % 16, values 16
// (l / 16) to + 15.  A tile in LDS is a list of fragments, which LDS-DMA copies
// as they are and which reads without bank conflicts.
#include "rowvec.hpp"

namespace pulse {
namespace {

typedef int i32x4_t __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) void* lds_ptr_t;

constexpr int FRAG = 1024;
constexpr int ROWS = 256;  // rows of both operands are padded to whole tiles

__host__ __device__ inline long pad_to(long v, long m) { return (v + m - 1) / m * m; }

// A scale m 2^e, 0.5 <= m < 1: a sum times two of them passes fp32's range only
// where the result does.
struct Scale {
  float m;
  int e;
};
// a laid-out operand: the scales of its padded rows, then [rows / 16][k / 64]
// fragments
struct Laid {
  const Scale* scale;
  const char* frag;
};
__host__ __device__ inline Laid laid(const void* p, int rows) {
  const char* c = static_cast<const char*>(p);
  return Laid{reinterpret_cast<const Scale*>(c), c + pad_to(rows, ROWS) * sizeof(Scale)};
}
size_t laid_bytes(int rows, int K) {
  return (size_t)pad_to(rows, ROWS) * sizeof(Scale) + (size_t)pad_to(rows, ROWS) * pad_to(K, 64);
}

// One wave per row: its largest value, then its bytes.  Rows of zeros fill the
// last 16.
template <typename T>
__global__ __launch_bounds__(256) void k_rows8(int rows, int K, const T* x, long xt, Scale* scale,
                                               char* frag) {
#pragma clang fp contract(off)
  const int row = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (row >= (int)pad_to(rows, 16)) return;
  const int KS = (int)pad_to(K, 64) / 64;
  const T* px = x + (long)row * xt;
  uint32_t m = 0;
  if (row < rows)
    for (int k = 8 * lane; k < K; k += 512) {
      Vec8<T> v;
      v.load(px + k);
#pragma unroll
      for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(v.get(i)) & 0x7fffffffu);
    }
#pragma unroll
  for (int o = 32; o; o >>= 1) m = max(m, (uint32_t)__shfl_xor((int)m, o, 64));
  const float top = fmaxf(__uint_as_float(m), 0x1p-100f);
  const bool bad = m >= 0x7f800000u;
  const float r = bad ? 0.f : 127.f / top;
  if (lane == 0) {
    const float s = top / 127.f;  // at least 2^-107: never denormal
    scale[row] = Scale{bad ? __uint_as_float(0x7fc00000u) : __builtin_amdgcn_frexp_mantf(s),
                       bad ? 0 : __builtin_amdgcn_frexp_expf(s)};
  }
  char* pf = frag + (long)(row >> 4) * KS * FRAG + (row & 15) * 16;
  for (int k = 8 * lane; k < KS * 64; k += 512) {
    uint32_t b[8];
    Vec8<T> v;
    v.zero();
    if (row < rows && k < K && !bad) v.load(px + k);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float t = v.get(i) * r;
      b[i] = __float_as_uint(t + 12582912.f) & 255u;  // to nearest even, as an integer
    }
    *reinterpret_cast<uint2*>(pf + (long)(k >> 6) * FRAG + ((k >> 4) & 3) * 256 + (k & 8)) =
        uint2{b[0] | b[1] << 8 | b[2] << 16 | b[3] << 24,
              b[4] | b[5] << 8 | b[6] << 16 | b[7] << 24};
  }
}

// What four outputs share: their scales and biases.
struct Outs {
  float m[4], b[4];
  int e[4];
  __device__ __forceinline__ void load(const Lin8Args& a, const Scale* sw, int n) {
    const int4* pw = reinterpret_cast<const int4*>(sw + n);
    const int4 w0 = pw[0], w1 = pw[1];
    m[0] = __int_as_float(w0.x), m[1] = __int_as_float(w0.z);
    m[2] = __int_as_float(w1.x), m[3] = __int_as_float(w1.z);
    e[0] = w0.y, e[1] = w0.w, e[2] = w1.y, e[3] = w1.w;
    const float4 v = a.bias ? *reinterpret_cast<const float4*>(a.bias + n)
                            : make_float4(0.f, 0.f, 0.f, 0.f);
    b[0] = v.x, b[1] = v.y, b[2] = v.z, b[3] = v.w;
  }
};

// four outputs of a row
template <int ACT>
__device__ __forceinline__ uint2 out4(i32x4_t acc, Scale sx, const Outs& o) {
  float v[4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
    v[i] = act_f<ACT>(ldexpf((float)acc[i] * sx.m * o.m[i], sx.e + o.e[i]) + o.b[i]);
  return uint2{pack2(v[0], v[1]), pack2(v[2], v[3])};
}

// Few rows: a block of 4 waves takes 16 outputs and TT x 16 rows, its waves a
// quarter of K each, straight from memory; their sums meet in LDS.
template <int ACT, int TT>
__global__ __launch_bounds__(256) void k_lin8_few(Lin8Args a, Laid x, Laid w) {
  __shared__ i32x4_t part[4][TT][64];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int KS = (int)pad_to(a.K, 64) / 64;
  const int tn = blockIdx.x, tt = blockIdx.y * TT;
  const char* pw = w.frag + (long)tn * KS * FRAG + lane * 16;
  const char* px = x.frag + (long)tt * KS * FRAG + lane * 16;
  i32x4_t acc[TT];
#pragma unroll
  for (int i = 0; i < TT; ++i) acc[i] = i32x4_t{0, 0, 0, 0};
#pragma unroll 4
  for (int k = wave; k < KS; k += 4) {
    const i32x4_t fw = *reinterpret_cast<const i32x4_t*>(pw + (long)k * FRAG);
#pragma unroll
    for (int i = 0; i < TT; ++i) {
      const i32x4_t fx = *reinterpret_cast<const i32x4_t*>(px + ((long)i * KS + k) * FRAG);
      acc[i] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fw, fx, acc[i], 0, 0, 0);
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
          out4<ACT>(s, x.scale[t], o);
    }
  }
}

// BT rows x BN outputs per block, WT x WN per wave
template <int BT_, int BN_, int WT_, int WN_, int STAGES_>
struct Tile {
  static constexpr int BT = BT_, BN = BN_, WT = WT_, WN = WN_, STAGES = STAGES_;
  static constexpr int WAVES_T = BT / WT, NW = WAVES_T * (BN / WN), NT = NW * 64;
  static constexpr int TT = WT / 16, TN = WN / 16;
  static constexpr int FT = BT / 16, FN = BN / 16, STAGE = (FT + FN) * FRAG;
  static constexpr int NU = (FT + FN) / NW;  // fragments per wave and step
  static constexpr int LDS = STAGES * STAGE;
  // outputs on their way out: WT rows of each wave, which start 16 bytes apart
  // modulo the banks
  static constexpr int PY = WN * 2 + 16, OUT = WT * PY, CPR = WN / 8;
  static_assert(NU * NW == FT + FN && FT % NW == 0, "loads");
  static_assert(NW * OUT <= LDS, "outputs");
  static_assert(LDS <= 160 * 1024 && (STAGES - 2) * NU < 64, "LDS, vmcnt");
};

template <int N>
__device__ __forceinline__ void wait_vmcnt() {
  __builtin_amdgcn_s_waitcnt((N & 15) | ((N >> 4) << 14) | (7 << 4) | (15 << 8));
}
__device__ __forceinline__ void lgkm_wait0() {
  __builtin_amdgcn_s_waitcnt(15 | (7 << 4) | (0 << 8) | (3 << 14));
}
// ds_read_b128 at addr + OFF; inline, since the compiler would wait for the
// LDS-DMA before it; the caller waits
template <int OFF>
__device__ __forceinline__ i32x4_t ds_rd128(uint32_t addr) {
  i32x4_t v;
  asm volatile("ds_read_b128 %0, %1 offset:%2" : "=v"(v) : "v"(addr), "i"(OFF));
  return v;
}
template <int N>
__device__ __forceinline__ void ds_rd_n(i32x4_t* f, uint32_t addr) {
  if constexpr (N > 0) {
    ds_rd_n<N - 1>(f, addr);
    f[N - 1] = ds_rd128<(N - 1) * FRAG>(addr);
  }
}
__device__ __forceinline__ void tie(i32x4_t& v) { asm volatile("" : "+v"(v)); }
__device__ __forceinline__ uint32_t lds_at(const void* p) {
  return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) char*)p;
}
__device__ __forceinline__ int xcd_order(int b, int n) {
  const int q = n >> 3, r = n & 7, x = b & 7;
  return x * q + (x < r ? x : r) + (b >> 3);
}

template <class C, int ACT>
__global__ __launch_bounds__(C::NT, 2) void k_lin8(Lin8Args a, Laid x, Laid w, int tilesN) {
#if defined(__HIP_DEVICE_COMPILE__)
  __shared__ __attribute__((aligned(1024))) char smem[C::LDS];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wt = wave % C::WAVES_T, wn = wave / C::WAVES_T;
  const int lb = xcd_order(blockIdx.x, gridDim.x);
  const int tt = lb / tilesN, tn = lb - tt * tilesN;
  const int KT = (int)pad_to(a.K, 64) / 64;
  // rows are padded to whole tiles: every fragment of a tile exists
  const char* src[C::NU];
#pragma unroll
  for (int u = 0; u < C::NU; ++u) {
    const int f = u * C::NW + wave;
    src[u] = (f < C::FT ? x.frag + ((long)tt * C::FT + f) * KT * FRAG
                        : w.frag + ((long)tn * C::FN + f - C::FT) * KT * FRAG) +
             lane * 16;
  }
  auto issue = [&](int kt, int stage) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < C::NU; ++u)
      __builtin_amdgcn_global_load_lds(
          src[u] + (long)kt * FRAG,
          (lds_ptr_t)(smem + stage * C::STAGE + (u * C::NW + wave) * FRAG), 16, 0, 0);
  };
  i32x4_t acc[C::TN][C::TT];
#pragma unroll
  for (int j = 0; j < C::TN; ++j)
#pragma unroll
    for (int i = 0; i < C::TT; ++i) acc[j][i] = i32x4_t{0, 0, 0, 0};
  const uint32_t base = lds_at(smem) + lane * 16;
#pragma unroll
  for (int i = 0; i < C::STAGES - 1; ++i)
    if (i < KT) issue(i, i);
  int stage = 0;
  for (int kt = 0; kt < KT; ++kt) {
    // this step's fragments are there: at most the later stages' loads are not
    if (kt + C::STAGES - 2 < KT)
      wait_vmcnt<(C::STAGES - 2) * C::NU>();
    else
      wait_vmcnt<0>();
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
    if (kt + C::STAGES - 1 < KT)
      issue(kt + C::STAGES - 1, stage == 0 ? C::STAGES - 1 : stage - 1);
    const uint32_t sb = base + stage * C::STAGE;
    i32x4_t fx[C::TT], fw[C::TN];
    ds_rd_n<C::TT>(fx, sb + wt * C::TT * FRAG);
    ds_rd_n<C::TN>(fw, sb + (C::FT + wn * C::TN) * FRAG);
    lgkm_wait0();
#pragma unroll
    for (int i = 0; i < C::TT; ++i) tie(fx[i]);
#pragma unroll
    for (int j = 0; j < C::TN; ++j) tie(fw[j]);
#pragma unroll
    for (int j = 0; j < C::TN; ++j)
#pragma unroll
      for (int i = 0; i < C::TT; ++i)
        acc[j][i] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fw[j], fx[i], acc[j][i], 0, 0, 0);
    __builtin_amdgcn_sched_barrier(0);
    stage = stage + 1 == C::STAGES ? 0 : stage + 1;
  }
  // lane: outputs 4 (lane / 16) .. + 3 of row lane % 16 of each 16 x 16.  They
  // go through LDS, so that whole rows of a wave's outputs leave together: 8
  // bytes a lane straight to memory took 90 us more at 8192 x 1408 x 5632.
  __syncthreads();  // all waves are done with the stages
  char* out = smem + wave * C::OUT;
  const long t0 = (long)tt * C::BT + wt * C::WT;
  const int n0 = tn * C::BN + wn * C::WN;
  Scale sx[C::TT];
#pragma unroll
  for (int i = 0; i < C::TT; ++i) sx[i] = x.scale[t0 + i * 16 + (lane & 15)];
#pragma unroll
  for (int j = 0; j < C::TN; ++j) {
    const int n = j * 16 + 4 * (lane >> 4);
    if (n0 + n >= a.N) continue;
    Outs o;
    o.load(a, w.scale, n0 + n);
#pragma unroll
    for (int i = 0; i < C::TT; ++i)
      *reinterpret_cast<uint2*>(out + (i * 16 + (lane & 15)) * C::PY + n * 2) =
          out4<ACT>(acc[j][i], sx[i], o);
  }
  lgkm_wait0();
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
  hipLaunchKernelGGL((k_lin8<C, ACT>), dim3(tilesN * tilesT), dim3(C::NT), 0, st, a, x, w, tilesN);
  return hipGetLastError();
}

template <int ACT>
hipError_t run(const Lin8Args& a, Laid x, Laid w, hipStream_t st) {
  if (a.tokens <= 64) {
    const int tn = (a.N + 15) / 16;
    if (a.tokens <= 16)
      hipLaunchKernelGGL((k_lin8_few<ACT, 1>), dim3(tn, 1), dim3(256), 0, st, a, x, w);
    else
      hipLaunchKernelGGL((k_lin8_few<ACT, 2>), dim3(tn, (a.tokens + 31) / 32), dim3(256), 0, st, a,
                         x, w);
    return hipGetLastError();
  }
  const long big = (long)((a.tokens + 127) / 128) * ((a.N + 255) / 256);
  return big >= 256 ? tiles<Tile<128, 256, 64, 128, 3>, ACT>(a, x, w, st)
                    : tiles<Tile<64, 128, 32, 64, 3>, ACT>(a, x, w, st);
}

template <typename T>
hipError_t rows8(int rows, int K, const void* x, long xt, Laid to, hipStream_t st) {
  hipLaunchKernelGGL(k_rows8<T>, dim3((pad_to(rows, 16) + 3) / 4), dim3(256), 0, st, rows, K,
                     static_cast<const T*>(x), xt, const_cast<Scale*>(to.scale),
                     const_cast<char*>(to.frag));
  return hipGetLastError();
}

}  // namespace

size_t lin8_weight_bytes(int K, int N) { return laid_bytes(N, K); }
size_t lin8_ws_bytes(int tokens, int K, int) { return tokens ? laid_bytes(tokens, K) : 0; }

hipError_t launch_lin8_pack(int K, int N, const void* w, int w_dtype, void* weights,
                            hipStream_t st) {
  const Laid to = laid(weights, N);
  return w_dtype == PULSE_BF16 ? rows8<uint16_t>(N, K, w, K, to, st)
                               : rows8<float>(N, K, w, K, to, st);
}

hipError_t launch_lin8(const Lin8Args& a, hipStream_t st) {
  if (a.tokens == 0) return hipSuccess;
  const Laid x = laid(a.ws, a.tokens), w = laid(a.weights, a.N);
  const hipError_t e = rows8<uint16_t>(a.tokens, a.K, a.x, a.xt, x, st);
  if (e != hipSuccess) return e;
  switch (a.act) {
    case PULSE_ACT_GELU: return run<PULSE_ACT_GELU>(a, x, w, st);
    case PULSE_ACT_SILU: return run<PULSE_ACT_SILU>(a, x, w, st);
    default: return run<PULSE_ACT_NONE>(a, x, w, st);
  }
}

}  // namespace pulse
