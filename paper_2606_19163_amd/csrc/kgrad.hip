// Weight gradient of a linear layer whose input is kept in 8 bits (gfx950):
// dw[n][c] = sum_t dy[t][n] x[t][c] on bf16 MFMA.  A kept value is a whole
// number of at most 7 bits times a power of two, which bf16 holds exactly, so
// that products are exact and only the fp32 sums round.
//
// Bound by what feeds the MFMAs.  Turning a value to bf16 takes two and a half
// vector instructions, and vector and matrix instructions hardly overlap on a
// SIMD: turned in every block that reads it (once per 64 outputs), 16384 x 1408
// x 5632 took 300 us.  From 7 GFLOP on a launch of its own turns x once, to the
// fragments that the MFMAs take (15 us there), and the product runs at 1.03
// PFLOP/s: 251 us traced, MFMA busy 55 %, behind the LDS-DMA of both operands, 64 KB
// per 2 x 128 x 128 x 64 and CU (a pass in a loop of such 256 to 260 us in all).
// 256 x 128 tiles move a quarter less, but leave one block per CU: 272 against 260 us
// then, 518 against 565 for 16384 x 2048 x 8192.  Four waves of 128 x 64 took 450: the
// compiler moves accumulators between register files.  Below 7 GFLOP, or with an
// axis of 64, a block of 64 x 64 turns its own x, both operands by way of registers:
// 2747 x 320 x 1280 in five parts 16.5 us with their sums, ten steps of load latency.
#include "keepvec.hpp"
#include "ldscopy.hpp"

namespace pulse {
namespace {

typedef __attribute__((__vector_size__(8 * sizeof(__bf16)))) __bf16 bf16x8_t;
typedef __attribute__((__vector_size__(4 * sizeof(float)))) float f32x4_t;
typedef short v4s __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));

// what lanes past the last token, output or channel fetch
__device__ __attribute__((aligned(16))) const uint32_t kgrad_zero[4] = {0, 0, 0, 0};

constexpr int BK = 64;  // tokens per step

// Tiles are token-major rows of P bytes, row r rotated by a (r & 3) + b ((r >>
// 3) & 1) units of 32 bytes, so that each half-wave of a transpose read (rows
// {0..3, 8..11} or {16..19, 24..27} of a 32-row slice, 32 bytes per row) hits
// 8 distinct 32-byte bank groups of the 64-bank LDS.
constexpr int rot_bad(int P, int a, int b) {
  const int U = P / 32;
  int bad = 0;
  for (int hw = 0; hw < 2; ++hw)
    for (int u = 0; u < U; ++u) {
      int seen = 0;
      for (int g = 2 * hw; g < 2 * hw + 2; ++g)
        for (int q = 0; q < 4; ++q) {
          const int r = 8 * g + q;
          const int grp = (r * U + (u + a * (r & 3) + b * ((r >> 3) & 1)) % U) % 8;
          if ((seen >> grp) & 1) ++bad;
          seen |= 1 << grp;
        }
    }
  return bad;
}
constexpr int best_rot(int P) {  // a + 256 b of the first pair with the fewest conflicts
  const int U = P / 32;
  int best = 0, least = 1 << 30;
  for (int a = 0; a < U; ++a)
    for (int b = 0; b < U; ++b) {
      const int bad = rot_bad(P, a, b);
      if (bad < least) {
        best = a + 256 * b;
        least = bad;
      }
    }
  return best;
}
template <int P>
__device__ __forceinline__ int rot_of(int r) {
  constexpr int R = best_rot(P);
  return 2 * ((R % 256) * (r & 3) + (R / 256) * ((r >> 3) & 1));
}
// slot of 16-byte chunk c of row r, and the chunk in slot s
template <int P>
__device__ __forceinline__ int slot_of(int c, int r) {
  return (c + rot_of<P>(r)) % (P / 16);
}
template <int P>
__device__ __forceinline__ int chunk_in(int s, int r) {
  return (s + 4 * (P / 16) - rot_of<P>(r)) % (P / 16);
}

// The rotation turns by at most four rows of chunks, which chunk_in adds.
template <int P>
constexpr bool rot_fits = 2 * (3 * (best_rot(P) % 256) + best_rot(P) / 256) <= 4 * (P / 16);

// four tokens of a column of a tile at p
__device__ __forceinline__ v4s read_tr(const char* p) {
#if defined(__HIP_DEVICE_COMPILE__)
  return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4s*)p);
#else
  return v4s{};
#endif
}
// eight tokens of it, in rows of P bytes
template <int P>
__device__ __forceinline__ bf16x8_t read_col(const char* p) {
  const v4s lo = read_tr(p), hi = read_tr(p + 4 * P);
  return __builtin_bit_cast(bf16x8_t, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
}

// One load from memory, whatever the compiler knows of the address: it would turn the
// choice of a pad into a branch around the load, behind which it waits for all.
template <typename T>
__device__ __forceinline__ T ld_once(const void* p) {
  uint64_t at = reinterpret_cast<uint64_t>(p);
#if defined(__HIP_DEVICE_COMPILE__)
  asm volatile("" : "+v"(at));
#endif
  return *(const __attribute__((address_space(1))) T*)at;
}

// sixteen kept values as bf16, at `to` and at the chunk behind it
__device__ __forceinline__ void turn16(char* to, u32x4_t q, float step) {
  float v[16];
  unkeep4(v, q.x, step);
  unkeep4(v + 4, q.y, step);
  unkeep4(v + 8, q.z, step);
  unkeep4(v + 12, q.w, step);
  u32x4_t* p = reinterpret_cast<u32x4_t*>(to);
  p[0] = u32x4_t{pack2(v[0], v[1]), pack2(v[2], v[3]), pack2(v[4], v[5]), pack2(v[6], v[7])};
  p[1] = u32x4_t{pack2(v[8], v[9]), pack2(v[10], v[11]), pack2(v[12], v[13]), pack2(v[14], v[15])};
}

struct Split {
  int tilesC, tiles, chunk;  // chunk: tokens per split, a multiple of BK
  int splits;
  float *part, *bias;        // partial dw [split][N][C] (splits > 1), db [split tilesC][N]
};

// 64 outputs x 64 channels per block, four waves of 32 x 32.
struct Small {
  static constexpr int BN = 64, BC = 64, NT = 256, TN = 2, TC = 2;
  static constexpr int PY = BN * 2, PX = BC * 2;  // row bytes
  static constexpr int Y_BYTES = BK * PY, STAGE = Y_BYTES + BK * PX;
  static constexpr int YU = Y_BYTES / (NT * 16);  // 16-byte loads of dy per thread and step
  static_assert(BK * BC == NT * 16, "one load of x");
  static_assert(rot_fits<PY> && rot_fits<PX>, "chunk_in");
};

template <bool BIAS>
__global__ __launch_bounds__(Small::NT, 3) void k_kgrad(KgradArgs a, Split s, const uint8_t* q,
                                                        const uint8_t* e) {
  using C = Small;
  __shared__ __attribute__((aligned(1024))) char smem[2 * C::STAGE];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wn = wave & 1, wc = wave >> 1;
  const int lb = xcd_order(blockIdx.x, gridDim.x);
  const int z = lb / s.tiles, tile = lb - z * s.tiles;
  const int tn = tile / s.tilesC, tc = tile - tn * s.tilesC;
  const int n0 = tn * C::BN, c0 = tc * C::BC;
  const long P = (a.C + 31) / 32 * 32, E = keep_exp_pitch(a.C);
  const long tbeg = (long)z * s.chunk;
  const int len = (int)min((long)s.chunk, a.tokens - tbeg);  // tokens of this split
  const int KT = (len + BK - 1) / BK;

  // slot i of dy's tile is chunk_in(i) of its row; outputs and channels past the last
  // read the first ones', and are not stored
  const uint16_t* ysrc[C::YU];
  int yrow[C::YU];
#pragma unroll
  for (int u = 0; u < C::YU; ++u) {
    const int i = u * C::NT + tid, r = i / (C::PY / 16);
    const int n = n0 + 8 * chunk_in<C::PY>(i - r * (C::PY / 16), r);
    yrow[u] = r;
    ysrc[u] = static_cast<const uint16_t*>(a.dy) + (tbeg + r) * a.dyt + (n < a.N ? n : 0);
  }
  // 16 bytes of a row of x become 32
  const int xrow = tid / (C::BC / 16), xk = tid - xrow * (C::BC / 16);
  const int xc = c0 + 16 * xk < P ? c0 + 16 * xk : 0;
  const uint8_t* xsrc = q + (tbeg + xrow) * P + xc;
  const uint8_t* esrc = e + (tbeg + xrow) * E + (xc >> 7) * 4;
  const int eshift = (xc >> 5 & 3) * 8;
  const int xdst = C::Y_BYTES + xrow * C::PX + 16 * slot_of<C::PX>(2 * xk, xrow);

  // two steps' worth of both on its way, in two sets of registers; zeros past the
  // last token.  Steps are fetched in order.
  struct Step {
    u32x4_t y[C::YU], q;
    uint32_t e;
  };
  const uint8_t* const pad = reinterpret_cast<const uint8_t*>(kgrad_zero);
  auto fetch = [&](int kt, Step& in) __attribute__((always_inline)) {
    const bool ok = kt * BK + xrow < len;
    in.q = ld_once<u32x4_t>(ok ? xsrc : pad);
    in.e = ld_once<uint32_t>(ok ? esrc : pad);
#pragma unroll
    for (int u = 0; u < C::YU; ++u)
      in.y[u] = ld_once<u32x4_t>(
          kt * BK + yrow[u] < len ? reinterpret_cast<const uint8_t*>(ysrc[u]) : pad);
    xsrc += BK * P;
    esrc += BK * E;
#pragma unroll
    for (int u = 0; u < C::YU; ++u) ysrc[u] += BK * a.dyt;
  };
  auto store = [&](int kt, const Step& in) __attribute__((always_inline)) {
    char* sb = smem + (kt & 1) * C::STAGE;
#pragma unroll
    for (int u = 0; u < C::YU; ++u)
      *reinterpret_cast<u32x4_t*>(sb + (u * C::NT + tid) * 16) = in.y[u];
    // here, and not as soon as they are there: the compiler would wait for that
    u32x4_t v = in.q;
    uint32_t b = in.e;
#if defined(__HIP_DEVICE_COMPILE__)
    asm volatile("" : "+v"(v), "+v"(b));
#endif
    turn16(sb + xdst, v, keep_step(b >> eshift & 255u));
  };

  // a lane's column and first token in the transpose reads
  const int g16 = lane >> 4, j16 = lane & 15;
  const int trow = 8 * g16 + (j16 >> 2), tcol = 4 * (j16 & 3);
  int rx[C::TC], ry[C::TN];
#pragma unroll
  for (int i = 0; i < C::TC; ++i) {
    const int col = (wc * C::TC + i) * 16 + tcol;
    rx[i] = C::Y_BYTES + trow * C::PX + slot_of<C::PX>(col >> 3, trow) * 16 + (col & 7) * 2;
  }
#pragma unroll
  for (int j = 0; j < C::TN; ++j) {
    const int col = (wn * C::TN + j) * 16 + tcol;
    ry[j] = trow * C::PY + slot_of<C::PY>(col >> 3, trow) * 16 + (col & 7) * 2;
  }
  f32x4_t acc[C::TC][C::TN], sum[C::TN];
#pragma unroll
  for (int j = 0; j < C::TN; ++j) {
    sum[j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < C::TC; ++i) acc[i][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  }
  bf16x8_t ones;
#pragma unroll
  for (int i = 0; i < 8; ++i) ones[i] = (__bf16)1.0f;

  // Step kt computes from stage kt % 2, while kt + 1 is turned into the other one, which
  // all waves are done with.
  bf16x8_t fx[2][C::TC], fy[2][C::TN];
  auto read = [&](int kt, int h) __attribute__((always_inline)) {
    const char* sb = smem + (kt & 1) * C::STAGE;
#pragma unroll
    for (int i = 0; i < C::TC; ++i) fx[h][i] = read_col<C::PX>(sb + rx[i] + h * 32 * C::PX);
#pragma unroll
    for (int j = 0; j < C::TN; ++j) fy[h][j] = read_col<C::PY>(sb + ry[j] + h * 32 * C::PY);
  };
  auto mma = [&](int h) __attribute__((always_inline)) {
#if defined(__HIP_DEVICE_COMPILE__)
#pragma unroll
    for (int i = 0; i < C::TC; ++i)
#pragma unroll
      for (int j = 0; j < C::TN; ++j)
        acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fx[h][i], fy[h][j], acc[i][j], 0, 0, 0);
#endif
  };
  auto add_bias = [&](int h) __attribute__((always_inline)) {
#if defined(__HIP_DEVICE_COMPILE__)
#pragma unroll
    for (int j = 0; j < C::TN; ++j)
      sum[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, fy[h][j], sum[j], 0, 0, 0);
#endif
  };
  int turn = 0;  // kt % tilesC: the tiles along C share the steps of db
  auto step = [&](int kt, Step& in) __attribute__((always_inline)) {
    read(kt, 0);
    read(kt, 1);
    store(kt + 1, in);
    fetch(kt + 3, in);
    mma(0);
    mma(1);
    if (BIAS) {
      if (turn == tc && wc == 0) {
        add_bias(0);
        add_bias(1);
      }
      turn = turn + 1 == s.tilesC ? 0 : turn + 1;
    }
    __syncthreads();
  };
  Step in[2];
  fetch(0, in[0]);
  fetch(1, in[1]);
  store(0, in[0]);
  fetch(2, in[0]);
  __syncthreads();
  for (int kt = 0; kt < KT; kt += 2) {  // a step past an odd last one adds zeros
    step(kt, in[1]);
    step(kt + 1, in[0]);
  }

  // lane: channels 4 g16 .. + 3 of output j16 of each 16 x 16
  float* dst = s.splits > 1 ? s.part + (long)z * a.N * a.C : a.dw;
  const bool add = s.splits == 1 && a.accumulate;
#pragma unroll
  for (int j = 0; j < C::TN; ++j) {
    const int n = n0 + (wn * C::TN + j) * 16 + j16;
    if (n >= a.N) continue;
#pragma unroll
    for (int i = 0; i < C::TC; ++i) {
      const int c = c0 + (wc * C::TC + i) * 16 + 4 * g16;
      if (c >= a.C) continue;
      f32x4_t* p = reinterpret_cast<f32x4_t*>(dst + (long)n * a.C + c);
      *p = add ? *p + acc[i][j] : acc[i][j];
    }
    if (BIAS && wc == 0 && g16 == 0) s.bias[((long)z * s.tilesC + tc) * a.N + n] = sum[j][0];
  }
}

// Fragments of x in bf16 for many outputs: [c / 16][t / 32] of 1 KB, lane l
// holding channel l % 16 of tokens 8 (l / 16) to + 7, zeros past the last
// token and channel.  A block turns 64 tokens of 128 channels.
constexpr int WIDE_C = 128;
__global__ __launch_bounds__(256) void k_kgrad_turn(KgradArgs a, const uint8_t* q,
                                                    const uint8_t* e, char* frags) {
  constexpr int PX = WIDE_C * 2;
  static_assert(rot_fits<PX>, "chunk_in");
  __shared__ __attribute__((aligned(1024))) char smem[BK * PX];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const long P = (a.C + 31) / 32 * 32, E = keep_exp_pitch(a.C);
  const int c0 = blockIdx.y * WIDE_C;
  const long t0 = (long)blockIdx.x * BK;
  const long blocks32 = (long)gridDim.x * 2;
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    const int i = u * 256 + tid, r = i >> 3, k = i & 7, c = c0 + 16 * k;
    u32x4_t w = {0, 0, 0, 0};
    float step = 0.f;
    if (t0 + r < a.tokens && c < P) {
      w = *reinterpret_cast<const u32x4_t*>(q + (t0 + r) * P + c);
      step = keep_step(e[(t0 + r) * E + (c >> 5)]);
    }
    turn16(smem + r * PX + 16 * slot_of<PX>(2 * k, r), w, step);
  }
  __syncthreads();
  const int trow = 8 * (lane >> 4) + ((lane & 15) >> 2), tcol = 4 * (lane & 3);
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int col = (2 * wave + i) * 16 + tcol;
    const char* from = smem + trow * PX + slot_of<PX>(col >> 3, trow) * 16 + (col & 7) * 2;
    char* dst = frags + ((c0 / 16 + 2 * wave + i) * blocks32 + 2 * blockIdx.x) * 1024 + lane * 16;
    *reinterpret_cast<bf16x8_t*>(dst) = read_col<PX>(from);
    *reinterpret_cast<bf16x8_t*>(dst + 1024) = read_col<PX>(from + 32 * PX);
  }
}

// The gradient from such fragments: 128 outputs x 128 channels per block, four
// waves of 64 x 64.
struct Wide {
  static constexpr int BN = 128, BC = WIDE_C, NW = 4, NT = NW * 64, TN = 4, TC = 4;
  static constexpr int PY = BN * 2, Y_BYTES = BK * PY, X_BYTES = BK * BC * 2;
  static constexpr int STAGE = Y_BYTES + X_BYTES;
  static constexpr int YU = Y_BYTES / (NT * 16), XU = X_BYTES / (NT * 16);
  static_assert(rot_fits<PY>, "chunk_in");
};

template <bool BIAS>
__global__ __launch_bounds__(Wide::NT, 2) void k_kgrad_wide(KgradArgs a, Split s,
                                                            const char* frags) {
  using C = Wide;
  __shared__ __attribute__((aligned(1024))) char smem[2 * C::STAGE];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wn = wave & 1, wc = wave >> 1;
  const int lb = xcd_order(blockIdx.x, gridDim.x);
  const int z = lb / s.tiles, tile = lb - z * s.tiles;
  const int tn = tile / s.tilesC, tc = tile - tn * s.tilesC;
  const int n0 = tn * C::BN, c0 = tc * C::BC;
  const long tbeg = (long)z * s.chunk;
  const int len = (int)min((long)s.chunk, a.tokens - tbeg);
  const int KT = (len + BK - 1) / BK;
  const long blocks32 = (long)((a.tokens + BK - 1) / BK) * 2;

  // lane slot i of a load is chunk_in(i) of its row; outputs past the last read
  // the first ones', and are not stored
  const uint16_t* ysrc[C::YU];
  int yrow[C::YU];
#pragma unroll
  for (int u = 0; u < C::YU; ++u) {
    const int i = u * C::NT + tid;
    const int r = i / (C::PY / 16);
    const int n = n0 + 8 * chunk_in<C::PY>(i - r * (C::PY / 16), r);
    yrow[u] = r;
    ysrc[u] = static_cast<const uint16_t*>(a.dy) + (tbeg + r) * a.dyt + (n < a.N ? n : 0);
  }
  // fragment f of a stage: channels f / 2, half f % 2
  const char* xsrc[C::XU];
#pragma unroll
  for (int u = 0; u < C::XU; ++u) {
    const int f = u * C::NW + wave;
    xsrc[u] = frags + ((c0 / 16 + f / 2) * blocks32 + tbeg / 32 + f % 2) * 1024 + lane * 16;
  }
  const uint32_t sbase = lds_at(smem) + wave * 1024;
  auto fetch = [&](int kt) __attribute__((always_inline)) {
    const uint32_t base = sbase + (kt & 1) * C::STAGE;
    if ((kt + 1) * BK <= len) {
#pragma unroll
      for (int u = 0; u < C::YU; ++u) lds_copy16(ysrc[u], base + u * C::NT * 16);
    } else {
#pragma unroll
      for (int u = 0; u < C::YU; ++u)
        lds_copy16(kt * BK + yrow[u] < len ? static_cast<const void*>(ysrc[u])
                                           : static_cast<const void*>(kgrad_zero),
                   base + u * C::NT * 16);
    }
#pragma unroll
    for (int u = 0; u < C::YU; ++u) ysrc[u] += BK * a.dyt;
#pragma unroll
    for (int u = 0; u < C::XU; ++u) {
      lds_copy16(xsrc[u], base + C::Y_BYTES + u * C::NW * 1024);
      xsrc[u] += 2 * 1024;
    }
  };

  const int g16 = lane >> 4, j16 = lane & 15;
  const int trow = 8 * g16 + (j16 >> 2), tcol = 4 * (j16 & 3);
  const int rx = C::Y_BYTES + wc * C::TC * 2048 + lane * 16;
  int ry[C::TN];
#pragma unroll
  for (int j = 0; j < C::TN; ++j) {
    const int col = (wn * C::TN + j) * 16 + tcol;
    ry[j] = trow * C::PY + slot_of<C::PY>(col >> 3, trow) * 16 + (col & 7) * 2;
  }
  f32x4_t acc[C::TC][C::TN], sum[C::TN];
#pragma unroll
  for (int j = 0; j < C::TN; ++j) {
    sum[j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < C::TC; ++i) acc[i][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  }
  bf16x8_t ones;
#pragma unroll
  for (int i = 0; i < 8; ++i) ones[i] = (__bf16)1.0f;

  bf16x8_t fx[2][C::TC], fy[2][C::TN];
  auto read = [&](int kt, int h) __attribute__((always_inline)) {
    const char* sb = smem + (kt & 1) * C::STAGE;
#pragma unroll
    for (int i = 0; i < C::TC; ++i)
      fx[h][i] = *reinterpret_cast<const bf16x8_t*>(sb + rx + h * 1024 + i * 2048);
#pragma unroll
    for (int j = 0; j < C::TN; ++j) fy[h][j] = read_col<C::PY>(sb + ry[j] + h * 32 * C::PY);
  };
  auto mma = [&](int h) __attribute__((always_inline)) {
#if defined(__HIP_DEVICE_COMPILE__)
#pragma unroll
    for (int i = 0; i < C::TC; ++i)
#pragma unroll
      for (int j = 0; j < C::TN; ++j)
        acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fx[h][i], fy[h][j], acc[i][j], 0, 0, 0);
#endif
  };
  auto add_bias = [&](int h) __attribute__((always_inline)) {
#if defined(__HIP_DEVICE_COMPILE__)
#pragma unroll
    for (int j = 0; j < C::TN; ++j)
      sum[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, fy[h][j], sum[j], 0, 0, 0);
#endif
  };

  // Step kt computes from stage kt % 2, while kt + 1 is on its way to the other,
  // which all waves are done with.  Fragments are read, then multiplied: what one
  // block waits for, the other on the CU covers.  Halves overlapped in one wave
  // (reads behind the other half's MFMAs) take 270 us instead of 256.
  fetch(0);
  int turn = 0;  // kt % tilesC: the tiles along C share the steps of db
  for (int kt = 0; kt < KT; ++kt) {
    lds_meet<0>();
    if (kt + 1 < KT) fetch(kt + 1);
    __builtin_amdgcn_sched_barrier(0);
    read(kt, 0);
    read(kt, 1);
    __builtin_amdgcn_sched_barrier(0);
    mma(0);
    mma(1);
    if (BIAS) {
      if (turn == tc && wc == 0) {
        add_bias(0);
        add_bias(1);
      }
      turn = turn + 1 == s.tilesC ? 0 : turn + 1;
    }
    __builtin_amdgcn_sched_barrier(0);
  }

  float* dst = s.splits > 1 ? s.part + (long)z * a.N * a.C : a.dw;
  const bool add = s.splits == 1 && a.accumulate;
#pragma unroll
  for (int j = 0; j < C::TN; ++j) {
    const int n = n0 + (wn * C::TN + j) * 16 + j16;
    if (n >= a.N) continue;
#pragma unroll
    for (int i = 0; i < C::TC; ++i) {
      const int c = c0 + (wc * C::TC + i) * 16 + 4 * g16;
      if (c >= a.C) continue;
      f32x4_t* p = reinterpret_cast<f32x4_t*>(dst + (long)n * a.C + c);
      *p = add ? *p + acc[i][j] : acc[i][j];
    }
    if (BIAS && wc == 0 && g16 == 0) s.bias[((long)z * s.tilesC + tc) * a.N + n] = sum[j][0];
  }
}

// Blocks below `wblocks`: four values of dw each thread, summed over the
// splits; the others: db, 16 outputs x 16 partial sums of the rows. Eight loads
// are in flight together: a load's latency, and no rate, is what bounds both.
__global__ __launch_bounds__(256) void k_kgrad_sum(KgradArgs a, Split s, int wblocks) {
  if ((int)blockIdx.x < wblocks) {
    const long at = 4 * ((long)blockIdx.x * 256 + threadIdx.x), total = (long)a.N * a.C;
    if (at >= total) return;
    float4 v = *reinterpret_cast<const float4*>(s.part + at);
    for (int z = 1; z < s.splits; z += 8) {
      float4 w[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const int i = z + k < s.splits ? z + k : z;
        w[k] = *reinterpret_cast<const float4*>(s.part + i * total + at);
      }
#pragma unroll
      for (int k = 0; k < 8; ++k)
        if (z + k < s.splits) v.x += w[k].x, v.y += w[k].y, v.z += w[k].z, v.w += w[k].w;
    }
    float4* p = reinterpret_cast<float4*>(a.dw + at);
    if (a.accumulate) {
      const float4 w = *p;
      v.x += w.x, v.y += w.y, v.z += w.z, v.w += w.w;
    }
    *p = v;
    return;
  }
  __shared__ float sm[16][16];
  const int lane = threadIdx.x & 15, g = threadIdx.x >> 4;
  const int n = (blockIdx.x - wblocks) * 16 + lane, rows = s.splits * s.tilesC;
  float v = 0.f;
  if (n < a.N)
    for (int r = g; r < rows; r += 128) {
      float w[8];
#pragma unroll
      for (int k = 0; k < 8; ++k)
        w[k] = s.bias[(long)(r + 16 * k < rows ? r + 16 * k : r) * a.N + n];
#pragma unroll
      for (int k = 0; k < 8; ++k) v += r + 16 * k < rows ? w[k] : 0.f;
    }
  sm[g][lane] = v;
  __syncthreads();
  if (g == 0 && n < a.N) {
    v = 0.f;
#pragma unroll
    for (int k = 0; k < 16; ++k) v += sm[k][lane];
    a.db[n] = a.accumulate ? a.db[n] + v : v;
  }
}

__global__ __launch_bounds__(256) void k_kgrad_clear(float* p, long n) {
  const long i = 4 * ((long)blockIdx.x * 256 + threadIdx.x);  // n is a multiple of 8
  if (i < n) *reinterpret_cast<float4*>(p + i) = make_float4(0.f, 0.f, 0.f, 0.f);
}

struct Plan {
  bool large;
  Split s;
  size_t sums;   // bytes of the partial sums
  size_t bytes;  // with the fragments of x
};

Plan plan_of(int tokens, int C, int N) {
  Plan p{};
  // The launch that turns x first pays from 7 GFLOP on: 16.5 against 12.7 us at
  // 512 x 768 x 2304, 28.4 against 28.3 at 2048 x 768 x 2304, 31.3 against 36.7 at
  // 8192 x 768 x 768, 23.5 against 30.2 at 512 x 1408 x 5632. An axis of 64 fills
  // half of its tile: 56 against 129 us at 20000 x 6000 x 64, 58 against 67 at
  // 20000 x 64 x 6000.
  p.large = (double)tokens * N * C >= 3.5e9 && N > 64 && C > 64;
  const int bn = p.large ? Wide::BN : Small::BN, bc = p.large ? Wide::BC : Small::BC;
  p.s.tilesC = (C + bc - 1) / bc;
  p.s.tiles = (N + bn - 1) / bn * p.s.tilesC;
  const int steps = (tokens + BK - 1) / BK;
  const int room = 512;
  int splits = p.s.tiles >= room ? 1 : room / p.s.tiles;
  if (splits > (steps + 7) / 8) splits = (steps + 7) / 8;
  if (splits < 1) splits = 1;
  p.s.chunk = (steps + splits - 1) / splits * BK;
  p.s.splits = tokens ? (tokens + p.s.chunk - 1) / p.s.chunk : 1;
  const size_t part = p.s.splits > 1 ? (size_t)p.s.splits * N * C : 0;
  p.sums = ((part + (size_t)p.s.splits * p.s.tilesC * N) * 4 + 1023) / 1024 * 1024;
  p.bytes = p.sums + (p.large ? (size_t)steps * BK * p.s.tilesC * WIDE_C * 2 : 0);
  return p;
}

hipError_t run(const KgradArgs& a, const Plan& p, const uint8_t* q, const uint8_t* e,
               hipStream_t st) {
  if (!p.large) {
    auto kern = a.db ? k_kgrad<true> : k_kgrad<false>;
    hipLaunchKernelGGL(kern, dim3(p.s.tiles * p.s.splits), dim3(Small::NT), 0, st, a, p.s, q, e);
    return hipGetLastError();
  }
  char* frags = reinterpret_cast<char*>(a.ws) + p.sums;
  hipLaunchKernelGGL(k_kgrad_turn, dim3((a.tokens + BK - 1) / BK, p.s.tilesC), dim3(256), 0, st, a,
                     q, e, frags);
  const hipError_t err = hipGetLastError();
  if (err != hipSuccess) return err;
  auto kern = a.db ? k_kgrad_wide<true> : k_kgrad_wide<false>;
  hipLaunchKernelGGL(kern, dim3(p.s.tiles * p.s.splits), dim3(Wide::NT), 0, st, a, p.s, frags);
  return hipGetLastError();
}

hipError_t clear(float* p, long n, hipStream_t st) {
  hipLaunchKernelGGL(k_kgrad_clear, dim3((n / 4 + 255) / 256), dim3(256), 0, st, p, n);
  return hipGetLastError();
}

// Tokens at a time: their fragments take at most 512 MB.
int chunk_of(int tokens, int C) {
  const long most = (INT64_C(1) << 28) / ((C + WIDE_C - 1) / WIDE_C * WIDE_C) / BK * BK;
  return tokens < most ? tokens : (int)most;
}

}  // namespace

size_t kgrad_bytes(int tokens, int C, int N) {
  if (tokens == 0) return 0;
  const int chunk = chunk_of(tokens, C), rest = tokens % chunk;
  const size_t a = plan_of(chunk, C, N).bytes, b = rest ? plan_of(rest, C, N).bytes : 0;
  return a > b ? a : b;
}

hipError_t launch_kgrad(const KgradArgs& args, hipStream_t st) {
  if (args.tokens == 0) {
    if (args.accumulate) return hipSuccess;
    const hipError_t e = clear(args.dw, (long)args.N * args.C, st);
    return e != hipSuccess || !args.db ? e : clear(args.db, args.N, st);
  }
  const uint8_t* q = static_cast<const uint8_t*>(args.kept);
  const uint8_t* e = q + keep_exps_at(args.C, args.tokens);
  const int chunk = chunk_of(args.tokens, args.C);
  for (int t = 0; t < args.tokens; t += chunk) {
    KgradArgs a = args;
    a.tokens = args.tokens - t < chunk ? args.tokens - t : chunk;
    a.dy = static_cast<const uint16_t*>(args.dy) + t * args.dyt;
    if (t) a.accumulate = 1;
    Plan p = plan_of(a.tokens, a.C, a.N);
    p.s.part = a.ws;
    p.s.bias = a.ws + (p.s.splits > 1 ? (size_t)p.s.splits * a.N * a.C : 0);
    hipError_t err = run(a, p, q + t * keep_pitch(a.C), e + t * keep_exp_pitch(a.C), st);
    if (err != hipSuccess) return err;
    const int wblocks = p.s.splits > 1 ? (int)(((long)a.N * a.C / 4 + 255) / 256) : 0;
    const int blocks = wblocks + (a.db ? (a.N + 15) / 16 : 0);
    if (!blocks) continue;
    hipLaunchKernelGGL(k_kgrad_sum, dim3(blocks), dim3(256), 0, st, a, p.s, wblocks);
    err = hipGetLastError();
    if (err != hipSuccess) return err;
  }
  return hipSuccess;
}

}  // namespace pulse
