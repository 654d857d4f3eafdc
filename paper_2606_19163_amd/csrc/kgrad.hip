// Weight gradient of a linear layer whose input is kept in 8 bits (gfx950):
// dw[n][c] = sum_t dy[t][n] x[t][c] on bf16 MFMA.  A kept value is a whole
// number of at most 7 bits times a power of two, which bf16 holds exactly, so
// that products are exact and only the fp32 sums round.
//
// Bound by what feeds the MFMAs.  Turning a value to bf16 takes two and a half
// vector instructions, and vector and matrix instructions hardly overlap on a
// SIMD: turned in every block that reads it (once per 64 outputs), 16384 x 1408
// x 5632 took 300 us.  From 7 GFLOP on a launch of its own turns x once, to the
// fragments that the MFMAs take (15 us there), and the product runs at 1.0 to 1.1
// PFLOP/s: 244 us, MFMA busy 53 %, behind the LDS-DMA of both operands, 64 KB per
// 2 x 128 x 128 x 64 and CU.  256 x 128 tiles move a quarter less, but leave one
// block per CU: 272 against 260 us in all, 518 against 565 for 16384 x 2048 x 8192.
// Four waves of 128 x 64 took 450: the compiler moves accumulators between
// register files.  Below 7 GFLOP, or with an axis of 64, a block of 64 x 64
// turns its own x: 2747 x 320 x 1280 in five parts 16.4 us with their sums, ten
// steps of load latency.
#include "keepvec.hpp"

namespace pulse {
namespace {

typedef __attribute__((__vector_size__(8 * sizeof(__bf16)))) __bf16 bf16x8_t;
typedef __attribute__((__vector_size__(4 * sizeof(float)))) float f32x4_t;
typedef short v4s __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) void* lds_ptr_t;

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

// BN outputs x BC channels per block, WN x WC per wave
template <int BN_, int BC_, int WN_, int WC_>
struct Tile {
  static constexpr int BN = BN_, BC = BC_, WN = WN_, WC = WC_;
  static constexpr int WAVES_N = BN / WN, WAVES_C = BC / WC, NW = WAVES_N * WAVES_C;
  static constexpr int NT = NW * 64;
  static constexpr int TN = WN / 16, TC = WC / 16;
  static constexpr int PY = BN * 2, PX = BC * 2;  // row bytes
  static constexpr int Y_BYTES = BK * PY, X_BYTES = BK * PX, STAGE = Y_BYTES + X_BYTES;
  static constexpr int YU = Y_BYTES / (NT * 16);  // 16-byte loads per thread and step
  static constexpr int XU = BK * BC / (NT * 16);
  static constexpr int STAGES = 3, LDS = STAGES * STAGE;
  static_assert(YU * NT * 16 == Y_BYTES && XU * NT * 16 == BK * BC && XU >= 1, "loads");
  static_assert(36 * PY < 65536 && Y_BYTES + 36 * PX < 65536 && LDS <= 160 * 1024, "LDS");
  static_assert(4 * 3 * (BN / 16 + 4) < 4096, "rotations stay below 4 rows of chunks");
};

__device__ __forceinline__ uint32_t lds_at(const void* p) {
  return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) char*)p;
}

// ds_read_b64_tr_b16 at addr + OFF: four tokens of a column.  Inline, since the
// compiler would wait for the LDS-DMA before it; the caller waits (lgkm_wait).
template <int OFF>
__device__ __forceinline__ v4s ds_rdtr(uint32_t addr) {
  v4s v;
  asm volatile("ds_read_b64_tr_b16 %0, %1 offset:%2" : "=v"(v) : "v"(addr), "i"(OFF));
  return v;
}
// ds_write_b128 at addr + OFF, inline for the same reason
template <int OFF>
__device__ __forceinline__ void ds_wr128(uint32_t addr, uint32_t a, uint32_t b, uint32_t c,
                                         uint32_t d) {
  typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
  const u32x4 v = {a, b, c, d};
  asm volatile("ds_write_b128 %0, %1 offset:%2" ::"v"(addr), "v"(v), "i"(OFF));
}
__device__ __forceinline__ void lgkm_wait0() {
  __builtin_amdgcn_s_waitcnt(15 | (7 << 4) | (0 << 8) | (3 << 14));
}
template <int N>
__device__ __forceinline__ void vm_wait() {
  static_assert(N >= 0 && N < 64, "vmcnt");
  __builtin_amdgcn_s_waitcnt((N & 15) | ((N >> 4) << 14) | (7 << 4) | (15 << 8));
}
// the MFMAs that use v stay below the waits before this
__device__ __forceinline__ void tie(bf16x8_t& v) { asm volatile("" : "+v"(v)); }

// One load instruction, whatever the compiler knows of the address: the waits
// count them.
template <typename T>
__device__ __forceinline__ T ld_once(const void* p) {
  typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
  uint64_t at = reinterpret_cast<uint64_t>(p);
  asm volatile("" : "+v"(at));
  if constexpr (sizeof(T) == 16) {
    const u32x4 v = *(const __attribute__((address_space(1))) u32x4*)at;
    return uint4{v.x, v.y, v.z, v.w};
  } else {
    return *(const __attribute__((address_space(1))) T*)at;
  }
}

__device__ __forceinline__ int xcd_order(int b, int n) {
  const int q = n >> 3, r = n & 7, x = b & 7;
  return x * q + (x < r ? x : r) + (b >> 3);
}

struct Split {
  int tilesC, tiles, chunk;  // chunk: tokens per split, a multiple of BK
  int splits;
  float *part, *bias;        // partial dw [split][N][C] (splits > 1), db [split tilesC][N]
};

template <class C, bool BIAS>
__global__ __launch_bounds__(C::NT, 3) void k_kgrad(KgradArgs a, Split s, const uint8_t* q,
                                                 const uint8_t* e) {
#if defined(__HIP_DEVICE_COMPILE__)
  __shared__ __attribute__((aligned(1024))) char smem[C::LDS];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wn = wave % C::WAVES_N, wc = wave / C::WAVES_N;
  const int lb = xcd_order(blockIdx.x, gridDim.x);
  const int z = lb / s.tiles, tile = lb - z * s.tiles;
  const int tn = tile / s.tilesC, tc = tile - tn * s.tilesC;
  const int n0 = tn * C::BN, c0 = tc * C::BC;
  const long P = (a.C + 31) / 32 * 32, E = keep_exp_pitch(a.C);
  const long tbeg = (long)z * s.chunk;
  const int len = (int)min((long)s.chunk, a.tokens - tbeg);  // tokens of this split
  const int KT = (len + BK - 1) / BK;

  const uint32_t sbase = lds_at(smem);

  // dy goes straight to LDS: lane slot i of a load is chunk_in(i) of its row
  const uint16_t* ysrc[C::YU];
  int yrow[C::YU];
#pragma unroll
  for (int u = 0; u < C::YU; ++u) {
    const int i = u * C::NT + tid;
    const int r = i / (C::PY / 16);
    const int n = n0 + 8 * chunk_in<C::PY>(i - r * (C::PY / 16), r);
    yrow[u] = n < a.N ? r : 1 << 30;
    ysrc[u] = static_cast<const uint16_t*>(a.dy) + (tbeg + r) * a.dyt + n;
  }
  // x goes through registers: 16 bytes of a row become 32
  const uint8_t *xsrc[C::XU], *esrc[C::XU];
  int xrow[C::XU];
  uint32_t xdst[C::XU], eshift[C::XU];
#pragma unroll
  for (int u = 0; u < C::XU; ++u) {
    const int i = u * C::NT + tid;
    const int r = i / (C::BC / 16), k = i - r * (C::BC / 16);
    const int c = c0 + 16 * k;
    xrow[u] = c < P ? r : 1 << 30;
    xsrc[u] = q + (tbeg + r) * P + c;
    esrc[u] = e + (tbeg + r) * E + (c >> 7) * 4;
    eshift[u] = (c >> 5 & 3) * 8;
    xdst[u] = (uint32_t)(C::Y_BYTES + r * C::PX + 16 * slot_of<C::PX>(2 * k, r));
  }
  // two steps' worth of x on its way, in two sets of registers
  struct X {
    uint4 q[C::XU];
    uint32_t e[C::XU];
  };
  const uint8_t* const pad = reinterpret_cast<const uint8_t*>(kgrad_zero);
  // steps are fetched in order
  auto fetch_x = [&](int kt, X& x) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < C::XU; ++u) {
      const bool ok = kt * BK + xrow[u] < len;
      x.q[u] = ld_once<uint4>(ok ? xsrc[u] : pad);
      x.e[u] = ld_once<uint32_t>(ok ? esrc[u] : pad);
      xsrc[u] += BK * P;
      esrc[u] += BK * E;
    }
  };
  auto store_x = [&](int stage, const X& x) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < C::XU; ++u) {
      const float step = keep_step(x.e[u] >> eshift[u] & 255u);
      float v[16];
      unkeep4(v, x.q[u].x, step);
      unkeep4(v + 4, x.q[u].y, step);
      unkeep4(v + 8, x.q[u].z, step);
      unkeep4(v + 12, x.q[u].w, step);
      const uint32_t d = sbase + (uint32_t)(stage * C::STAGE) + xdst[u];
      ds_wr128<0>(d, pack2(v[0], v[1]), pack2(v[2], v[3]), pack2(v[4], v[5]), pack2(v[6], v[7]));
      ds_wr128<16>(d, pack2(v[8], v[9]), pack2(v[10], v[11]), pack2(v[12], v[13]),
                   pack2(v[14], v[15]));
    }
  };
  auto fetch_y = [&](int kt, int stage) __attribute__((always_inline)) {
    char* base = smem + stage * C::STAGE;
#pragma unroll
    for (int u = 0; u < C::YU; ++u) {
      const void* g = kt * BK + yrow[u] < len ? static_cast<const void*>(ysrc[u])
                                              : static_cast<const void*>(kgrad_zero);
      ysrc[u] += BK * a.dyt;
      __builtin_amdgcn_global_load_lds(g, (lds_ptr_t)(base + (u * C::NT + wave * 64) * 16), 16, 0,
                                       0);
    }
  };

  // a lane's column and first token in the transpose reads
  const int g16 = lane >> 4, j16 = lane & 15;
  const int trow = 8 * g16 + (j16 >> 2), tcol = 4 * (j16 & 3);
  uint32_t rx[C::TC], ry[C::TN];
#pragma unroll
  for (int i = 0; i < C::TC; ++i) {
    const int col = wc * C::WC + i * 16 + tcol;
    rx[i] = (uint32_t)(C::Y_BYTES + trow * C::PX + slot_of<C::PX>(col >> 3, trow) * 16 +
                       (col & 7) * 2);
  }
#pragma unroll
  for (int j = 0; j < C::TN; ++j) {
    const int col = wn * C::WN + j * 16 + tcol;
    ry[j] = (uint32_t)(trow * C::PY + slot_of<C::PY>(col >> 3, trow) * 16 + (col & 7) * 2);
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
  auto read = [&](uint32_t sb, auto tag) __attribute__((always_inline)) {
    constexpr int S = decltype(tag)::value;
#pragma unroll
    for (int i = 0; i < C::TC; ++i) {
      const v4s lo = ds_rdtr<(S * 32 + 0) * C::PX>(sb + rx[i]);
      const v4s hi = ds_rdtr<(S * 32 + 4) * C::PX>(sb + rx[i]);
      fx[S][i] =
          __builtin_bit_cast(bf16x8_t, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    }
#pragma unroll
    for (int j = 0; j < C::TN; ++j) {
      const v4s lo = ds_rdtr<(S * 32 + 0) * C::PY>(sb + ry[j]);
      const v4s hi = ds_rdtr<(S * 32 + 4) * C::PY>(sb + ry[j]);
      fy[S][j] =
          __builtin_bit_cast(bf16x8_t, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    }
  };
  auto wait_read = [&](int S) __attribute__((always_inline)) {
    lgkm_wait0();
#pragma unroll
    for (int i = 0; i < C::TC; ++i) tie(fx[S][i]);
#pragma unroll
    for (int j = 0; j < C::TN; ++j) tie(fy[S][j]);
  };
  auto mma = [&](int S) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < C::TC; ++i)
#pragma unroll
      for (int j = 0; j < C::TN; ++j)
        acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fx[S][i], fy[S][j], acc[i][j], 0, 0, 0);
  };
  auto add_bias = [&](int S) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < C::TN; ++j)
      sum[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, fy[S][j], sum[j], 0, 0, 0);
  };

  // Step kt computes from stage kt % 3.  While the MFMAs of its first half run,
  // the second half is read and x of kt + 1 is turned into its stage; between the
  // halves all waves meet: then the first half of kt + 1 is read behind the second
  // half's MFMAs, and dy of kt + 3 may take this stage's place.  A load has two
  // steps to arrive; past the last step they fetch zeros.
  X xs[2];
  int cur = 0;   // kt % 3
  int turn = 0;  // kt % tilesC: the tiles along C share the steps of db
  auto step = [&](int kt, X& x) __attribute__((always_inline)) {
    const int next = cur == 2 ? 0 : cur + 1;
    read(sbase + (uint32_t)(cur * C::STAGE), std::integral_constant<int, 1>());
    vm_wait<2 * C::YU + 2 * C::XU>();  // x of kt + 1
    __builtin_amdgcn_sched_barrier(0);
    store_x(next, x);
    fetch_x(kt + 3, x);
    mma(0);
    // a matrix instruction takes as long as four vector ones beside it
#pragma unroll
    for (int i = 0; i < C::TC * C::TN; ++i) {
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
      __builtin_amdgcn_sched_group_barrier(0x002, 5, 0);
    }
    __builtin_amdgcn_sched_barrier(0);
    wait_read(1);
    if (BIAS) {
      if (turn == tc && wc == 0) {
        add_bias(0);
        add_bias(1);
      }
      turn = turn + 1 == s.tilesC ? 0 : turn + 1;
    }
    vm_wait<C::YU + 4 * C::XU>();
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
    read(sbase + (uint32_t)(next * C::STAGE), std::integral_constant<int, 0>());
    fetch_y(kt + 3, cur);
    mma(1);
    __builtin_amdgcn_sched_barrier(0);
    // here, not at the next step: no register may move while a read is on its
    // way to it, and the compiler does not know that it is
    wait_read(0);
    cur = next;
  };
  // the waits count loads, so that these keep their order
  fetch_x(0, xs[0]);
  store_x(0, xs[0]);
  __builtin_amdgcn_sched_barrier(0);
  fetch_y(0, 0);
  __builtin_amdgcn_sched_barrier(0);
  fetch_x(1, xs[1]);
  __builtin_amdgcn_sched_barrier(0);
  fetch_y(1, 1);
  __builtin_amdgcn_sched_barrier(0);
  fetch_x(2, xs[0]);
  __builtin_amdgcn_sched_barrier(0);
  fetch_y(2, 2);
  __builtin_amdgcn_sched_barrier(0);
  vm_wait<2 * C::YU + 4 * C::XU>();
  lgkm_wait0();
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_sched_barrier(0);
  read(sbase, std::integral_constant<int, 0>());
  wait_read(0);
  for (int kt = 0; kt < KT; kt += 2) {  // a step past an odd last one adds zeros
    step(kt, xs[1]);
    step(kt + 1, xs[0]);
  }
  vm_wait<0>();

  // lane: channels 4 g16 .. + 3 of output j16 of each 16 x 16
  float* dst = s.splits > 1 ? s.part + (long)z * a.N * a.C : a.dw;
  const bool add = s.splits == 1 && a.accumulate;
#pragma unroll
  for (int j = 0; j < C::TN; ++j) {
    const int n = n0 + wn * C::WN + j * 16 + j16;
    if (n >= a.N) continue;
#pragma unroll
    for (int i = 0; i < C::TC; ++i) {
      const int c = c0 + wc * C::WC + i * 16 + 4 * g16;
      if (c >= a.C) continue;
      f32x4_t* p = reinterpret_cast<f32x4_t*>(dst + (long)n * a.C + c);
      *p = add ? *p + acc[i][j] : acc[i][j];
    }
    if (BIAS && wc == 0 && g16 == 0) s.bias[((long)z * s.tilesC + tc) * a.N + n] = sum[j][0];
  }
#endif
}

// Fragments of x in bf16 for many outputs: [c / 16][t / 32] of 1 KB, lane l
// holding channel l % 16 of tokens 8 (l / 16) to + 7, zeros past the last
// token and channel.  A block turns 64 tokens of 128 channels.
constexpr int WIDE_C = 128;
__global__ __launch_bounds__(256) void k_kgrad_turn(KgradArgs a, const uint8_t* q,
                                                    const uint8_t* e, char* frags) {
#if defined(__HIP_DEVICE_COMPILE__)
  constexpr int PX = WIDE_C * 2;
  __shared__ __attribute__((aligned(1024))) char smem[BK * PX];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const long P = (a.C + 31) / 32 * 32, E = keep_exp_pitch(a.C);
  const int c0 = blockIdx.y * WIDE_C;
  const long t0 = (long)blockIdx.x * BK;
  const long blocks32 = (long)gridDim.x * 2;
  const uint32_t sbase = lds_at(smem);
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    const int i = u * 256 + tid, r = i >> 3, k = i & 7, c = c0 + 16 * k;
    uint4 w = uint4{0, 0, 0, 0};
    float step = 0.f;
    if (t0 + r < a.tokens && c < P) {
      w = *reinterpret_cast<const uint4*>(q + (t0 + r) * P + c);
      step = keep_step(e[(t0 + r) * E + (c >> 5)]);
    }
    float v[16];
    unkeep4(v, w.x, step);
    unkeep4(v + 4, w.y, step);
    unkeep4(v + 8, w.z, step);
    unkeep4(v + 12, w.w, step);
    const uint32_t d = sbase + (uint32_t)(r * PX + 16 * slot_of<PX>(2 * k, r));
    ds_wr128<0>(d, pack2(v[0], v[1]), pack2(v[2], v[3]), pack2(v[4], v[5]), pack2(v[6], v[7]));
    ds_wr128<16>(d, pack2(v[8], v[9]), pack2(v[10], v[11]), pack2(v[12], v[13]),
                 pack2(v[14], v[15]));
  }
  lgkm_wait0();
  __syncthreads();
  const int trow = 8 * (lane >> 4) + ((lane & 15) >> 2), tcol = 4 * (lane & 3);
  bf16x8_t f[2][2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int col = (2 * wave + i) * 16 + tcol;
    const uint32_t rx =
        sbase + (uint32_t)(trow * PX + slot_of<PX>(col >> 3, trow) * 16 + (col & 7) * 2);
    const v4s l0 = ds_rdtr<0>(rx), h0 = ds_rdtr<4 * PX>(rx);
    const v4s l1 = ds_rdtr<32 * PX>(rx), h1 = ds_rdtr<36 * PX>(rx);
    f[i][0] = __builtin_bit_cast(bf16x8_t, __builtin_shufflevector(l0, h0, 0, 1, 2, 3, 4, 5, 6, 7));
    f[i][1] = __builtin_bit_cast(bf16x8_t, __builtin_shufflevector(l1, h1, 0, 1, 2, 3, 4, 5, 6, 7));
  }
  lgkm_wait0();
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    tie(f[i][0]);
    tie(f[i][1]);
    char* dst = frags + ((c0 / 16 + 2 * wave + i) * blocks32 + 2 * blockIdx.x) * 1024 + lane * 16;
    *reinterpret_cast<bf16x8_t*>(dst) = f[i][0];
    *reinterpret_cast<bf16x8_t*>(dst + 1024) = f[i][1];
  }
#endif
}

// The gradient from such fragments: 256 outputs x 128 channels per block, eight
// waves of 64 x 64.
template <int BN_, int STAGES_>
struct Wide {
  static constexpr int BN = BN_, BC = WIDE_C, NW = BN / 32, NT = NW * 64, TN = 4, TC = 4;
  static constexpr int WAVES_N = NW / 2;
  static constexpr int PY = BN * 2, Y_BYTES = BK * PY, X_BYTES = BK * BC * 2;
  static constexpr int STAGE = Y_BYTES + X_BYTES, STAGES = STAGES_;
  static constexpr int YU = Y_BYTES / (NT * 16), XU = X_BYTES / (NT * 16), LOADS = YU + XU;
};

template <int OFF>
__device__ __forceinline__ bf16x8_t ds_rd128(uint32_t addr) {
  bf16x8_t v;
  asm volatile("ds_read_b128 %0, %1 offset:%2" : "=v"(v) : "v"(addr), "i"(OFF));
  return v;
}

template <class C, bool BIAS>
__global__ __launch_bounds__(C::NT, 2) void k_kgrad_wide(KgradArgs a, Split s,
                                                         const char* frags) {
#if defined(__HIP_DEVICE_COMPILE__)
  __shared__ __attribute__((aligned(1024))) char smem[C::STAGES * C::STAGE];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wn = wave % C::WAVES_N, wc = wave / C::WAVES_N;
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
  auto fetch = [&](int kt, int stage) __attribute__((always_inline)) {
    char* base = smem + stage * C::STAGE;
    if ((kt + 1) * BK <= len) {
#pragma unroll
      for (int u = 0; u < C::YU; ++u)
        __builtin_amdgcn_global_load_lds(
            ysrc[u], (lds_ptr_t)(base + (u * C::NT + wave * 64) * 16), 16, 0, 0);
    } else {
#pragma unroll
      for (int u = 0; u < C::YU; ++u) {
        const void* g = kt * BK + yrow[u] < len ? static_cast<const void*>(ysrc[u])
                                                : static_cast<const void*>(kgrad_zero);
        __builtin_amdgcn_global_load_lds(g, (lds_ptr_t)(base + (u * C::NT + wave * 64) * 16), 16,
                                         0, 0);
      }
    }
#pragma unroll
    for (int u = 0; u < C::YU; ++u) ysrc[u] += BK * a.dyt;
#pragma unroll
    for (int u = 0; u < C::XU; ++u) {
      __builtin_amdgcn_global_load_lds(
          xsrc[u], (lds_ptr_t)(base + C::Y_BYTES + (u * C::NW + wave) * 1024), 16, 0, 0);
      xsrc[u] += 2 * 1024;
    }
  };

  const int g16 = lane >> 4, j16 = lane & 15;
  const int trow = 8 * g16 + (j16 >> 2), tcol = 4 * (j16 & 3);
  const uint32_t sbase = lds_at(smem);
  const uint32_t rx = sbase + (uint32_t)(C::Y_BYTES + wc * C::TC * 2048 + lane * 16);
  uint32_t ry[C::TN];
#pragma unroll
  for (int j = 0; j < C::TN; ++j) {
    const int col = (wn * C::TN + j) * 16 + tcol;
    ry[j] = sbase +
            (uint32_t)(trow * C::PY + slot_of<C::PY>(col >> 3, trow) * 16 + (col & 7) * 2);
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
  auto read = [&](uint32_t off, auto tag) __attribute__((always_inline)) {
    constexpr int S = decltype(tag)::value;
    fx[S][0] = ds_rd128<S * 1024>(rx + off);
    fx[S][1] = ds_rd128<S * 1024 + 2048>(rx + off);
    fx[S][2] = ds_rd128<S * 1024 + 4096>(rx + off);
    fx[S][3] = ds_rd128<S * 1024 + 6144>(rx + off);
#pragma unroll
    for (int j = 0; j < C::TN; ++j) {
      const v4s lo = ds_rdtr<(S * 32 + 0) * C::PY>(ry[j] + off);
      const v4s hi = ds_rdtr<(S * 32 + 4) * C::PY>(ry[j] + off);
      fy[S][j] =
          __builtin_bit_cast(bf16x8_t, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    }
  };
  auto wait_read = [&](int S) __attribute__((always_inline)) {
    lgkm_wait0();
#pragma unroll
    for (int i = 0; i < C::TC; ++i) tie(fx[S][i]);
#pragma unroll
    for (int j = 0; j < C::TN; ++j) tie(fy[S][j]);
  };
  auto mma = [&](int S) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < C::TC; ++i)
#pragma unroll
      for (int j = 0; j < C::TN; ++j)
        acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fx[S][i], fy[S][j], acc[i][j], 0, 0, 0);
  };
  auto add_bias = [&](int S) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < C::TN; ++j)
      sum[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, fy[S][j], sum[j], 0, 0, 0);
  };
  const std::integral_constant<int, 0> first{};
  const std::integral_constant<int, 1> second{};

  // Step kt computes from stage kt % STAGES: its second half is read while the first
  // half's MFMAs run; then all waves meet, and the first half of kt + 1 is read
  // behind the second half's MFMAs, while kt + STAGES takes this stage's place.
  // Reads end before the step does: no register may move while a read is on its
  // way to it, and the compiler does not know that it is.
#pragma unroll
  for (int i = 0; i < C::STAGES; ++i)
    if (i < KT) fetch(i, i);
  // stage kt is there: at most the later ones are on their way
  auto wait_stage = [&](int kt, int later) __attribute__((always_inline)) {
    if (later > 1 && kt + 2 < KT)
      vm_wait<2 * C::LOADS>();
    else if (later > 0 && kt + 1 < KT)
      vm_wait<C::LOADS>();
    else
      vm_wait<0>();
  };
  wait_stage(0, C::STAGES - 1);
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_sched_barrier(0);
  read(0, first);
  wait_read(0);
  int cur = 0;   // kt % STAGES
  int turn = 0;  // kt % tilesC: the tiles along C share the steps of db
  for (int kt = 0; kt < KT; ++kt) {
    const int next = cur + 1 == C::STAGES ? 0 : cur + 1;
    read((uint32_t)(cur * C::STAGE), second);
    __builtin_amdgcn_sched_barrier(0);
    mma(0);
    __builtin_amdgcn_sched_barrier(0);
    wait_read(1);
    if (BIAS) {
      if (turn == tc && wc == 0) {
        add_bias(0);
        add_bias(1);
      }
      turn = turn + 1 == s.tilesC ? 0 : turn + 1;
    }
    wait_stage(kt + 1, C::STAGES - 2);
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
    if (kt + C::STAGES < KT) fetch(kt + C::STAGES, cur);
    __builtin_amdgcn_sched_barrier(0);
    read((uint32_t)(next * C::STAGE), first);
    __builtin_amdgcn_sched_barrier(0);
    mma(1);
    __builtin_amdgcn_sched_barrier(0);
    wait_read(0);
    cur = next;
  }

  float* dst = s.splits > 1 ? s.part + (long)z * a.N * a.C : a.dw;
  const bool add = s.splits == 1 && a.accumulate;
#pragma unroll
  for (int j = 0; j < C::TN; ++j) {
    const int n = n0 + (wn * C::TN + j) * 16 + j16;
    if (n >= a.N) continue;
#pragma unroll
    for (int i = 0; i < C::TC; ++i) {
      const int c = c0 + wc * 64 + i * 16 + 4 * g16;
      if (c >= a.C) continue;
      f32x4_t* p = reinterpret_cast<f32x4_t*>(dst + (long)n * a.C + c);
      *p = add ? *p + acc[i][j] : acc[i][j];
    }
    if (BIAS && wc == 0 && g16 == 0) s.bias[((long)z * s.tilesC + tc) * a.N + n] = sum[j][0];
  }
#endif
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
  const int bn = p.large ? 128 : 64, bc = p.large ? 128 : 64;
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
  using Small = Tile<64, 64, 32, 32>;
  using W = Wide<128, 2>;
  if (!p.large) {
    auto kern = a.db ? k_kgrad<Small, true> : k_kgrad<Small, false>;
    hipLaunchKernelGGL(kern, dim3(p.s.tiles * p.s.splits), dim3(Small::NT), 0, st, a, p.s, q, e);
    return hipGetLastError();
  }
  char* frags = reinterpret_cast<char*>(a.ws) + p.sums;
  hipLaunchKernelGGL(k_kgrad_turn, dim3((a.tokens + BK - 1) / BK, p.s.tilesC), dim3(256), 0, st, a,
                     q, e, frags);
  const hipError_t err = hipGetLastError();
  if (err != hipSuccess) return err;
  auto kern = a.db ? k_kgrad_wide<W, true> : k_kgrad_wide<W, false>;
  hipLaunchKernelGGL(kern, dim3(p.s.tiles * p.s.splits), dim3(W::NT), 0, st, a, p.s, frags);
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
