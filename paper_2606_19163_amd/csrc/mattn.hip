// Attention under a row mask (gfx950, bf16 MFMA 32x32x16, fp32
// accumulation).  Query row i attends keys lo_i <= j < hi_i:
//   z = scale q k^T, capped: z = cap tanh(z / cap), then - slope |pos_i - j|
//   p = softmax over the attended keys, o = p v, lse = log sum exp z
// backward: p from z and lse; D = rowsum(do o), dp = do v^T,
//   ds = p (dp - D) (1 - tanh^2) scale, dq = ds k, dk = ds^T q, dv = p^T do.
// dq has a kernel over query rows, dk and dv one over keys, each of which
// computes z and dp again, so that nothing is accumulated across blocks.
// Scores are kept in the log2 domain (z log2 e).
//
// The four waves of a block are G groups of 32 rows (or keys) by 4 / G shares
// of the other side, which streams through LDS in tiles of 64, and a wave
// works on 32 x 32 scores at a time.  For o and dq it computes
//   s^T = k q^T    A = k rows (LDS), B = q (registers)
//   o^T += v^T p^T A = v read down the tile, B = p^T
// and for dk and dv the same with the sides exchanged, so that p and ds stay
// in registers: lane (n, hl) of the MFMA's output holds rows
// 8 (i / 4) + 4 hl + i % 4 of column n (i < 16) and its B operand wants rows
// 8 hl + t of 16 (t < 8), which is the same set if row r of the first product
// is row swap23(r) of the tile (bits 2 and 3 exchanged): element i then is
// row 16 (i / 8) + 8 hl + i % 8.
//
// A row that does not attend a key must not be reached by it even when it
// holds a NaN or an infinity, which the product's zero weight does not ensure
// (0 NaN = NaN).  In a tile that some row attends only in part, such values
// are cleared in the operand that is summed over, and the rows that do attend
// them get them at the end.
//
// p and ds are rounded to bf16, as operands of the products that they enter; in
// fp32 those would run at a sixteenth of the matrix units' bf16 rate.  With it
// outputs and gradients are 0.0023 to 0.0024 (relative L2) off the float64 ones;
// in fp32 throughout, rounded once at the end, they are 0.0017 off.
#include <type_traits>

#include "common.hpp"
#include "okernels.hpp"

namespace pulse {
namespace {

typedef __attribute__((__vector_size__(8 * sizeof(__bf16)))) __bf16 bf16x8;
typedef __attribute__((__vector_size__(4 * sizeof(float)))) float f32x4;
typedef __attribute__((__vector_size__(16 * sizeof(float)))) float f32x16;
typedef short v4s __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) v4s lds_v4s;

constexpr int KT = 64;  // keys (or rows) per streamed tile
constexpr float LOG2E = 1.44269504088896341f;
constexpr float LN2 = 0.693147180559945309f;
constexpr float LOWEST = -3.0e38f;  // finite: below every finite score
// Forward: a row's reference moves up to its maximum only when a score passes
// it by more than GROW (log2 units), decided for the whole wave, so that most
// steps skip the rescaling; weights stay below 2^GROW.
constexpr float GROW = 8.f;

struct Dev {  // device view of MattnArgs
  int Tq, Tk, H, rep, hd8;
  float c1, c2;  // no cap: scale log2e; cap: scale / cap and cap log2e
  float inv_c1;  // no cap, over keys
  float scale, cap;
  const uint16_t *q, *k, *v, *dout, *o_in;
  uint16_t *o, *dq, *dk, *dv;
  long qt, qh, kt, kh, vt, vh, ot, oh, dot, doh, dqt, dqh, dkt, dkh, dvt, dvh;
  const pulse_mask_row* rows;
  const MaskTile* tiles;
  const float* slopes;
  float* lse;
  uint16_t* o_low;  // [Tq][H][8 hd8] or null
  float* dsum;
  // Work split further than rows and heads: `parts` blocks share a tile, each
  // with a range of the other side (or some of the group's heads) and fp32
  // results of its own, [parts][rows][heads][8 hd8], which a second kernel
  // adds up.
  int parts, head_parts;  // head_parts of them by the group's heads (dk, dv),
  int head_per;           // of so many heads each, the last of what is left
  float *part0, *part1, *part_lse;
};

// The value is opaque: knowing its range, the compiler splits every LDS
// address into parts that it keeps in registers across the loops, and spills.
__device__ __forceinline__ int tid() {
  int t = threadIdx.x;
  asm("" : "+v"(t));
  return t;
}

__device__ __forceinline__ f32x16 mma(bf16x8 a, bf16x8 b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
// 2^x as one v_exp_f32: results below 2^-126 flush to zero
__device__ __forceinline__ float ex2(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ f32x16 splat(float x) {
  f32x16 v;
#pragma unroll
  for (int i = 0; i < 16; ++i) v[i] = x;
  return v;
}
__device__ __forceinline__ int swap23(int r) { return (r & ~12) | ((r & 4) << 1) | ((r & 8) >> 1); }
// offset of element i of an output column from its first row (8 hl)
__device__ __forceinline__ constexpr int elem(int i) { return 16 * (i / 8) + i % 8; }

// Tiles are [rows][D] with the 16-byte chunks of a row permuted (chunk c of
// row r at c ^ mix(r)), so that the rows that one LDS access reads fall on
// distinct banks: {0-3, 8-11} (+4, +16) of one chunk (rows32), {0-3} of two
// (cols32).
template <int D>
__device__ __forceinline__ int mix(int r) {
  return D == 64 ? ((((r >> 1) & 1) << 1) | ((r >> 2) & 1) | (((r >> 3) & 1) << 2))
       : D == 96 ? ((r >> 2) & 3)
                 : ((r & 3) << 1) | ((r >> 2) & 1) | (((r >> 3) & 1) << 3);
}
template <int D>
__device__ __forceinline__ int toff(int r, int c) {  // in elements
  return r * D + ((c ^ mix<D>(r)) << 3);
}

// operand of 8 consecutive channels straight from memory (0 where absent)
__device__ __forceinline__ bf16x8 row_frag(const uint16_t* p, int c, bool ok, int hd8) {
  uint4 v{0, 0, 0, 0};
  if (ok && c < hd8) v = *reinterpret_cast<const uint4*>(p + c * 8);
  return __builtin_bit_cast(bf16x8, v);
}

// Fragment addresses are a lane's byte offset in the tile, changed by an xor
// of a constant (the channels) and a constant offset (the rows): few registers
// hold them all.

// A operand of rows: lane (n, hl) gets channels 16 kk + 8 hl .. + 7 of row
// swap23(n) (+ rows in `at`)
template <int D>
__device__ __forceinline__ int rows_base(int lane) {
  const int r = swap23(lane & 31);
  return r * 2 * D + (((lane >> 5) ^ mix<D>(r)) << 4);
}
template <int D>
__device__ __forceinline__ bf16x8 rows32(const char* tile, int base, int kk, int at) {
  const int x = D == 96 ? (base ^ ((kk & 1) << 5)) + 64 * (kk >> 1) : base ^ (kk << 5);
  return *reinterpret_cast<const bf16x8*>(tile + x + at);
}

// A operand read down the tile: lane (n, hl) gets rows 8 hl .. + 7 (+ rows in
// `at`) of channel 32 d + n.  ds_read_b64_tr_b16: within 16 lanes, lane j
// receives element j % 4 of the rows addressed by lanes 4 t + j / 4
// (t = 0..3).
template <int D>
__device__ __forceinline__ int cols_base(int lane) {
  const int j = lane & 15, r = 8 * (lane >> 5) + (j >> 2);
  const int c = 2 * ((lane >> 4) & 1) + ((j & 3) >> 1);
  return r * 2 * D + ((c ^ mix<D>(r)) << 4) + 8 * (j & 1);
}
template <int D>
__device__ __forceinline__ bf16x8 cols32(const char* tile, int base, int d, int at) {
  const int x = D == 96 ? base + 64 * d : base ^ (d << 6);
  const v4s lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s*)(tile + x + at));
  // rows + 4: one bit of their chunks' permutation changes
  const v4s hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s*)(tile + (x ^ 16) + at + 8 * D));
  return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
}

__device__ __forceinline__ bool odd_lo(uint32_t x) { return (x & 0x7f80u) == 0x7f80u; }
__device__ __forceinline__ bool odd_hi(uint32_t x) { return (x & 0x7f800000u) == 0x7f800000u; }

// NaN and infinities among 8 values become 0, or with MAX infinities the
// largest finite value of their sign; whether there were any
template <bool MAX>
__device__ __forceinline__ bool clean8(uint4& w) {
  uint32_t x[4] = {w.x, w.y, w.z, w.w};
  bool odd = false;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const bool lo = odd_lo(x[i]), hi = odd_hi(x[i]);
    if (MAX) {  // the value below an infinity, as an integer
      if ((x[i] & 0x7fffu) == 0x7f80u) x[i] -= 1u;
      if ((x[i] & 0x7fff0000u) == 0x7f800000u) x[i] -= 0x10000u;
    }
    const bool l0 = odd_lo(x[i]), h0 = odd_hi(x[i]);
    x[i] &= (l0 ? 0xffff0000u : ~0u) & (h0 ? 0xffffu : ~0u);
    odd |= lo | hi;
  }
  w = uint4{x[0], x[1], x[2], x[3]};
  return odd;
}

// whether there are any: the largest magnitude, as integers
__device__ __forceinline__ bool odd8(uint4 w) {
  typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
  const uint32_t x[4] = {w.x, w.y, w.z, w.w};
  u16x2 m = {0, 0};
#pragma unroll
  for (int i = 0; i < 4; ++i)
    m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, x[i] & 0x7fff7fffu));
  return m[0] >= 0x7f80 || m[1] >= 0x7f80;
}

// o += those of 8 values that are NaN or infinite (a weight p > 0 leaves them
// what they are); with `nan` they make it NaN
__device__ __forceinline__ void add_odd(float (&o)[8], uint4 w, bool nan) {
  const uint32_t x[4] = {w.x, w.y, w.z, w.w};
  const float q = __uint_as_float(0x7fc00000u);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (odd_lo(x[i])) o[2 * i] += nan ? q : __uint_as_float(x[i] << 16);
    if (odd_hi(x[i])) o[2 * i + 1] += nan ? q : __uint_as_float(x[i] & 0xffff0000u);
  }
}

// Whether nothing added to them can change 8 sums any more
__device__ __forceinline__ bool all_nan(const float (&o)[8]) {
  bool n = true;
#pragma unroll
  for (int i = 0; i < 8; ++i) n &= o[i] != o[i];
  return n;
}

// The tiles of keys (or rows) [lo, hi) that a block has left values out of: one
// bit for every 2^shift tiles, so that 2048 bits hold the tiles of `all` keys.
// What is added at the end is looked for in these only, so that one NaN costs
// a tile and not all of them.  It lies in LDS with its range, of which the
// loops then hold nothing: registers spent on it cost dq 6 % (8192 tokens of 16
// heads, D = 64: 496 us instead of 465).
struct Left {
  uint32_t w[64];
  int lo, hi, any;
  __device__ static __forceinline__ int shift(int all) { return max(15 - __builtin_clz(all), 0); }
  // before the barrier that precedes the first mark
  __device__ __forceinline__ void init(int t, int first, int end) {
    if (t < 64) w[t] = 0;
    if (t == 0) lo = first, hi = end, any = 0;
  }
  // some of tile t, counted from lo
  __device__ __forceinline__ void mark(int t, int all) {
    t >>= shift(all);
    atomicOr(&w[t >> 5], 1u << (t & 31));
    any = 1;
  }
  // f(first, end) of the marked tiles, until it returns false
  template <typename F>
  __device__ __forceinline__ void each(int all, F f) const {
    const int n = KT << shift(all);
    for (int i = 0; i < 64; ++i)
      for (uint32_t x = w[i]; x; x &= x - 1) {
        const int at = lo + (32 * i + __builtin_ctz(x)) * n;
        if (!f(at, min(at + n, hi))) return;
      }
  }
};

// x, or NaN where x is not finite
__device__ __forceinline__ float finite_or_nan(float x) {
  const uint32_t b = __float_as_uint(x);
  return __uint_as_float((b & 0x7f800000u) == 0x7f800000u ? 0x7fc00000u : b);
}

// A thread's 16-byte chunks of a [KT][D] tile of a strided tensor, in
// registers on their way from memory to LDS.  The chunks are whole rows apart
// (D = 64, 128) or columns apart (96), so that one address serves them all.
template <int D>
struct Stage {
  static constexpr int N = KT * D / 8 / 256;
  static constexpr int ROUND = D == 96 ? 4 : D / 8;  // chunks of a row in one round
  static constexpr int RR = 256 / ROUND;             // rows in one round
  static_assert(N * 256 == KT * D / 8 && (D == 96 ? KT == RR : KT % RR == 0), "whole rounds");
  uint4 v[N];
  const uint16_t* p;
  long stride;
  int r, c;
  __device__ __forceinline__ void init(const uint16_t* src, long row, long st) {
    r = tid() / ROUND;
    c = tid() % ROUND;
    stride = st;
    p = src + (row + r) * st + 8 * c;
#pragma unroll
    for (int u = 0; u < N; ++u) v[u] = uint4{0, 0, 0, 0};
  }
  // the tile at p, of which `valid` >= 1 rows exist: the last one stands in
  // for those past it (no row attends them).  Channels past hd8 stay 0.
  __device__ __forceinline__ void load(int valid, int hd8) {
    if constexpr (D == 96) {
      const uint16_t* q = r < valid ? p : p + (valid - 1 - r) * stride;
#pragma unroll
      for (int u = 0; u < N; ++u)
        if (c + 4 * u < hd8) v[u] = *reinterpret_cast<const uint4*>(q + 32 * u);
    } else if (c < hd8) {
      if (valid >= KT) {
#pragma unroll
        for (int u = 0; u < N; ++u) v[u] = *reinterpret_cast<const uint4*>(p + RR * u * stride);
      } else {
#pragma unroll
        for (int u = 0; u < N; ++u)
          v[u] = *reinterpret_cast<const uint4*>(p + (min(r + RR * u, valid - 1) - r) * stride);
      }
    }
  }
  __device__ __forceinline__ void next() { p += KT * stride; }
  __device__ __forceinline__ void store(uint16_t* t) const {
#pragma unroll
    for (int u = 0; u < N; ++u)
      *reinterpret_cast<uint4*>(
          t + (D == 96 ? toff<D>(r, c + 4 * u) : toff<D>(r + RR * u, c))) = v[u];
  }
  // NaN and infinities become 0 (MAX: see clean8); whether there were any.
  // bad[row] = tag for the rows that held one.
  template <bool MAX = false>
  __device__ __forceinline__ bool clean(int* bad = nullptr, int tag = 0) {
    bool any = false;
#pragma unroll
    for (int u = 0; u < N; ++u) any |= odd8(v[u]);
    if (!__any(any)) return false;
    any = false;
#pragma unroll
    for (int u = 0; u < N; ++u) {
      const bool b = clean8<MAX>(v[u]);
      any |= b;
      if (bad && b) bad[D == 96 ? r : r + RR * u] = tag;
    }
    return any;
  }
};

// Between an MFMA and the VALU work that it covers: the scheduler, left to
// itself, puts every MFMA before the VALU work that does not depend on it.  LDS
// reads and scalar work may pass.  Backward of 8 x 1024 tokens of 16 heads of
// 88: 235 us without, 220 us with; at 64 channels, where three waves share a
// SIMD, 1062 and 1091 us (8192 tokens of 16 heads), so not there.
template <int D>
__device__ __forceinline__ void in_order() {
  if constexpr (D > 64) __builtin_amdgcn_sched_barrier(0x104);
}

// Scores.  t = z - ref from a raw product, all in the log2 domain.
//
// LOW: tanh(x) = 1 - 2 r with r = 1 / (1 + e^(2x)), so that 1 - tanh^2 =
// 4 r (1 - r); e^(2x) may overflow to inf: r = 0.  Near 0 it is a difference
// of numbers near 1, which leaves an error of 1.5e-7 cap whatever the score:
// up to caps of CAP_LOW that is less than 2e-5.  ANY: beyond, scores of |x| <
// 1/4 come from the series of tanh, whose error there is 1e-8 of the score
// (8192 tokens of 16 heads, D = 64, forward and backward: 751 and 2161 us, LOW
// 476 and 1506).
enum Cap { NONE, LOW, ANY };
constexpr float CAP_LOW = 128.f;

template <int CAP, bool BIAS>
struct Score {
  float k;   // of the raw product: scale log2e; capped: scale / cap 2 log2e
  float c2;  // cap log2e
  float c1;  // ANY: scale / cap
  float kz;  // ANY: scale log2e
  float sl;  // slope log2e
  __device__ __forceinline__ Score(const Dev& a, int h) {
    k = CAP ? a.c1 * (2.f * LOG2E) : a.c1;
    c2 = a.c2;
    c1 = a.c1;
    kz = a.scale * LOG2E;
    sl = BIAS ? a.slopes[h] * LOG2E : 0.f;
  }
  // far: the signed distance |pos - j|; dz receives d z / d (scale q.k)
  __device__ __forceinline__ float operator()(float raw, float ref, float far, float& dz) const {
    float t;
    if (CAP) {
      const float r = __builtin_amdgcn_rcpf(1.f + ex2(raw * k));
      dz = 4.f * r * (1.f - r);
      t = fmaf(-2.f * c2, r, c2 - ref);
      if (CAP == ANY) {
        const float x = raw * c1, y = x * x;
        // tanh(x) / x
        float g = fmaf(y, 62.f / 2835.f, -17.f / 315.f);
        g = fmaf(y, fmaf(y, fmaf(y, g, 2.f / 15.f), -1.f / 3.f), 1.f);
        const bool near = y < 0.0625f;
        dz = near ? fmaf(-y, g * g, 1.f) : dz;
        t = near ? fmaf(raw * kz, g, -ref) : t;
      }
    } else {
      dz = 1.f;
      t = fmaf(raw, k, -ref);
    }
    return BIAS ? fmaf(-sl, fabsf(far), t) : t;
  }
};

// A mask in memory may hold anything (one that was never built, rows written
// since).  Rows are compared with and are left as they are: cutting them waits
// for their load, which the kernel over keys has in flight across a tile (1 x
// 4096 tokens of 12 heads: 199 us instead of 165).  What becomes an address is
// cut to the keys: tiles_at, and the walks over a row's keys.
struct Row {
  int lo, hi, pos;
};
__device__ __forceinline__ Row row_at(const Dev& a, int i) {
  if (i >= a.Tq) return Row{0, 0, 0};
  const pulse_mask_row r = a.rows[i];
  return Row{r.lo, r.hi, r.pos};
}

// Bit e of the result: key k + e is attended, for e in 0..31.
__device__ __forceinline__ uint32_t attended(const Row& r, int k) {
  const int lo = min(max(r.lo - k, 0), 32), hi = min(max(r.hi - k, 0), 32);
  const uint32_t below = (uint32_t)((uint64_t{1} << hi) - 1);
  return below & ~(uint32_t)((uint64_t{1} << lo) - 1);
}
// all ones if bit e of m is set, else 0
__device__ __forceinline__ uint32_t bit(uint32_t m, int e) {
  return (uint32_t)((int32_t)(m << (31 - e)) >> 31);
}
__device__ __forceinline__ float keep_or(uint32_t on, float x, uint32_t other) {
  return __uint_as_float((__float_as_uint(x) & on) | (other & ~on));
}
constexpr uint32_t NEG_INF = 0xff800000u;
constexpr int PAST = 1 << 30;  // lo of a row past the last

// mask entry of rows [r0, r0 + n), n a multiple of the table's tile, its keys
// within [0, Tk)
__device__ __forceinline__ MaskTile tiles_at(const Dev& a, int r0, int n) {
  MaskTile b{1 << 30, 0, 0, 1 << 30};
  for (int r = r0; r < r0 + n && r < a.Tq; r += MASK_TILE) {
    const MaskTile t = a.tiles[r / MASK_TILE];
    if (t.hi > t.lo) b.lo = min(b.lo, t.lo), b.hi = max(b.hi, t.hi);
    b.all_lo = max(b.all_lo, t.all_lo);
    b.all_hi = min(b.all_hi, t.all_hi);
  }
  b.lo = max(b.lo, 0);
  b.hi = min(b.hi, a.Tk);
  return b;
}

// (tile, head) of this block.  Blocks go round-robin over the 8 XCDs; each
// XCD takes a contiguous range of the head-major order, so that a head's
// tensors are fetched into one L2.  Tiles run from the last, which under a
// causal mask has the most keys (first from the first, for the kernel over
// keys).
__device__ __forceinline__ void block_of(const Dev& a, int tiles, int heads, bool last, int& tile,
                                         int& head, int& part) {
  const int nb = tiles * heads * a.parts, bid = blockIdx.x;
  const int q = nb >> 3, r = nb & 7, x = bid & 7;
  const int lb = x * q + (x < r ? x : r) + (bid >> 3);
  const int hp = lb / tiles;
  tile = lb - hp * tiles;
  if (last) tile = tiles - 1 - tile;
  head = hp / a.parts;
  part = hp - head * a.parts;
}

// this part's share of keys [lo, hi), whole tiles
__device__ __forceinline__ void share(const Dev& a, int part, int& lo, int& hi) {
  if (a.parts == 1 || hi <= lo) return;
  const int n = ((hi - lo + a.parts - 1) / a.parts + KT - 1) / KT * KT;
  lo += part * n;
  hi = min(hi, lo + n);
}

constexpr int MP = 36;                  // row pitch of a merge buffer (floats)
constexpr int MERGE = 4 * 32 * MP * 4;  // its bytes

// 8 values rounded to bf16, and what that leaves out, rounded
__device__ __forceinline__ uint4 rounded(const float (&o)[8]) {
  return uint4{pack2(o[0], o[1]), pack2(o[2], o[3]), pack2(o[4], o[5]), pack2(o[6], o[7])};
}
__device__ __forceinline__ uint4 left_out(const float (&o)[8]) {
  float r[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) r[i] = o[i] - bf2f(f2bf(o[i]));
  return rounded(r);
}

// Write the waves' column accumulators [channels][32 columns], times f, to
// rows row0 + .. of out (or of the part's fp32 results), and to `low` what the
// rounding leaves out: 32 channels at a time meet in LDS, where the shares of
// a group are added in order.  fix(row, chunk, o) may change 8 channels before
// they are rounded.
template <int D, int G, typename F>
__device__ __forceinline__ void write_rows(float* buf, const f32x16 (&acc)[D / 32], float f,
                                           uint16_t* out, long stride, float* part,
                                           uint16_t* low, int row0, int rows, int heads, int hd8,
                                           F fix) {
  constexpr int SH = 4 / G;
  const int lane = tid() & 63, w = tid() >> 6, n = lane & 31, hl = lane >> 5;
#pragma unroll
  for (int d = 0; d < D / 32; ++d) {
    __syncthreads();
#pragma unroll
    for (int x = 0; x < 4; ++x)
      *reinterpret_cast<f32x4*>(buf + (w * 32 + n) * MP + 8 * x + 4 * hl) =
          f32x4{acc[d][4 * x] * f, acc[d][4 * x + 1] * f, acc[d][4 * x + 2] * f,
                acc[d][4 * x + 3] * f};
    __syncthreads();
    for (int e = tid(); e < G * 128; e += 256) {
      const int rb = e >> 2, c = e & 3, row = row0 + rb;
      float o[8] = {};
#pragma unroll
      for (int i = 0; i < SH; ++i) {
        const float* s = buf + (((rb >> 5) * SH + i) * 32 + (rb & 31)) * MP + 8 * c;
#pragma unroll
        for (int t = 0; t < 8; ++t) o[t] += s[t];
      }
      if (row >= rows || 4 * d + c >= hd8) continue;
      fix(row, 4 * d + c, o);
      if (part) {
        float4* q = reinterpret_cast<float4*>(part + ((long)row * heads * hd8 + 4 * d + c) * 8);
        q[0] = make_float4(o[0], o[1], o[2], o[3]);
        q[1] = make_float4(o[4], o[5], o[6], o[7]);
        continue;
      }
      *reinterpret_cast<uint4*>(out + row * stride + 32 * d + 8 * c) = rounded(o);
      if (low)
        *reinterpret_cast<uint4*>(low + ((long)row * heads * hd8 + 4 * d + c) * 8) = left_out(o);
    }
  }
}

// the part's fp32 results of a head, or null where there is one part
__device__ __forceinline__ float* part_of(const Dev& a, float* p, int part, int rows, int heads,
                                          int head) {
  return a.parts > 1 ? p + (((long)part * rows) * heads + head) * a.hd8 * 8 : nullptr;
}

constexpr int max_of(int a, int b) { return a > b ? a : b; }
// two stages of two tiles, later the merge buffer
template <int D>
constexpr int SMEM = max_of(4 * KT * D * 2, MERGE);

// ---------------------------------------------------------------------------
// Forward: o^T += v^T p^T with the running reference and sum of a row in the
// lane that holds its column, so that a step's only exchange between lanes is
// the vote on the reference.
// Bound by the vector units and the matrix units in turn, which overlap little
// within a wave: a 32 x 32 step of D = 64 is 112 quarter-cycles of vector work
// (exponential, scale and subtract, sum, maximum, rounding: 16 scores a lane)
// and 64 of MFMA, of 160 in all.  8192 tokens of 16 heads: D = 64 330 us (833
// TFLOP/s), D = 128 565 us (973 TFLOP/s).  64 rows per wave instead of 32 run
// at one wave per SIMD and were slower (D = 128: 637 TFLOP/s), 8 waves per block
// too (16 x 256 tokens of 12 heads: 16.8 us instead of 13.1).
// ---------------------------------------------------------------------------
template <int D, int G, int WPE, int CAP, bool BIAS>
__global__ __launch_bounds__(256, WPE) void k_mattn_fwd(Dev a) {
  constexpr int SH = 4 / G, RB = 32 * G, TILE = KT * D;
  __shared__ __attribute__((aligned(16))) char smem[SMEM<D>];
  __shared__ float ml[4][2][32];
  __shared__ Left left;
  int tile, h, part;
  block_of(a, (a.Tq + RB - 1) / RB, a.H, true, tile, h, part);
  const int kh = h / a.rep;
  const int lane = tid() & 63, w = tid() >> 6, n = lane & 31, hl = lane >> 5;
  const int grp = w / SH, shr = w % SH;
  const int rbase = rows_base<D>(lane) + shr * 64 * D, cbase = cols_base<D>(lane) + shr * 64 * D;
  const int qrow = tile * RB + grp * 32 + n;
  const MaskTile bt = tiles_at(a, tile * RB, RB);
  int klo = bt.lo, khi = bt.hi;
  share(a, part, klo, khi);
  const uint16_t* vbase = a.v + kh * a.vh;
  Stage<D> sk, sv;
  sk.init(a.k + kh * a.kh, klo, a.kt);
  sv.init(vbase, klo, a.vt);
  if (klo < khi) {
    sk.load(a.Tk - klo, a.hd8);
    sv.load(a.Tk - klo, a.hd8);
  }
  left.init(tid(), klo, khi);
  Score<CAP, BIAS> score(a, h);
  // q carries the sign of the scale.  With the sign in the scale D = 64 needs
  // 131 registers instead of 128, three waves per SIMD instead of four: 8192
  // tokens of 16 heads 367 us, 347 so.
  const bool neg = score.k < 0.f;
  score.k = fabsf(score.k);
  score.kz = fabsf(score.kz);
  const Row rw = row_at(a, qrow);
  const bool past = qrow >= a.Tq;  // nothing of such a row is kept
  bf16x8 qf[D / 16];
#pragma unroll
  for (int kk = 0; kk < D / 16; ++kk) {
    qf[kk] = row_frag(a.q + qrow * a.qt + h * a.qh, 2 * kk + hl, qrow < a.Tq, a.hd8);
    if (neg) qf[kk] = -qf[kk];
  }
  float ref = 0.f, l = 0.f;  // l == 0: no reference yet
  f32x16 acc[D / 32];
#pragma unroll
  for (int d = 0; d < D / 32; ++d) acc[d] = splat(0.f);
  __syncthreads();  // left

  int it = 0;
  for (int k0 = klo; k0 < khi; k0 += KT, ++it) {
    const int stage = (it & 1) * 4 * TILE;  // bytes
    uint16_t* Ks = reinterpret_cast<uint16_t*>(smem + stage);
    // this stage was last read two tiles ago, before the previous barrier
    if ((bt.all_lo > k0 || bt.all_hi < k0 + KT) && sv.clean()) left.mark(it, a.Tk);
    sk.store(Ks);
    sv.store(Ks + TILE);
    __syncthreads();
    if (k0 + KT < khi) {
      sk.next();
      sv.next();
      sk.load(a.Tk - k0 - KT, a.hd8);
      sv.load(a.Tk - k0 - KT, a.hd8);
    }
    // 32-key steps, NU of them taken together where two waves share a SIMD and
    // a step has MFMAs enough to cover the exponentials of another: against one
    // at a time, 8192 tokens of 16 heads of 128 take 6 % less, of 64 4 % more,
    // and 8 x 1024 tokens of 88 6 % more
    constexpr int NU = D == 128 ? 2 / SH : 1;
#pragma unroll
    for (int y = 0; y < 2 / SH / NU; ++y) {
      const int kb = k0 + 32 * (shr + SH * y);  // the first key
      const int at = 64 * D * SH * y;
      if (!__any(rw.lo < kb + 32 * NU && rw.hi > kb)) continue;
      f32x16 s[NU];
#pragma unroll
      for (int u = 0; u < NU; ++u) {
        s[u] = splat(0.f);
#pragma unroll
        for (int kk = 0; kk < D / 16; ++kk)
          s[u] = mma(rows32<D>(smem, rbase + stage, kk, at + 64 * D * u), qf[kk], s[u]);
      }
      const float far = (float)(rw.pos - kb - 8 * hl);
#pragma unroll
      for (int u = 0; u < NU; ++u)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          float dz;
          s[u][i] = score(s[u][i], ref, far - (float)(32 * u + elem(i)), dz);
        }
      if (!__all(past || (rw.lo <= kb && rw.hi >= kb + 32 * NU))) {
#pragma unroll
        for (int u = 0; u < NU; ++u) {
          const uint32_t on = attended(rw, kb + 32 * u + 8 * hl);
#pragma unroll
          for (int i = 0; i < 16; ++i) s[u][i] = keep_or(bit(on, elem(i)), s[u][i], NEG_INF);
        }
      }
      float mx = s[0][0];
#pragma unroll
      for (int u = 0; u < NU; ++u)
#pragma unroll
        for (int i = 0; i < 16; ++i) mx = fmaxf(mx, s[u][i]);
      if (__any(mx > (l == 0.f ? LOWEST : GROW))) {
        // relative to the old reference; the first may lie below it
        mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
        const bool first = l + __shfl_xor(l, 32, 64) == 0.f;
        const float up = mx > LOWEST && (first || mx > 0.f) ? mx : 0.f;
        const float al = first ? 0.f : ex2(-up);
        ref += up;
        l *= al;
#pragma unroll
        for (int u = 0; u < NU; ++u)
#pragma unroll
          for (int i = 0; i < 16; ++i) s[u][i] -= up;
#pragma unroll
        for (int d = 0; d < D / 32; ++d)
#pragma unroll
          for (int i = 0; i < 16; ++i) acc[d][i] *= al;
      }
#pragma unroll
      for (int u = 0; u < NU; ++u) {
        bf16x8 p[2];
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const float e = ex2(s[u][i]);
          l += e;
          p[i / 8][i % 8] = (__bf16)e;
        }
#pragma unroll
        for (int d = 0; d < D / 32; ++d)
#pragma unroll
          for (int ks = 0; ks < 2; ++ks)
            acc[d] = mma(
                cols32<D>(smem, cbase + stage, d, at + 64 * D * u + 32 * D * ks + 2 * TILE), p[ks],
                acc[d]);
      }
    }
  }

  // merge: R = max ref, l = sum l 2^(ref - R), o = sum o 2^(ref - R) / l
  l += __shfl_xor(l, 32, 64);
  if (l == 0.f) ref = LOWEST;
  if (hl == 0) {
    ml[w][0][n] = ref;
    ml[w][1][n] = l;
  }
  __syncthreads();  // also: every wave is done with the tiles
  float R = ref, t = 0.f;
#pragma unroll
  for (int i = 0; i < SH; ++i) R = fmaxf(R, ml[grp * SH + i][0][n]);
#pragma unroll
  for (int i = 0; i < SH; ++i) t += ml[grp * SH + i][1][n] * ex2(ml[grp * SH + i][0][n] - R);
  const bool empty = rw.hi <= rw.lo;
  float* po = part_of(a, a.part0, part, a.Tq, a.H, h);
  // a part in which the row attends nothing has no weight
  const bool none = empty || (po && t == 0.f);
  if (shr == 0 && hl == 0 && qrow < a.Tq) {
    const float e = none ? -INFINITY : R + __builtin_amdgcn_logf(t);
    if (po)
      a.part_lse[((long)part * a.H + h) * a.Tq + qrow] = e;
    else
      a.lse[(long)h * a.Tq + qrow] = e * LN2;
  }
  // an empty row's accumulators are 0
  write_rows<D, G>(reinterpret_cast<float*>(smem), acc, none ? 0.f : ex2(ref - R) / t,
                   a.o + h * a.oh, a.ot, po, a.o_low ? a.o_low + (long)h * a.hd8 * 8 : nullptr,
                   tile * RB, a.Tq, a.H, a.hd8,
                   [&](int row, int c, float (&o)[8]) {
                     if (!left.any) return;
                     const Row x = row_at(a, row);
                     left.each(a.Tk, [&](int first, int end) {
                       for (int j = max(x.lo, first); j < min(x.hi, end); ++j)
                         add_odd(o, *reinterpret_cast<const uint4*>(vbase + j * a.vt + 8 * c),
                                 false);
                       return !all_nan(o);
                     });
                   });
}

// ---------------------------------------------------------------------------
// Backward over query rows: D = rowsum(do o), dq = ds k.  Three products a
// step; a row's lse and D sit in the lane of its column, and -D starts the sum
// of dp.  Bound as the forward is: about 1000 TFLOP/s over its three products
// at 8192 tokens of 16 heads.
// ---------------------------------------------------------------------------
template <int D, int G, int WPE, int CAP, bool BIAS>
__global__ __launch_bounds__(256, WPE) void k_mattn_bwd_q(Dev a) {
  constexpr int SH = 4 / G, RB = 32 * G, TILE = KT * D;
  __shared__ __attribute__((aligned(16))) char smem[SMEM<D>];
  __shared__ int bad[2][KT];  // tile in which a key held a NaN or infinity
  __shared__ int odd_at[2];
  __shared__ Left left;
  int tile, h, part;
  block_of(a, (a.Tq + RB - 1) / RB, a.H, true, tile, h, part);
  const int kh = h / a.rep;
  const int lane = tid() & 63, w = tid() >> 6, n = lane & 31, hl = lane >> 5;
  const int grp = w / SH, shr = w % SH;
  const int rbase = rows_base<D>(lane) + shr * 64 * D, cbase = cols_base<D>(lane) + shr * 64 * D;
  const int qrow = tile * RB + grp * 32 + n;
  const MaskTile bt = tiles_at(a, tile * RB, RB);
  int klo = bt.lo, khi = bt.hi;
  share(a, part, klo, khi);
  const uint16_t* kbase = a.k + kh * a.kh;
  Stage<D> sk, sv;
  sk.init(kbase, klo, a.kt);
  sv.init(a.v + kh * a.vh, klo, a.vt);
  if (klo < khi) {
    sk.load(a.Tk - klo, a.hd8);
    sv.load(a.Tk - klo, a.hd8);
  }
  if (tid() < 2 * KT) bad[tid() / KT][tid() % KT] = -1;
  if (tid() < 2) odd_at[tid()] = -1;
  left.init(tid(), klo, khi);
  const Score<CAP, BIAS> score(a, h);
  const Row rw = row_at(a, qrow);
  const bool past = qrow >= a.Tq;  // nothing of such a row is kept
  const bool in = qrow < a.Tq;
  bf16x8 qf[D / 16], df[D / 16];
  float Dq = 0.f;
#pragma unroll
  for (int kk = 0; kk < D / 16; ++kk) {
    qf[kk] = row_frag(a.q + qrow * a.qt + h * a.qh, 2 * kk + hl, in, a.hd8);
    df[kk] = row_frag(a.dout + qrow * a.dot + h * a.doh, 2 * kk + hl, in, a.hd8);
    const bf16x8 ov = row_frag(a.o_in + qrow * a.ot + h * a.oh, 2 * kk + hl, in, a.hd8);
    // with what o's rounding left out: D is a difference's second term
    const bf16x8 ol = row_frag(a.o_low + ((long)qrow * a.H + h) * a.hd8 * 8, 2 * kk + hl,
                               in && a.o_low, a.hd8);
#pragma unroll
    for (int t = 0; t < 8; ++t) Dq += (float)df[kk][t] * ((float)ov[t] + (float)ol[t]);
  }
  Dq += __shfl_xor(Dq, 32, 64);
  float l2 = 0.f;
  if (in) {
    if (part == 0 && shr == 0 && hl == 0) a.dsum[(long)h * a.Tq + qrow] = Dq;
    // of a row that attends something: no score of it makes a p then
    l2 = finite_or_nan(a.lse[(long)h * a.Tq + qrow]) * LOG2E;
  }
  f32x16 acc[D / 32];
#pragma unroll
  for (int d = 0; d < D / 32; ++d) acc[d] = splat(0.f);
  __syncthreads();  // bad, left

  int it = 0;
  for (int k0 = klo; k0 < khi; k0 += KT, ++it) {
    const int stage = (it & 1) * 4 * TILE;
    uint16_t* Ks = reinterpret_cast<uint16_t*>(smem + stage);
    const bool partly = bt.all_lo > k0 || bt.all_hi < k0 + KT;
    if (partly && sk.clean(bad[it & 1], it)) {
      odd_at[it & 1] = it;
      left.mark(it, a.Tk);
    }
    sk.store(Ks);
    sv.store(Ks + TILE);
    __syncthreads();
    if (k0 + KT < khi) {
      sk.next();
      sv.next();
      sk.load(a.Tk - k0 - KT, a.hd8);
      sv.load(a.Tk - k0 - KT, a.hd8);
    }
#pragma unroll
    for (int u = 0; u < 2 / SH; ++u) {
      const int at = 64 * D * SH * u;
      const int r0 = 32 * (SH * u + shr), kb = k0 + r0;
      if (!__any(rw.lo < kb + 32 && rw.hi > kb)) continue;
      f32x16 s = splat(0.f), dp = splat(-Dq);
#pragma unroll
      for (int kk = 0; kk < D / 16; ++kk)
        s = mma(rows32<D>(smem, rbase + stage, kk, at), qf[kk], s);
      // p under the MFMAs of dp
      const float far = (float)(rw.pos - kb - 8 * hl);
      float dz[16];
      constexpr int NK = D / 16;
#pragma unroll
      for (int kk = 0; kk < NK; ++kk) {
        in_order<D>();
        dp = mma(rows32<D>(smem, rbase + stage, kk, at + 2 * TILE), df[kk], dp);
        in_order<D>();
#pragma unroll
        for (int i = 16 * kk / NK; i < 16 * (kk + 1) / NK; ++i)
          s[i] = ex2(score(s[i], l2, far - (float)elem(i), dz[i]));
      }
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        s[i] *= dp[i];
        if (CAP) s[i] *= dz[i];
      }
      if (!__all(past || (rw.lo <= kb && rw.hi >= kb + 32))) {
        const uint32_t on = attended(rw, kb + 8 * hl);
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = keep_or(bit(on, elem(i)), s[i], 0);
      }
      if (partly && odd_at[it & 1] == it) {
        // a cleared key's score is not what it was; the rows that attend it
        // get their NaN at the end
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (bad[it & 1][r0 + 8 * hl + elem(i)] == it) s[i] = 0.f;
      }
      bf16x8 ds[2];
#pragma unroll
      for (int i = 0; i < 16; ++i) ds[i / 8][i % 8] = (__bf16)s[i];
#pragma unroll
      for (int d = 0; d < D / 32; ++d)
#pragma unroll
        for (int ks = 0; ks < 2; ++ks)
          acc[d] = mma(cols32<D>(smem, cbase + stage, d, at + 32 * D * ks), ds[ks], acc[d]);
    }
  }
  if (left.any) {  // set before the last barrier, if at all
    // a row whose lse is not finite may have attended cleared keys only
    const float e = rw.hi > rw.lo ? l2 * 0.f : 0.f;
#pragma unroll
    for (int d = 0; d < D / 32; ++d)
#pragma unroll
      for (int i = 0; i < 16; ++i) acc[d][i] += e;
  }
  write_rows<D, G>(reinterpret_cast<float*>(smem), acc, a.scale, a.dq + h * a.dqh, a.dqt,
                   part_of(a, a.part0, part, a.Tq, a.H, h), nullptr, tile * RB, a.Tq, a.H, a.hd8,
                   [&](int row, int c, float (&o)[8]) {
                     if (!left.any) return;
                     const Row x = row_at(a, row);
                     left.each(a.Tk, [&](int first, int end) {
                       for (int j = max(x.lo, first); j < min(x.hi, end); ++j)
                         add_odd(o, *reinterpret_cast<const uint4*>(kbase + j * a.kt + 8 * c),
                                 true);
                       return !all_nan(o);
                     });
                   });
}

// The tiles of query rows, in order, some of whose rows attend some of keys
// [k0, k1), and of these every step-th from the first-th on.  Every wave of a
// block sees the same ones: a wave looks at 64 table entries at a time.
struct Hits {
  int base, k0, k1, first, step, skip;
  uint64_t bits;
  __device__ __forceinline__ void look(const Dev& a, int lane) {
    const int t = base + lane;
    bool hit = false;
    if (t < mask_tiles(a.Tq)) {
      const MaskTile m = a.tiles[t];
      hit = m.lo < k1 && m.hi > k0;
    }
    bits = __ballot(hit);
  }
  __device__ __forceinline__ void start(const Dev& a, int lane) {
    base = 0;
    skip = first;
    look(a, lane);
  }
  // the next tile, or -1
  __device__ __forceinline__ int next(const Dev& a, int lane) {
    for (;;) {
      while (bits == 0) {
        base += 64;
        if (base >= mask_tiles(a.Tq)) return -1;
        look(a, lane);
      }
      const int t = base + __builtin_ctzll(bits);
      bits &= bits - 1;
      if (skip-- == 0) {
        skip = step - 1;
        return t;
      }
    }
  }
};

// ---------------------------------------------------------------------------
// Backward over keys: dk = ds^T q, dv = p^T do, the query rows of every head
// of the group that attend any of the block's keys streaming by.  Computing s
// and dp again here costs two products of seven, but needs neither atomics
// (whose order would change results) nor partial sums of dq per key tile.
// Both accumulators and both operands of D = 128 do not fit the registers of
// two waves per SIMD: dv and dk then have a pass each, with s computed in both
// (8192 tokens of 16 heads: 1370 us instead of 1489; at D = 96 one pass, 143
// us, and two, 174, 8 x 1024 tokens).  About 900 TFLOP/s over its products.
// The whole backward at 8192 tokens of 16 heads: D = 64 1050 us, D = 128 2165.
// ---------------------------------------------------------------------------
template <int D, int G, int WPE, int CAP, bool BIAS, bool DK, bool DV>
__global__ __launch_bounds__(256, WPE) void k_mattn_bwd_kv(Dev a) {
  constexpr int SH = 4 / G, RB = 32 * G, TILE = KT * D;
  __shared__ __attribute__((aligned(16))) char smem[SMEM<D>];
  // Pos: a row's place, from the block's first key
  __shared__ __attribute__((aligned(16))) float Ls[2][KT], Ds[2][KT], Pos[2][KT];
  __shared__ __attribute__((aligned(16))) int Lo[2][KT], Hi[2][KT];
  __shared__ int odd_q, odd_do;  // whether values of q and dout were left out
  __shared__ Left left;
  int tile, kh, part;
  block_of(a, (a.Tk + RB - 1) / RB, a.H / a.rep, false, tile, kh, part);
  const int lane = tid() & 63, w = tid() >> 6, n = lane & 31, hl = lane >> 5;
  const int grp = w / SH, shr = w % SH;
  const int rbase = rows_base<D>(lane) + shr * 64 * D, cbase = cols_base<D>(lane) + shr * 64 * D;
  const int kb0 = tile * RB + grp * 32, key = kb0 + n;
  const float kfn = (float)(grp * 32 + n);  // as Pos
  if (tid() == 0) odd_q = odd_do = 0;
  left.init(tid(), 0, a.Tq);
  bf16x8 kf[D / 16], vf[D / 16];
#pragma unroll
  for (int kk = 0; kk < D / 16; ++kk) {
    kf[kk] = row_frag(a.k + key * a.kt + kh * a.kh, 2 * kk + hl, key < a.Tk, a.hd8);
    if (DK) vf[kk] = row_frag(a.v + key * a.vt + kh * a.vh, 2 * kk + hl, key < a.Tk, a.hd8);
  }
  f32x16 dk[D / 32], dv[D / 32];
#pragma unroll
  for (int d = 0; d < D / 32; ++d) {
    if (DK) dk[d] = splat(0.f);
    if (DV) dv[d] = splat(0.f);
  }
  Stage<D> sq, sd;
  sq.init(a.q, 0, a.qt);
  sd.init(a.dout, 0, a.dot);
  Hits hits;
  hits.k0 = tile * RB;
  hits.k1 = tile * RB + RB;
  // the part's heads, and its share of the tiles of rows
  const int hp = part % a.head_parts;
  int h = kh * a.rep + hp * a.head_per;
  const int hend = min(h + a.head_per, (kh + 1) * a.rep);
  hits.first = part / a.head_parts;
  hits.step = a.parts / a.head_parts;
  float ln = 0.f, dn = 0.f;  // of the next tile's rows (threads 0..63)
  Row rn{0, 0, 0};
  __syncthreads();  // left, odd_q, odd_do

  // (h, qt) is the tile in the registers, which goes to LDS next
  const auto fetch = [&](int h, int qt) {
    const long r = (long)qt * KT;
    sq.p = a.q + (r + sq.r) * a.qt + h * a.qh + 8 * sq.c;
    sd.p = a.dout + (r + sd.r) * a.dot + h * a.doh + 8 * sd.c;
    sq.load(a.Tq - qt * KT, a.hd8);
    sd.load(a.Tq - qt * KT, a.hd8);
    if (tid() < KT) {
      const int i = qt * KT + tid();
      rn = i < a.Tq ? row_at(a, i) : Row{PAST, 0, 0};
      if (i < a.Tq) {
        ln = a.lse[(long)h * a.Tq + i];
        dn = a.dsum[(long)h * a.Tq + i];
      }
    }
  };
  hits.start(a, lane);
  int qt = hits.next(a, lane);
  if (qt >= 0) fetch(h, qt);
  for (int it = 0; qt >= 0; ++it) {
    const int stage = (it & 1) * 4 * TILE;
    uint16_t* Qs = reinterpret_cast<uint16_t*>(smem + stage);
    const Score<CAP, BIAS> score(a, h);
    const MaskTile mt = a.tiles[qt];
    if (mt.all_lo > hits.k0 || mt.all_hi < hits.k1) {
      // A row with such a q has no finite lse, but under a cap, where infinite
      // scores are +-cap: the largest finite q gives the same p and ds = 0,
      // and dk its NaN (0 inf) at the end.
      if (sq.template clean<(CAP > 0)>() && CAP) {
        left.mark(qt, a.Tq);
        odd_q = 1;
      }
      if (sd.clean()) {
        left.mark(qt, a.Tq);
        odd_do = 1;
      }
    }
    sq.store(Qs);
    sd.store(Qs + TILE);
    if (tid() < KT) {
      // a row past the last has p = 0 and is not masked
      const float l2 = rn.lo == PAST ? INFINITY : finite_or_nan(ln) * LOG2E;
      Ls[it & 1][tid()] = CAP ? l2 : -l2 * a.inv_c1;
      Ds[it & 1][tid()] = rn.lo == PAST ? 0.f : -finite_or_nan(dn);
      Lo[it & 1][tid()] = rn.lo;
      Hi[it & 1][tid()] = rn.hi;
      Pos[it & 1][tid()] = rn.lo == PAST ? (float)PAST : (float)(rn.pos - tile * RB);
    }
    __syncthreads();
    int qn = hits.next(a, lane);
    if (qn < 0 && h + 1 < hend) {
      ++h;
      hits.start(a, lane);
      qn = hits.next(a, lane);
    }
    if (qn >= 0) fetch(h, qn);
#pragma unroll
    for (int u = 0; u < 2 / SH; ++u) {
      const int at = 64 * D * SH * u;
      const int rb = 32 * (SH * u + shr) + 8 * hl;  // the lane's first row in the tile
      if (kb0 >= mt.hi || kb0 + 32 <= mt.lo) continue;
      bool part = mt.all_lo > kb0 || mt.all_hi < kb0 + 32;
      if (part) {
        // the step's rows (lane n: row n) against the wave's keys
        const int lo = Lo[it & 1][rb - 8 * hl + n], hi = Hi[it & 1][rb - 8 * hl + n];
        if (!__any(lo < kb0 + 32 && hi > kb0)) continue;
        part = !__all(lo == PAST || (lo <= kb0 && hi >= kb0 + 32));
      }
      // Uncapped, -lse / k and the bias / k start the sum of s, so that
      // p = 2^(k s); -D starts dp, so that ds = p dp.  2 x 6120 tokens of 16
      // heads on 4, D = 128, with a bias, whole backward: 1730 us, 1770 with
      // the bias added to s; 1750 with a form linear in the place where the
      // rows lie on one side of the keys.
      const float* Lr = Ls[it & 1] + rb;
      const float* Dr = Ds[it & 1] + rb;
      const float* Pr = Pos[it & 1] + rb;
      f32x16 s;
      if constexpr (CAP) {
        s = splat(0.f);
      } else if constexpr (BIAS) {
        const float b = -score.sl * a.inv_c1;
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = fmaf(b, fabsf(Pr[elem(i)] - kfn), Lr[elem(i)]);
      } else {
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = Lr[elem(i)];
      }
#pragma unroll
      for (int kk = 0; kk < D / 16; ++kk)
        s = mma(rows32<D>(smem, rbase + stage, kk, at), kf[kk], s);
      bf16x8 p[2], ds[2];
      float dz[16];
      f32x16 dp;
      if (DK) {
#pragma unroll
        for (int i = 0; i < 16; ++i) dp[i] = Dr[elem(i)];
      }
      // p under the MFMAs of dp
      constexpr int NK = D / 16;
#pragma unroll
      for (int kk = 0; kk < NK; ++kk) {
        if (DK) {
          in_order<D>();
          dp = mma(rows32<D>(smem, rbase + stage, kk, at + 2 * TILE), vf[kk], dp);
          in_order<D>();
        }
#pragma unroll
        for (int i = 16 * kk / NK; i < 16 * (kk + 1) / NK; ++i)
          s[i] = CAP ? ex2(score(s[i], Lr[elem(i)], BIAS ? Pr[elem(i)] - kfn : 0.f, dz[i]))
                     : ex2(s[i] * score.k);
      }
      if (DK) {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          dp[i] *= s[i];
          if (CAP) dp[i] *= dz[i];
        }
      }
      if (part) {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int r = rb + elem(i);
          // no short cut: a branch per element costs more than the compares
          const bool out = (key < Lo[it & 1][r]) | (key >= Hi[it & 1][r]);
          s[i] = out ? 0.f : s[i];
          if (DK) dp[i] = out ? 0.f : dp[i];
        }
      }
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        if (DV) p[i / 8][i % 8] = (__bf16)s[i];
        if (DK) ds[i / 8][i % 8] = (__bf16)dp[i];
      }
      if (DV) {
#pragma unroll
        for (int d = 0; d < D / 32; ++d)
#pragma unroll
          for (int ks = 0; ks < 2; ++ks)
            dv[d] = mma(cols32<D>(smem, cbase + stage, d, at + 32 * D * ks + 2 * TILE), p[ks],
                        dv[d]);
      }
      if (DK) {
#pragma unroll
        for (int d = 0; d < D / 32; ++d)
#pragma unroll
          for (int ks = 0; ks < 2; ++ks)
            dk[d] = mma(cols32<D>(smem, cbase + stage, d, at + 32 * D * ks), ds[ks], dk[d]);
      }
    }
    qt = qn;
  }
  // o += the values left out of x (q or dout) in the rows that attend key j, of
  // every head of the group: what another part adds too stays what it is
  const auto add_left = [&](const uint16_t* x, long xt, long xh, bool nan, int j, int c,
                            float (&o)[8]) {
    left.each(a.Tq, [&](int first, int end) {
      for (int i = first; i < end; ++i) {
        const Row r = row_at(a, i);
        if (j < r.lo || j >= r.hi) continue;
        for (int g = kh * a.rep; g < (kh + 1) * a.rep; ++g)
          add_odd(o, *reinterpret_cast<const uint4*>(x + i * xt + g * xh + 8 * c), nan);
      }
      return !all_nan(o);
    });
  };
  float* mb = reinterpret_cast<float*>(smem);
  if constexpr (DK)
    write_rows<D, G>(mb, dk, a.scale, a.dk + kh * a.dkh, a.dkt,
                     part_of(a, a.part0, part, a.Tk, a.H / a.rep, kh), nullptr, tile * RB, a.Tk,
                     a.H / a.rep, a.hd8, [&](int j, int c, float (&o)[8]) {
                       if (CAP && odd_q) add_left(a.q, a.qt, a.qh, true, j, c, o);
                     });
  if constexpr (DV)
    write_rows<D, G>(mb, dv, 1.f, a.dv + kh * a.dvh, a.dvt,
                     part_of(a, a.part1, part, a.Tk, a.H / a.rep, kh), nullptr, tile * RB, a.Tk,
                     a.H / a.rep, a.hd8, [&](int j, int c, float (&o)[8]) {
                       if (odd_do) add_left(a.dout, a.dot, a.doh, false, j, c, o);
                     });
}

Dev view(const MattnArgs& a) {
  Dev d{};
  d.Tq = a.Tq, d.Tk = a.Tk, d.H = a.H, d.rep = a.H / a.KV, d.hd8 = a.hd / 8;
  d.scale = a.scale, d.cap = a.cap;
  d.c1 = a.cap > 0.f ? a.scale / a.cap : a.scale * LOG2E;
  d.c2 = a.cap * LOG2E;
  // of a cap so small that all but scores of 0 reach it
  if (a.cap > 0.f && fabsf(d.c1) > 1e30f) d.c1 = copysignf(1e30f, d.c1);
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
  d.o_low = static_cast<uint16_t*>(a.o_low);
  return d;
}

// ---------------------------------------------------------------------------
// joining the parts
// ---------------------------------------------------------------------------

// out = sum of the parts, in order (workgroup y: dq or dk; dv).  Memory-bound:
// each partial is read once.
__global__ __launch_bounds__(256) void k_mattn_sum(int parts, long rows, int heads, int hd8,
                                                   const float* p0, const float* p1, uint16_t* o0,
                                                   uint16_t* o1, long t0, long h0, long t1,
                                                   long h1) {
  const bool y = blockIdx.y;
  const float* p = y ? p1 : p0;
  uint16_t* out = y ? o1 : o0;
  const long ts = y ? t1 : t0, hs = y ? h1 : h0;
  const long n = rows * heads * hd8;
  const long e = (long)blockIdx.x * 256 + tid();
  if (e >= n) return;
  float o[8] = {};
  for (int i = 0; i < parts; ++i) {
    const float4* q = reinterpret_cast<const float4*>(p + (i * n + e) * 8);
    const float4 a = q[0], b = q[1];
    o[0] += a.x, o[1] += a.y, o[2] += a.z, o[3] += a.w;
    o[4] += b.x, o[5] += b.y, o[6] += b.z, o[7] += b.w;
  }
  const long rh = e / hd8, row = rh / heads;
  const int c = e - rh * hd8, h = rh - row * heads;
  *reinterpret_cast<uint4*>(out + row * ts + h * hs + 8 * c) = rounded(o);
}

// o = sum o_p 2^(lse_p - lse), lse = log2 sum 2^lse_p over the forward's parts;
// memory-bound
__global__ __launch_bounds__(256) void k_mattn_join(Dev a) {
  const long n = (long)a.Tq * a.H * a.hd8;
  const long e = (long)blockIdx.x * 256 + tid();
  if (e >= n) return;
  const long rh = e / a.hd8;
  const int c = e - rh * a.hd8, row = rh / a.H, h = rh - (long)row * a.H;
  const Row x = row_at(a, row);
  const bool empty = x.hi <= x.lo;
  const float* l = a.part_lse + (long)h * a.Tq + row;
  const long lp = (long)a.H * a.Tq;
  float R = l[0], t = 0.f, o[8] = {};
  for (int i = 1; i < a.parts; ++i) R = fmaxf(R, l[i * lp]);
  for (int i = 0; i < a.parts; ++i) {
    const float w = ex2(l[i * lp] - R);
    t += w;
    const float4* q = reinterpret_cast<const float4*>(a.part0 + (i * n + e) * 8);
    const float4 u = q[0], v = q[1];
    o[0] += w * u.x, o[1] += w * u.y, o[2] += w * u.z, o[3] += w * u.w;
    o[4] += w * v.x, o[5] += w * v.y, o[6] += w * v.z, o[7] += w * v.w;
  }
  const float f = 1.f / t;
#pragma unroll
  for (int i = 0; i < 8; ++i) o[i] = empty ? 0.f : o[i] * f;
  *reinterpret_cast<uint4*>(a.o + row * a.ot + h * a.oh + 8 * c) = rounded(o);
  if (a.o_low) *reinterpret_cast<uint4*>(a.o_low + e * 8) = left_out(o);
  if (c == 0)
    a.lse[(long)h * a.Tq + row] = empty ? -INFINITY : (R + __builtin_amdgcn_logf(t)) * LN2;
}

enum Pass { FWD, BWD_Q, BWD_KV };

struct Plan {
  int group;                        // groups of 32 rows per block
  int parts, head_parts, head_per;  // as in Dev
};

// How a pass is spread over the GPU (256 CUs, two or three blocks each); us
// of forward and backward in what follows.
//
// Shared key heads: where there are fewer than 1024 blocks over keys, each takes
// a part of the heads that share its keys, as many as leave 3072 blocks (one
// at least).  12240 tokens, 16 heads on 2, D = 64: 1505 in parts, 3135 without;
// at 1024 blocks (65536 tokens in 128 documents, 16 heads on 4) 854 and 652.
// With 1024 left instead of 3072 the backward of 16384 tokens, 32 heads on 2,
// D = 128, causal, takes 9442 instead of 8727.  There are fewer than 7168
// blocks then, whose fp32 partials take less than 1 GB (128 channels).
//
// Blocks of 128 rows where there are 512 of them, else of 64.  4096 tokens of
// 16 heads (512 blocks) in 16 documents: 15.9 + 39.1 with 128 rows, 16.4 +
// 50.7 with 64; 4001 of 12 heads (384) in 21 documents of 60 to 958: 37.5 +
// 106.9 and 28.3 + 92.4 (D = 128: 51.7 + 204 and 47.5 + 185; where all
// documents are alike, 10 % the other way).
//
// Fewer than 256 blocks: in parts along the other side, up to one block per
// CU, of 256 rows or more (512 beyond 8 parts), where that takes at least 1024
// rows off each block, since the second kernel costs 4 us.  1 row on 16384
// keys, 8 heads: 26 + 46 in parts, 189 + 302 without; 2048 on 2048, 2 heads,
// D = 64, in one document 18 + 41 and 27 + 73, in 4 documents, of which a part
// may see none, 13 + 28 and 10 + 27.  Two blocks per CU gain 10 % on one
// document and lose 40 % on four; 1024 on 1024 in two parts or more: 12 + 24
// and 10 + 27 on two documents, 20 + 52 and 17 + 44 with 12 heads.
Plan plan(Pass p, int Tq, int Tk, int H, int KV) {
  const int rows = p == BWD_KV ? Tk : Tq, heads = p == BWD_KV ? KV : H;
  const int other = p == BWD_KV ? Tq : Tk;
  Plan x{4, 1, 1, H / KV};
  long blocks = (long)((rows + 127) / 128) * heads;
  if (p == BWD_KV && blocks < 1024 && H > KV) {
    const long per = H / KV * blocks / 3072;
    x.head_per = per > 1 ? (int)per : 1;
    x.parts = x.head_parts = (H / KV + x.head_per - 1) / x.head_per;
    blocks *= x.parts;
  }
  if (blocks < 512) {
    x.group = 2;
    blocks = (long)((rows + 63) / 64) * heads * x.parts;
  }
  if (blocks > 0 && blocks < 256) {
    const long most = max_of(other / 512, other / 256 < 8 ? other / 256 : 8);
    long n = 256 / blocks;
    if (n > most) n = most;
    if (n > 64) n = 64;
    if (n > 1 && other - other / n >= 1024) x.parts *= (int)n;
  }
  return x;
}

template <Pass P, int D, int G, int WPE, int CAP, bool BIAS>
hipError_t launch(const Dev& d, hipStream_t st) {
  constexpr int RB = 32 * G;
  const int rows = P == BWD_KV ? d.Tk : d.Tq, heads = P == BWD_KV ? d.H / d.rep : d.H;
  const dim3 grid((long)((rows + RB - 1) / RB) * heads * d.parts), block(256);
  if constexpr (P == FWD)
    hipLaunchKernelGGL((k_mattn_fwd<D, G, WPE, CAP, BIAS>), grid, block, 0, st, d);
  else if constexpr (P == BWD_Q)
    hipLaunchKernelGGL((k_mattn_bwd_q<D, G, WPE, CAP, BIAS>), grid, block, 0, st, d);
  else if constexpr (D < 128)
    hipLaunchKernelGGL((k_mattn_bwd_kv<D, G, WPE, CAP, BIAS, true, true>), grid, block, 0, st, d);
  else {
    hipLaunchKernelGGL((k_mattn_bwd_kv<D, G, WPE, CAP, BIAS, false, true>), grid, block, 0, st, d);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((k_mattn_bwd_kv<D, G, WPE, CAP, BIAS, true, false>), grid, block, 0, st, d);
  }
  return hipGetLastError();
}

template <Pass P, int D, int G, int WPE>
hipError_t launch_mode(const Dev& d, hipStream_t st) {
  const auto cap = [&](auto bias) {
    constexpr bool B = decltype(bias)::value;
    if (d.cap > CAP_LOW) return launch<P, D, G, WPE, ANY, B>(d, st);
    if (d.cap > 0.f) return launch<P, D, G, WPE, LOW, B>(d, st);
    return launch<P, D, G, WPE, NONE, B>(d, st);
  };
  return d.slopes ? cap(std::true_type{}) : cap(std::false_type{});
}

template <Pass P, int D>
hipError_t launch_rows(const Dev& d, int group, hipStream_t st) {
  // waves per SIMD.  Three at D = 64: 16 x 256 tokens of 12 heads, backward
  // 38.6 us, with two 40.6, though over rows up to 20 bytes a lane spill (52
  // under a cap, 144 under one above CAP_LOW).  Three at 96, and over keys,
  // spill more (8 x 1024 tokens of 16 heads of 88, backward: 220 us with two,
  // 338 with three over rows).  With two, what spills is 12 to 60 bytes over
  // keys at 96 (92 above CAP_LOW) and, under a cap, up to 60 over rows and 80
  // over keys at 128.
  constexpr int W = P != BWD_KV && D == 64 ? 3 : 2;
  return group == 4 ? launch_mode<P, D, 4, W>(d, st) : launch_mode<P, D, 2, W>(d, st);
}

template <Pass P>
hipError_t launch_dim(const Dev& d, int group, hipStream_t st) {
  if (d.hd8 <= 8) return launch_rows<P, 64>(d, group, st);
  if (d.hd8 <= 12) return launch_rows<P, 96>(d, group, st);
  return launch_rows<P, 128>(d, group, st);
}

size_t al256(size_t x) { return (x + 255) & ~(size_t)255; }

// Workspace of a pass: D of every row (backward), then the parts' results.
struct Space {
  size_t dsum, part0, part1, lse, bytes;
};
Space space(Pass p, const Plan& x, int Tq, int Tk, int H, int KV, int hd) {
  Space s{};
  size_t at = p == FWD ? 0 : al256((size_t)H * Tq * 4);
  if (x.parts > 1) {
    const size_t one = al256((size_t)x.parts * (p == BWD_KV ? (size_t)Tk * KV : (size_t)Tq * H) *
                             hd * 4);
    s.part0 = at;
    at += one;
    if (p == BWD_KV) s.part1 = at, at += one;
    if (p == FWD) s.lse = at, at += al256((size_t)x.parts * H * Tq * 4);
  }
  s.bytes = at;
  return s;
}

template <Pass P>
hipError_t run(const MattnArgs& a, hipStream_t st) {
  const int rows = P == BWD_KV ? a.Tk : a.Tq, heads = P == BWD_KV ? a.KV : a.H;
  if (rows == 0) return hipSuccess;
  const Plan x = plan(P, a.Tq, a.Tk, a.H, a.KV);
  const Space s = space(P, x, a.Tq, a.Tk, a.H, a.KV, a.hd);
  char* ws = static_cast<char*>(a.ws);
  Dev d = view(a);
  if (P == BWD_KV && !(a.cap > 0.f)) {
    // which divides by it: a scale of 0 becomes one at which scores vanish too
    if (fabsf(d.c1) < 1e-30f) d.c1 = 1e-30f;
    d.inv_c1 = 1.f / d.c1;
  }
  d.parts = x.parts, d.head_parts = x.head_parts, d.head_per = x.head_per;
  d.dsum = reinterpret_cast<float*>(ws);
  d.part0 = reinterpret_cast<float*>(ws + s.part0);
  d.part1 = reinterpret_cast<float*>(ws + s.part1);
  d.part_lse = reinterpret_cast<float*>(ws + s.lse);
  const hipError_t e = launch_dim<P>(d, x.group, st);
  if (e != hipSuccess || x.parts == 1) return e;
  const long n = (long)rows * heads * d.hd8;
  const dim3 grid((n + 255) / 256, P == BWD_KV ? 2 : 1);
  if (P == FWD)
    hipLaunchKernelGGL(k_mattn_join, grid, dim3(256), 0, st, d);
  else if (P == BWD_Q)
    hipLaunchKernelGGL(k_mattn_sum, grid, dim3(256), 0, st, x.parts, (long)rows, heads, d.hd8,
                       d.part0, d.part0, d.dq, d.dq, d.dqt, d.dqh, d.dqt, d.dqh);
  else
    hipLaunchKernelGGL(k_mattn_sum, grid, dim3(256), 0, st, x.parts, (long)rows, heads, d.hd8,
                       d.part0, d.part1, d.dk, d.dv, d.dkt, d.dkh, d.dvt, d.dvh);
  return hipGetLastError();
}

template <Pass P>
size_t bytes(const pulse_attn_desc& d) {
  return space(P, plan(P, d.queries, d.keys, d.heads, d.kv_heads), d.queries, d.keys, d.heads,
               d.kv_heads, d.head_dim)
      .bytes;
}

}  // namespace

size_t mattn_fwd_bytes(const pulse_attn_desc& d) { return bytes<FWD>(d); }
size_t mattn_bwd_bytes(const pulse_attn_desc& d) {
  const size_t q = bytes<BWD_Q>(d), kv = bytes<BWD_KV>(d);
  return q > kv ? q : kv;  // one after the other
}

hipError_t launch_mattn_fwd(const MattnArgs& a, hipStream_t st) { return run<FWD>(a, st); }

hipError_t launch_mattn_bwd(const MattnArgs& a, hipStream_t st) {
  const hipError_t e = run<BWD_Q>(a, st);
  return e == hipSuccess ? run<BWD_KV>(a, st) : e;
}

}  // namespace pulse
