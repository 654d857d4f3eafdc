// Masks of packed sequences (gfx950): per query row the interval of keys it
// attends, and per tile of 64 rows the intervals that the attention kernels
// use to skip key tiles (nothing attended) and to leave out the comparisons
// (everything attended).  One wave per tile, one lane per row, which finds its
// document by bisection.  Bound by that chain of loads: 4096 rows of 16
// documents 3.0 us, 131072 of 1500 4.6, where 2 MB are written.
#include <limits.h>

#include "okernels.hpp"

namespace pulse {
namespace {

// number of entries of off[0, n) that are <= i (off ascending)
__device__ __forceinline__ int upper(const int32_t* off, int n, int i) {
  int a = 0, b = n;
  while (a < b) {
    const int m = (a + b) >> 1;
    if (off[m] <= i)
      a = m + 1;
    else
      b = m;
  }
  return a;
}

// Clamp row i to the keys, store it and reduce its tile's entry; every lane
// of the wave calls it, lanes past the last row with i >= Tq.
__device__ __forceinline__ void put(pulse_mask_row r, int i, int Tq, int Tk, pulse_mask_row* rows) {
  r.lo = max(r.lo, 0);
  r.hi = min(r.hi, Tk);
  if (i >= Tq || r.hi <= r.lo) r.lo = r.hi = 0;
  if (i < Tq) rows[i] = r;
  const bool any = r.hi > r.lo;
  int lo = any ? r.lo : INT_MAX, hi = r.hi, alo = r.lo, ahi = r.hi;
#pragma unroll
  for (int s = 1; s < 64; s <<= 1) {
    lo = min(lo, __shfl_xor(lo, s, 64));
    hi = max(hi, __shfl_xor(hi, s, 64));
    alo = max(alo, __shfl_xor(alo, s, 64));
    ahi = min(ahi, __shfl_xor(ahi, s, 64));
  }
  if ((threadIdx.x & 63) == 0 && i < Tq) {
    MaskTile* t = reinterpret_cast<MaskTile*>(rows + Tq) + i / MASK_TILE;
    *t = MaskTile{hi > 0 ? lo : 0, hi, alo, ahi};
  }
}

__global__ __launch_bounds__(256) void k_mask_build(int Tq, int Tk, int docs, int causal,
                                                    const int32_t* q_off, const int32_t* k_off,
                                                    const int32_t* prefix, pulse_mask_row* rows) {
  const int i = blockIdx.x * 256 + threadIdx.x;
  pulse_mask_row r{0, 0, 0, -1};
  const int d = upper(q_off, docs + 1, i) - 1;
  if (d >= 0 && d < docs) {
    // 64-bit, so that no offset in memory overflows
    const long q0 = q_off[d], nq = q_off[d + 1] - q0;
    const long k0 = k_off[d], k1 = k_off[d + 1];
    const long pos = k1 - nq + (i - q0);
    long hi = k1;
    if (causal) {
      long seen = pos + 1;
      if (prefix) seen = max(seen, k0 + prefix[d]);
      hi = min(hi, seen);
    }
    r.lo = (int)k0;
    r.hi = (int)max(hi, 0L);
    r.pos = (int)pos;
    r.doc = d;
  }
  put(r, i, Tq, Tk, rows);
}

__global__ __launch_bounds__(256) void k_mask_rows(int Tq, int Tk, const pulse_mask_row* in,
                                                   pulse_mask_row* rows) {
  const int i = blockIdx.x * 256 + threadIdx.x;
  pulse_mask_row r{0, 0, 0, -1};
  if (i < Tq) r = in[i];
  put(r, i, Tq, Tk, rows);
}

}  // namespace

hipError_t launch_mask_build(const pulse_mask_desc& d, const int32_t* q_off, const int32_t* k_off,
                             const int32_t* prefix, void* mask, hipStream_t st) {
  if (d.queries == 0) return hipSuccess;
  hipLaunchKernelGGL(k_mask_build, dim3((d.queries + 255) / 256), dim3(256), 0, st, d.queries,
                     d.keys, d.docs, d.causal, q_off, k_off ? k_off : q_off, prefix,
                     static_cast<pulse_mask_row*>(mask));
  return hipGetLastError();
}

hipError_t launch_mask_rows(const pulse_mask_desc& d, const pulse_mask_row* rows, void* mask,
                            hipStream_t st) {
  if (d.queries == 0) return hipSuccess;
  hipLaunchKernelGGL(k_mask_rows, dim3((d.queries + 255) / 256), dim3(256), 0, st, d.queries,
                     d.keys, rows, static_cast<pulse_mask_row*>(mask));
  return hipGetLastError();
}

}  // namespace pulse
