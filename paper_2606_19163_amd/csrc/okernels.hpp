// Internal launcher interface of the packed-sequence operators (mask.hip,
// rope.hip, mattn.hip, clip.hip); not part of the public ABI.  Arguments have
// been validated by ops.cpp.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "pulse_ops.h"

namespace pulse {

// ---- masks (mask.hip) -----------------------------------------------------

// Query rows per entry of a mask's tile table.
constexpr int MASK_TILE = 64;

// Over the rows of a tile: the attended keys lie in [lo, hi) (over the rows
// that attend any; lo = hi = 0 if none do), and every row attends all of
// [all_lo, all_hi) (a row that attends nothing, or that is past the last
// one, makes all_hi 0).
struct MaskTile {
  int32_t lo, hi, all_lo, all_hi;
};

__host__ __device__ inline int mask_tiles(int queries) {
  return (queries + MASK_TILE - 1) / MASK_TILE;
}
inline size_t mask_bytes(int queries) {
  return (size_t)queries * sizeof(pulse_mask_row) + (size_t)mask_tiles(queries) * sizeof(MaskTile);
}

hipError_t launch_mask_build(const pulse_mask_desc& d, const int32_t* q_off, const int32_t* k_off,
                             const int32_t* prefix, void* mask, hipStream_t st);
hipError_t launch_mask_rows(const pulse_mask_desc& d, const pulse_mask_row* rows, void* mask,
                            hipStream_t st);

// ---- rotary positions (rope.hip) ---------------------------------------------

hipError_t launch_rope(const pulse_rope_desc& d, int tokens, bool backward, const pulse_heads& x,
                       const float* pos, const float* freq, const pulse_heads& y, hipStream_t st);

// ---- attention (mattn.hip) ---------------------------------------------------

struct MattnArgs {
  int Tq, Tk, H, KV, hd;
  float scale, cap;
  pulse_heads q, k, v, o, dout, dq, dk, dv;
  const void* mask;
  const float* slopes;
  float* lse;
  void* o_low;  // or null
  void* ws;
};

size_t mattn_fwd_bytes(const pulse_attn_desc& d);
size_t mattn_bwd_bytes(const pulse_attn_desc& d);
hipError_t launch_mattn_fwd(const MattnArgs& a, hipStream_t st);
hipError_t launch_mattn_bwd(const MattnArgs& a, hipStream_t st);

// ---- gradient norm and clipping (clip.hip) -----------------------------------

// Up to CLIP_CHUNK consecutive elements of one tensor.
constexpr int CLIP_CHUNK = 8192;
struct ClipChunk {
  const void* g;
  void* o;
  int32_t n, dtype;
};
constexpr int CLIP_BLOCKS = 2048;  // most blocks, and partial sums
hipError_t launch_clip(const ClipChunk* chunks, int count, double* part, float max_norm, float eps,
                       float* norm, hipStream_t st);

}  // namespace pulse
