// Internal launcher interface of the packed-sequence operators (mask.hip,
// rope.hip, mattn.hip, clip.hip, bnorm.hip, keep.hip, kgrad.hip, lin8.hip); not
// part of the public ABI.  Arguments have been validated by ops.cpp and
// rowops.cpp.
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

// ---- norms of a block (bnorm.hip) --------------------------------------------

// strides in elements; unused pointers are null
struct NormArgs {
  int tokens, C, docs, pre, post, branch, dtype, stream_dtype;
  float eps, r;
  const int32_t* off;
  const float *gate, *scale, *shift;
  long gate_t, scale_t, shift_t;
  const float *weight, *bias, *post_weight;
  const void *x, *y, *du, *dh;
  void *h, *u, *dx, *dy;  // h is read by the backward pass
  long xt, yt, ht, ut, dut, dht, dxt, dyt;
};

size_t norm_bwd_bytes(const pulse_norm_desc& d, int tokens);
hipError_t launch_norm_fwd(const NormArgs& a, hipStream_t st);
hipError_t launch_norm_bwd(const NormArgs& a, const pulse_norm_grads& o, float* ws,
                           hipStream_t st);

// ---- activations in 8 bits (keep.hip, kgrad.hip) -----------------------------

inline int64_t keep_pitch(int channels) { return (channels + 31) / 32 * 32; }
// bytes of a row's exponents: whole words, so that four are one load
__host__ __device__ inline int64_t keep_exp_pitch(int channels) { return (channels + 127) / 128 * 4; }
inline size_t keep_values(int channels, int tokens) { return (size_t)tokens * keep_pitch(channels); }
inline size_t keep_exps_at(int channels, int tokens) {
  return (keep_values(channels, tokens) + 15) / 16 * 16;
}
inline size_t keep_bytes(int channels, int tokens) {
  return keep_exps_at(channels, tokens) + (size_t)tokens * keep_exp_pitch(channels);
}

// x (or da) read, y (a, the loaded rows, or dx) written; strides in elements
struct KeepArgs {
  int tokens, C, act, dtype;
  const void* x;
  void* y;
  long xt, yt;
  void* kept;    // values, then exponents
  void* a_kept;  // or null
};
hipError_t launch_keep_save(const KeepArgs& a, hipStream_t st);
hipError_t launch_keep_load(const KeepArgs& a, hipStream_t st);
hipError_t launch_keep_back(const KeepArgs& a, hipStream_t st);

struct KgradArgs {
  int tokens, C, N;
  const void* dy;
  long dyt;
  const void* kept;
  float *dw, *db;
  int accumulate;
  float* ws;
};
size_t kgrad_bytes(int tokens, int C, int N);
hipError_t launch_kgrad(const KgradArgs& a, hipStream_t st);

// ---- linear layers in 8-bit integers (lin8.hip) --------------------------------

struct Lin8Args {
  int tokens, K, N, act;
  const void* x;
  long xt;
  const void* weights;
  const float* bias;
  void* y;
  long yt;
  void* ws;
};
size_t lin8_weight_bytes(int K, int N);
size_t lin8_ws_bytes(int tokens, int K, int N);
hipError_t launch_lin8_pack(int K, int N, const void* w, int w_dtype, void* weights,
                            hipStream_t st);
hipError_t launch_lin8(const Lin8Args& a, hipStream_t st);

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
