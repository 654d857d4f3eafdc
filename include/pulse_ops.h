/*
 * pulse_ops.h -- C ABI of the packed-sequence operators (gfx950).
 *
 * A denoiser that trains on images and clips of several resolutions packs
 * them one after another into one sequence: each is a document, and a token
 * attends only within its own.  Four operators work on such a batch:
 *
 *   pulse_mask  which keys each query row attends, built on the GPU from the
 *               documents' offsets (document, causal and prefix masks) or
 *               from the caller's own intervals;
 *   pulse_rope  rotary positions with one to four axes (time, height,
 *               width), forward and backward;
 *   pulse_attn  softmax attention under such a mask, with shared key heads,
 *               tanh-capped scores and a bias linear in the distance,
 *               forward and backward;
 *   pulse_clip  the global norm over many gradient tensors, and clipping.
 *
 * Conventions (as in pulse_stage.h): tensor pointers are caller-owned DEVICE
 * memory valid until the enqueued work has run.  Nothing here allocates
 * device memory or synchronises; scratch is a workspace that the caller
 * passes, and calls that share one must be ordered by the caller.  Every call
 * validates its host arguments before it enqueues anything; on error it
 * returns a status != PULSE_OK, enqueues nothing and pulse_last_error() says
 * why.  Values in device memory (offsets, prefixes, intervals) cannot be
 * checked by the host: the kernels clamp them, so that no value makes a
 * kernel read or write out of range.  Results are the same bits on every
 * run: no float is accumulated with atomics.  All calls but those stated
 * otherwise may be captured into a HIP graph.
 */
#ifndef PULSE_OPS_H
#define PULSE_OPS_H

#include "pulse_stage.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Heads of a token-major or head-major tensor: element (t, h, c) lies at
 * ptr + t * token_stride + h * head_stride + c (strides in elements).  ptr is
 * 16-byte aligned and both strides are multiples of 16 bytes, >= 0 and such
 * that neither axis extends over more than 2^47 elements.  The elements of an
 * output must not overlap one another: one stride is at least the head
 * dimension and the other at least the extent of that whole axis. */
typedef struct {
  void* ptr;
  int64_t token_stride, head_stride;
} pulse_heads;

/* ---- rotary positions --------------------------------------------------- */

/* Which channels form a pair.  The turned channels are the first
 * R = sum axis_dim of the head, R / 2 pairs; the first axis_dim[0] / 2 pairs
 * belong to axis 0, the next to axis 1, and so on. */
typedef enum {
  PULSE_ROPE_ADJACENT = 0, /* pair p is channels (2p, 2p + 1)              */
  PULSE_ROPE_HALVES = 1    /* pair p is channels (p, p + R / 2)            */
} pulse_rope_pairs;

typedef struct {
  int32_t heads;       /* heads turned alike (queries and keys together)    */
  int32_t head_dim;    /* a multiple of 8, at most 256                      */
  int32_t axes;        /* 1..4                                              */
  int32_t axis_dim[4]; /* channels per axis: even, >= 0; R a multiple of 8,
                          8 <= R <= head_dim                                */
  int32_t pairs;       /* pulse_rope_pairs                                  */
  int32_t dtype;       /* PULSE_BF16 or PULSE_F32                           */
} pulse_rope_desc;

/* Pair p of axis a of token t turns by the angle pos[t][a] * freq[p]:
 *   (x0, x1) -> (x0 cos - x1 sin, x0 sin + x1 cos),
 * or by its negative with `backward` (the gradient: dout -> din).  pos is
 * fp32 [tokens][axes], freq fp32 [R / 2].  The angle is formed and reduced in
 * 64 bits, the turn computed in 32 and rounded once.  Channels beyond R are
 * copied.  y may be x itself (same pointer and strides); otherwise they must
 * not overlap.  tokens >= 0. */
pulse_status pulse_rope(const pulse_rope_desc* desc, int32_t tokens, int32_t backward,
                        const pulse_heads* x, const float* pos, const float* freq,
                        const pulse_heads* y, void* stream);

/* ---- masks ---------------------------------------------------------------- */

/* Query row i attends keys lo <= j < hi (none if hi <= lo).  pos is the row's
 * place on the key axis, from which distances |pos - j| are measured; doc is
 * the row's document, -1 for padding. */
typedef struct {
  int32_t lo, hi, pos, doc;
} pulse_mask_row;

typedef struct {
  int32_t queries; /* query rows Tq, 0..2^24                                */
  int32_t keys;    /* keys Tk, 0..2^24                                      */
  int32_t docs;    /* documents, 0..2^20                                    */
  int32_t causal;  /* 0: a row sees its whole document; 1: the keys up to its
                      own place, and the document's prefix                   */
} pulse_mask_desc;

/* Bytes of a mask: pulse_mask_row[Tq], then a table over tiles of rows that
 * the attention kernels read. */
pulse_status pulse_mask_sizes(const pulse_mask_desc* desc, size_t* bytes);

/* Document d holds query rows [q_offsets[d], q_offsets[d + 1]) and keys
 * [k_offsets[d], k_offsets[d + 1]) (k_offsets NULL: the same; needs Tq ==
 * Tk).  Offsets are int32 [docs + 1], ascending from 0; documents may be
 * empty, and rows from the last offset on are padding and attend nothing.
 * Row r of a document with nq rows and nk keys is placed at key r + nk - nq
 * of it, so that the last row stands at the last key.  With `causal` it sees
 * the document's keys up to its place, and the first prefix[d] keys (prefix:
 * int32 [docs] or NULL for none; PULSE_E_INVALID_ARG without `causal`).
 * Rows that see nothing get lo = hi = 0.  `mask` is 16-byte aligned. */
pulse_status pulse_mask_build(const pulse_mask_desc* desc, const int32_t* q_offsets,
                              const int32_t* k_offsets, const int32_t* prefix, void* mask,
                              size_t mask_bytes, void* stream);

/* A mask from the caller's own rows (windows, padding, any interval per row;
 * docs and causal of the descriptor are not used): lo and hi are clamped to
 * [0, Tk], and rows that see nothing get lo = hi = 0.  `rows` may be `mask`
 * itself. */
pulse_status pulse_mask_from_rows(const pulse_mask_desc* desc, const pulse_mask_row* rows,
                                  void* mask, size_t mask_bytes, void* stream);

/* ---- attention -------------------------------------------------------------- */

typedef struct {
  int32_t queries, keys;   /* Tq, Tk as in the mask                          */
  int32_t heads, kv_heads; /* query head h reads key head h / (heads /
                              kv_heads); 1 <= kv_heads, dividing heads <= 1024;
                              Tq heads and Tk kv_heads at most 2^30          */
  int32_t head_dim;        /* a multiple of 8, 8..128                        */
  float scale;             /* of the scores (finite)                         */
  float cap;               /* 0: none; else scores become cap tanh(s / cap)  */
  int32_t dtype;           /* PULSE_BF16 only                                */
} pulse_attn_desc;

/* Workspace bytes of a forward and of a backward call (either may be NULL). */
pulse_status pulse_attn_sizes(const pulse_attn_desc* desc, size_t* forward_bytes,
                              size_t* backward_bytes);

/* z_ij = scale q_i . k_j, capped, minus slopes[h] |pos_i - j| (slopes fp32
 * [heads] or NULL; they are constants of the model and get no gradient);
 * p = softmax over the keys that row i attends; o_i = sum_j p_ij v_j.  A row
 * that attends nothing gives o = 0.  Keys a row does not attend do not reach
 * it, NaN and infinities included; what it attends does, here and in the
 * gradients: where the formula gives no finite value, neither do they.
 * lse [heads][Tq] receives log sum_j exp(z_ij), -inf for empty rows.  o_low
 * (bf16 [Tq][heads][head_dim], contiguous, 16-byte aligned, or NULL) receives
 * what the rounding of o left out, for the backward.  Scores, sums and
 * accumulators are fp32; p is rounded to bf16 as the operand of p v.  `mask`
 * is the buffer filled by pulse_mask_build or _from_rows with the same Tq and
 * Tk.  Outputs must not overlap inputs.  The workspace is 256-byte aligned
 * (NULL if it needs 0). */
pulse_status pulse_attn_forward(const pulse_attn_desc* desc, const pulse_heads* q,
                                const pulse_heads* k, const pulse_heads* v, const void* mask,
                                const float* slopes, const pulse_heads* o, float* lse,
                                void* o_low, void* workspace, size_t workspace_bytes, void* stream);

/* Gradients from dout, the forward's inputs, its o, lse and o_low (NULL: o as
 * rounded stands for the output in rowsum(dout o), which costs dq and dk about
 * a tenth of their accuracy).  ds is rounded to bf16 as an operand.  dk and dv
 * sum over the query heads that share a key head; keys nobody attends get 0,
 * rows that attend nothing get dq = 0 and give nothing.  `mask` still holds what
 * the forward ran under: pulse_mask_build and _from_rows overwrite a mask in
 * place, so batches in flight need one each. */
pulse_status pulse_attn_backward(const pulse_attn_desc* desc, const pulse_heads* dout,
                                 const pulse_heads* q, const pulse_heads* k,
                                 const pulse_heads* v, const pulse_heads* o, const float* lse,
                                 const void* o_low, const void* mask, const float* slopes,
                                 const pulse_heads* dq, const pulse_heads* dk,
                                 const pulse_heads* dv, void* workspace, size_t workspace_bytes,
                                 void* stream);

/* ---- gradient norm and clipping ------------------------------------------- */

typedef struct pulse_clip pulse_clip; /* opaque, library-owned */

typedef struct {
  const void* grad; /* n elements, aligned to their type                    */
  void* out;        /* receives the clipped gradient; may be grad itself    */
  int64_t n;        /* >= 0                                                 */
  int32_t dtype;    /* of grad and out                                      */
} pulse_clip_tensor;

/* A set of up to 2^20 gradient tensors whose addresses stay the same from
 * step to step (a stage's gradients are such).  No two outputs may overlap,
 * nor an output and another tensor's gradient. */
pulse_status pulse_clip_create(const pulse_clip_tensor* tensors, int32_t count,
                               pulse_clip** out);
void pulse_clip_destroy(pulse_clip* clip);
pulse_status pulse_clip_sizes(const pulse_clip* clip, size_t* workspace_bytes);

/* Bind the workspace (256-byte aligned) and copy the tensors' table into it
 * on `stream`.  Not to be captured into a graph. */
pulse_status pulse_clip_bind(pulse_clip* clip, void* workspace, size_t workspace_bytes,
                             void* stream);

/* norm = sqrt(sum of squares over all tensors), summed in 64 bits;
 * out = grad * min(1, max_norm / (norm + eps)), the factor in fp32, rounded
 * once.  norm[0] (fp32, device) receives the norm.  Where the factor is 1,
 * an output that is its own gradient is not touched.  A norm that is not
 * finite gives what the formula gives: NaN makes every output NaN, and an
 * infinite norm makes finite gradients 0.  max_norm >= 0, eps >= 0. */
pulse_status pulse_clip_run(pulse_clip* clip, float max_norm, float eps, float* norm,
                            void* stream);

#ifdef __cplusplus
}
#endif

#endif /* PULSE_OPS_H */
