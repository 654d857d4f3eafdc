// C ABI of the packed-sequence operators (pulse_ops.h): checks of the host
// arguments, then one launcher call each (okernels.hpp).
#include <cmath>
#include <new>
#include <vector>

#include "ocheck.hpp"

using namespace pulse;

namespace {

constexpr int MAX_HEADS = 1024;

// a [tokens][heads][dim] view; `out`: written, so its elements are distinct
pulse_status check_heads(const pulse_heads* x, const char* name, int tokens, int heads, int dim,
                         int esz, bool out) {
  if (!x) return ofail(PULSE_E_INVALID_ARG, "%s is NULL", name);
  if (tokens == 0) return PULSE_OK;  // nothing is read or written
  if (!x->ptr) return ofail(PULSE_E_INVALID_ARG, "%s.ptr is NULL", name);
  const int64_t ts = x->token_stride, hs = x->head_stride;
  if (!aligned(x->ptr, 16)) return ofail(PULSE_E_INVALID_ARG, "%s is not 16-byte aligned", name);
  if (ts < 0 || hs < 0 || ts > INT64_C(1) << 40 || hs > INT64_C(1) << 40)
    return ofail(PULSE_E_INVALID_ARG, "%s has a stride below 0 or above 2^40", name);
  if (ts * esz % 16 || hs * esz % 16)
    return ofail(PULSE_E_INVALID_ARG, "%s has a stride that is not a multiple of 16 bytes", name);
  // no more than an address space, so that neither these sums nor the kernels'
  // offsets wrap around
  if ((tokens > 1 && ts > MAX_EXTENT / (tokens - 1)) ||
      (heads > 1 && hs > MAX_EXTENT / (heads - 1)))
    return ofail(PULSE_E_INVALID_ARG, "%s extends over more than 2^47 elements", name);
  if (out) {
    const bool th = (heads == 1 || hs >= dim) && (tokens == 1 || ts >= (heads - 1) * hs + dim);
    const bool ht = (tokens == 1 || ts >= dim) &&
                    (heads == 1 || hs >= (int64_t)(tokens - 1) * ts + dim);
    if (!th && !ht)
      return ofail(PULSE_E_INVALID_ARG, "%s: tokens or heads overlap with these strides", name);
  }
  return PULSE_OK;
}

pulse_status check_rope(const pulse_rope_desc* d) {
  if (!d) return ofail(PULSE_E_INVALID_ARG, "desc is NULL");
  if (d->dtype != PULSE_F32 && d->dtype != PULSE_BF16)
    return ofail(PULSE_E_INVALID_ARG, "dtype must be PULSE_F32 or PULSE_BF16");
  if (d->pairs != PULSE_ROPE_ADJACENT && d->pairs != PULSE_ROPE_HALVES)
    return ofail(PULSE_E_INVALID_ARG, "pairs must be PULSE_ROPE_ADJACENT or PULSE_ROPE_HALVES");
  if (d->heads < 1 || d->heads > MAX_HEADS)
    return ofail(PULSE_E_SHAPE, "heads must be in [1, %d]", MAX_HEADS);
  if (d->head_dim < 8 || d->head_dim > 256 || d->head_dim % 8)
    return ofail(PULSE_E_SHAPE, "head_dim must be a multiple of 8 in [8, 256]");
  if (d->axes < 1 || d->axes > 4) return ofail(PULSE_E_SHAPE, "axes must be in [1, 4]");
  int r = 0;
  for (int i = 0; i < d->axes; ++i) {
    if (d->axis_dim[i] < 0 || d->axis_dim[i] > 256 || d->axis_dim[i] % 2)
      return ofail(PULSE_E_SHAPE, "axis_dim[%d] must be even and in [0, 256]", i);
    r += d->axis_dim[i];
  }
  if (r < 8 || r % 8 || r > d->head_dim)
    return ofail(PULSE_E_SHAPE, "the axes' channels must sum to a multiple of 8 in [8, head_dim]");
  return PULSE_OK;
}

pulse_status check_mask(const pulse_mask_desc* d) {
  if (!d) return ofail(PULSE_E_INVALID_ARG, "desc is NULL");
  if (d->queries < 0 || d->queries > MAX_TOKENS || d->keys < 0 || d->keys > MAX_TOKENS)
    return ofail(PULSE_E_SHAPE, "queries and keys must be in [0, 2^24]");
  if (d->docs < 0 || d->docs > 1 << 20) return ofail(PULSE_E_SHAPE, "docs must be in [0, 2^20]");
  if (d->causal != 0 && d->causal != 1) return ofail(PULSE_E_INVALID_ARG, "causal must be 0 or 1");
  return PULSE_OK;
}

pulse_status check_mask_buffer(const pulse_mask_desc* d, const void* mask, size_t bytes) {
  if (d->queries == 0) return PULSE_OK;
  if (!mask) return ofail(PULSE_E_INVALID_ARG, "mask is NULL");
  if (!aligned(mask, 16)) return ofail(PULSE_E_INVALID_ARG, "mask is not 16-byte aligned");
  if (bytes < mask_bytes(d->queries))
    return ofail(PULSE_E_INVALID_ARG, "mask has %zu bytes, needs %zu", bytes,
                 mask_bytes(d->queries));
  return PULSE_OK;
}

pulse_status check_attn(const pulse_attn_desc* d) {
  if (!d) return ofail(PULSE_E_INVALID_ARG, "desc is NULL");
  if (d->dtype != PULSE_BF16) return ofail(PULSE_E_SHAPE, "attention runs bf16 only");
  if (d->queries < 0 || d->queries > MAX_TOKENS || d->keys < 0 || d->keys > MAX_TOKENS)
    return ofail(PULSE_E_SHAPE, "queries and keys must be in [0, 2^24]");
  if (d->heads < 1 || d->heads > MAX_HEADS || d->kv_heads < 1 || d->heads % d->kv_heads)
    return ofail(PULSE_E_SHAPE, "heads must be in [1, %d] and a multiple of kv_heads", MAX_HEADS);
  // a launch has less than 2^32 threads
  if ((int64_t)d->queries * d->heads > 1 << 30 || (int64_t)d->keys * d->kv_heads > 1 << 30)
    return ofail(PULSE_E_SHAPE, "queries * heads and keys * kv_heads must be at most 2^30");
  if (d->head_dim < 8 || d->head_dim > 128 || d->head_dim % 8)
    return ofail(PULSE_E_SHAPE, "head_dim must be a multiple of 8 in [8, 128]");
  if (!std::isfinite(d->scale)) return ofail(PULSE_E_INVALID_ARG, "scale must be finite");
  if (!(d->cap >= 0.f) || !std::isfinite(d->cap))
    return ofail(PULSE_E_INVALID_ARG, "cap must be finite and >= 0");
  return PULSE_OK;
}

// what forward and backward share
pulse_status check_attn_inputs(const pulse_attn_desc* d, const pulse_heads* q,
                               const pulse_heads* k, const pulse_heads* v, const void* mask,
                               const float* slopes) {
  OCHK(check_heads(q, "q", d->queries, d->heads, d->head_dim, 2, false));
  OCHK(check_heads(k, "k", d->keys, d->kv_heads, d->head_dim, 2, false));
  OCHK(check_heads(v, "v", d->keys, d->kv_heads, d->head_dim, 2, false));
  if (d->queries && !mask) return ofail(PULSE_E_INVALID_ARG, "mask is NULL");
  if (!aligned(mask, 16)) return ofail(PULSE_E_INVALID_ARG, "mask is not 16-byte aligned");
  if (!aligned(slopes, 4)) return ofail(PULSE_E_INVALID_ARG, "slopes is not 4-byte aligned");
  return PULSE_OK;
}

MattnArgs attn_args(const pulse_attn_desc* d, const pulse_heads* q, const pulse_heads* k,
                    const pulse_heads* v, const void* mask, const float* slopes, void* ws) {
  MattnArgs a{};
  a.Tq = d->queries, a.Tk = d->keys, a.H = d->heads, a.KV = d->kv_heads, a.hd = d->head_dim;
  a.scale = d->scale, a.cap = d->cap;
  a.q = *q, a.k = *k, a.v = *v;
  a.mask = mask, a.slopes = slopes, a.ws = ws;
  return a;
}

}  // namespace

struct pulse_clip {
  std::vector<ClipChunk> chunks;
  char* ws = nullptr;
};

namespace {
// workspace: partial sums, then the chunk table
constexpr size_t CLIP_TABLE = CLIP_BLOCKS * sizeof(double);
size_t clip_bytes(const pulse_clip* c) { return CLIP_TABLE + c->chunks.size() * sizeof(ClipChunk); }
}  // namespace

extern "C" {

pulse_status pulse_rope(const pulse_rope_desc* desc, int32_t tokens, int32_t backward,
                        const pulse_heads* x, const float* pos, const float* freq,
                        const pulse_heads* y, void* stream) {
  OCHK(check_rope(desc));
  if (tokens < 0 || tokens > MAX_TOKENS)
    return ofail(PULSE_E_SHAPE, "tokens must be in [0, 2^24]");
  const int esz = desc->dtype == PULSE_BF16 ? 2 : 4;
  OCHK(check_heads(x, "x", tokens, desc->heads, desc->head_dim, esz, false));
  OCHK(check_heads(y, "y", tokens, desc->heads, desc->head_dim, esz, true));
  if (tokens && (!pos || !freq)) return ofail(PULSE_E_INVALID_ARG, "pos or freq is NULL");
  if (!aligned(pos, 4) || !aligned(freq, 4))
    return ofail(PULSE_E_INVALID_ARG, "pos or freq is not 4-byte aligned");
  return launched(launch_rope(*desc, tokens, backward != 0, *x, pos, freq, *y,
                              static_cast<hipStream_t>(stream)),
                  "rope");
}

pulse_status pulse_mask_sizes(const pulse_mask_desc* desc, size_t* bytes) {
  OCHK(check_mask(desc));
  if (!bytes) return ofail(PULSE_E_INVALID_ARG, "bytes is NULL");
  *bytes = mask_bytes(desc->queries);
  return PULSE_OK;
}

pulse_status pulse_mask_build(const pulse_mask_desc* desc, const int32_t* q_offsets,
                              const int32_t* k_offsets, const int32_t* prefix, void* mask,
                              size_t mask_size, void* stream) {
  OCHK(check_mask(desc));
  OCHK(check_mask_buffer(desc, mask, mask_size));
  if (!q_offsets) return ofail(PULSE_E_INVALID_ARG, "q_offsets is NULL");
  if (!k_offsets && desc->queries != desc->keys)
    return ofail(PULSE_E_INVALID_ARG, "k_offsets is NULL and queries != keys");
  if (prefix && !desc->causal)
    return ofail(PULSE_E_INVALID_ARG, "a prefix needs a causal mask");
  if (!aligned(q_offsets, 4) || !aligned(k_offsets, 4) || !aligned(prefix, 4))
    return ofail(PULSE_E_INVALID_ARG, "offsets or prefix is not 4-byte aligned");
  return launched(launch_mask_build(*desc, q_offsets, k_offsets, prefix, mask,
                                    static_cast<hipStream_t>(stream)),
                  "mask");
}

pulse_status pulse_mask_from_rows(const pulse_mask_desc* desc, const pulse_mask_row* rows,
                                  void* mask, size_t mask_size, void* stream) {
  OCHK(check_mask(desc));
  OCHK(check_mask_buffer(desc, mask, mask_size));
  if (desc->queries && !rows) return ofail(PULSE_E_INVALID_ARG, "rows is NULL");
  if (!aligned(rows, 16)) return ofail(PULSE_E_INVALID_ARG, "rows is not 16-byte aligned");
  return launched(launch_mask_rows(*desc, rows, mask, static_cast<hipStream_t>(stream)), "mask");
}

pulse_status pulse_attn_sizes(const pulse_attn_desc* desc, size_t* forward_bytes,
                              size_t* backward_bytes) {
  OCHK(check_attn(desc));
  if (forward_bytes) *forward_bytes = mattn_fwd_bytes(*desc);
  if (backward_bytes) *backward_bytes = mattn_bwd_bytes(*desc);
  return PULSE_OK;
}

pulse_status pulse_attn_forward(const pulse_attn_desc* desc, const pulse_heads* q,
                                const pulse_heads* k, const pulse_heads* v, const void* mask,
                                const float* slopes, const pulse_heads* o, float* lse,
                                void* o_low, void* workspace, size_t workspace_bytes, void* stream) {
  OCHK(check_attn(desc));
  OCHK(check_attn_inputs(desc, q, k, v, mask, slopes));
  OCHK(check_heads(o, "o", desc->queries, desc->heads, desc->head_dim, 2, true));
  if (desc->queries && !lse) return ofail(PULSE_E_INVALID_ARG, "lse is NULL");
  if (!aligned(lse, 4)) return ofail(PULSE_E_INVALID_ARG, "lse is not 4-byte aligned");
  if (!aligned(o_low, 16)) return ofail(PULSE_E_INVALID_ARG, "o_low is not 16-byte aligned");
  OCHK(check_ws(workspace, workspace_bytes, mattn_fwd_bytes(*desc)));
  MattnArgs a = attn_args(desc, q, k, v, mask, slopes, workspace);
  a.o = *o;
  a.lse = lse;
  a.o_low = o_low;
  return launched(launch_mattn_fwd(a, static_cast<hipStream_t>(stream)), "attention forward");
}

pulse_status pulse_attn_backward(const pulse_attn_desc* desc, const pulse_heads* dout,
                                 const pulse_heads* q, const pulse_heads* k,
                                 const pulse_heads* v, const pulse_heads* o, const float* lse,
                                 const void* o_low, const void* mask, const float* slopes,
                                 const pulse_heads* dq, const pulse_heads* dk,
                                 const pulse_heads* dv, void* workspace, size_t workspace_bytes,
                                 void* stream) {
  OCHK(check_attn(desc));
  OCHK(check_attn_inputs(desc, q, k, v, mask, slopes));
  OCHK(check_heads(dout, "dout", desc->queries, desc->heads, desc->head_dim, 2, false));
  OCHK(check_heads(o, "o", desc->queries, desc->heads, desc->head_dim, 2, false));
  OCHK(check_heads(dq, "dq", desc->queries, desc->heads, desc->head_dim, 2, true));
  OCHK(check_heads(dk, "dk", desc->keys, desc->kv_heads, desc->head_dim, 2, true));
  OCHK(check_heads(dv, "dv", desc->keys, desc->kv_heads, desc->head_dim, 2, true));
  if (desc->queries && !lse) return ofail(PULSE_E_INVALID_ARG, "lse is NULL");
  if (!aligned(lse, 4)) return ofail(PULSE_E_INVALID_ARG, "lse is not 4-byte aligned");
  if (!aligned(o_low, 16)) return ofail(PULSE_E_INVALID_ARG, "o_low is not 16-byte aligned");
  OCHK(check_ws(workspace, workspace_bytes, mattn_bwd_bytes(*desc)));
  MattnArgs a = attn_args(desc, q, k, v, mask, slopes, workspace);
  a.o = *o, a.dout = *dout, a.dq = *dq, a.dk = *dk, a.dv = *dv;
  a.lse = const_cast<float*>(lse);
  a.o_low = const_cast<void*>(o_low);
  return launched(launch_mattn_bwd(a, static_cast<hipStream_t>(stream)), "attention backward");
}

pulse_status pulse_clip_create(const pulse_clip_tensor* tensors, int32_t count,
                               pulse_clip** out) {
  if (!out) return ofail(PULSE_E_INVALID_ARG, "out is NULL");
  *out = nullptr;
  if (count < 0 || count > 1 << 20) return ofail(PULSE_E_SHAPE, "count must be in [0, 2^20]");
  if (count && !tensors) return ofail(PULSE_E_INVALID_ARG, "tensors is NULL");
  int64_t chunks = 0;
  for (int32_t i = 0; i < count; ++i) {
    const pulse_clip_tensor& t = tensors[i];
    if (t.dtype != PULSE_F32 && t.dtype != PULSE_BF16)
      return ofail(PULSE_E_INVALID_ARG, "tensor %d: dtype must be PULSE_F32 or PULSE_BF16", i);
    if (t.n < 0 || t.n > INT64_C(1) << 38)
      return ofail(PULSE_E_SHAPE, "tensor %d: n must be in [0, 2^38]", i);
    if (t.n && (!t.grad || !t.out))
      return ofail(PULSE_E_INVALID_ARG, "tensor %d: grad or out is NULL", i);
    const uintptr_t esz = t.dtype == PULSE_BF16 ? 2 : 4;
    if (!aligned(t.grad, esz) || !aligned(t.out, esz))
      return ofail(PULSE_E_INVALID_ARG, "tensor %d is not aligned to its type", i);
    chunks += (t.n + CLIP_CHUNK - 1) / CLIP_CHUNK;
  }
  if (chunks > 1 << 26) return ofail(PULSE_E_SHAPE, "more than 2^26 chunks of gradients");
  try {
    pulse_clip* c = new pulse_clip;
    *out = c;
    c->chunks.reserve(chunks);
    for (int32_t i = 0; i < count; ++i) {
      const pulse_clip_tensor& t = tensors[i];
      const int64_t esz = t.dtype == PULSE_BF16 ? 2 : 4;
      for (int64_t a = 0; a < t.n; a += CLIP_CHUNK) {
        const int64_t n = t.n - a < CLIP_CHUNK ? t.n - a : CLIP_CHUNK;
        c->chunks.push_back(ClipChunk{static_cast<const char*>(t.grad) + a * esz,
                                      static_cast<char*>(t.out) + a * esz, (int32_t)n, t.dtype});
      }
    }
  } catch (const std::bad_alloc&) {
    delete *out;
    *out = nullptr;
    return ofail(PULSE_E_INVALID_ARG, "out of host memory");
  }
  return PULSE_OK;
}

void pulse_clip_destroy(pulse_clip* clip) { delete clip; }

pulse_status pulse_clip_sizes(const pulse_clip* clip, size_t* workspace_bytes) {
  if (!clip || !workspace_bytes) return ofail(PULSE_E_INVALID_ARG, "clip or result is NULL");
  *workspace_bytes = clip_bytes(clip);
  return PULSE_OK;
}

pulse_status pulse_clip_bind(pulse_clip* clip, void* workspace, size_t workspace_bytes,
                             void* stream) {
  if (!clip) return ofail(PULSE_E_INVALID_ARG, "clip is NULL");
  OCHK(check_ws(workspace, workspace_bytes, clip_bytes(clip)));
  char* ws = static_cast<char*>(workspace);
  if (!clip->chunks.empty())
    OCHK(launched(hipMemcpyAsync(ws + CLIP_TABLE, clip->chunks.data(),
                                 clip->chunks.size() * sizeof(ClipChunk), hipMemcpyHostToDevice,
                                 static_cast<hipStream_t>(stream)),
                  "copy of the tensor table"));
  clip->ws = ws;
  return PULSE_OK;
}

pulse_status pulse_clip_run(pulse_clip* clip, float max_norm, float eps, float* norm,
                            void* stream) {
  if (!clip) return ofail(PULSE_E_INVALID_ARG, "clip is NULL");
  if (!clip->ws) return ofail(PULSE_E_NOT_BOUND, "clip has no bound workspace");
  if (!(max_norm >= 0.f)) return ofail(PULSE_E_INVALID_ARG, "max_norm must be >= 0");
  if (!(eps >= 0.f)) return ofail(PULSE_E_INVALID_ARG, "eps must be >= 0");
  if (!norm || !aligned(norm, 4))
    return ofail(PULSE_E_INVALID_ARG, "norm is NULL or not 4-byte aligned");
  return launched(launch_clip(reinterpret_cast<const ClipChunk*>(clip->ws + CLIP_TABLE),
                              (int)clip->chunks.size(), reinterpret_cast<double*>(clip->ws),
                              max_norm, eps, norm, static_cast<hipStream_t>(stream)),
                  "gradient clipping");
}

}  // extern "C"
