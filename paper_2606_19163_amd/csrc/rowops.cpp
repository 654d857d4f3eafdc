// C ABI of the row operators (pulse_ops.h: pulse_norm, pulse_keep,
// pulse_lin8): checks of the host arguments, then one launcher call each
// (okernels.hpp).
#include <cmath>

#include "ocheck.hpp"

using namespace pulse;

namespace {

constexpr int MAX_ROWS = 1 << 23;  // a launch of a block per row has less than 2^32 threads

pulse_status check_tokens(int tokens) {
  if (tokens < 0 || tokens > MAX_ROWS) return ofail(PULSE_E_SHAPE, "tokens must be in [0, 2^23]");
  return PULSE_OK;
}

bool a_dtype(int d) { return d == PULSE_F32 || d == PULSE_BF16; }
int size_of(int dtype) { return dtype == PULSE_BF16 ? 2 : 4; }

// a [tokens][channels] view; `out`: written, so its rows are distinct
pulse_status check_rows(const pulse_rows* x, const char* name, int tokens, int channels, int esz,
                        bool out) {
  if (!x) return ofail(PULSE_E_INVALID_ARG, "%s is NULL", name);
  if (tokens == 0) return PULSE_OK;  // nothing is read or written
  if (!x->ptr) return ofail(PULSE_E_INVALID_ARG, "%s.ptr is NULL", name);
  if (!aligned(x->ptr, 16)) return ofail(PULSE_E_INVALID_ARG, "%s is not 16-byte aligned", name);
  const int64_t ts = x->token_stride;
  if (ts < 0 || ts > INT64_C(1) << 40)
    return ofail(PULSE_E_INVALID_ARG, "%s has a stride below 0 or above 2^40", name);
  if (ts * esz % 16)
    return ofail(PULSE_E_INVALID_ARG, "%s has a stride that is not a multiple of 16 bytes", name);
  if (tokens > 1 && ts > MAX_EXTENT / (tokens - 1))
    return ofail(PULSE_E_INVALID_ARG, "%s extends over more than 2^47 elements", name);
  if (out && tokens > 1 && ts < channels)
    return ofail(PULSE_E_INVALID_ARG, "%s: rows overlap with this stride", name);
  return PULSE_OK;
}

// Bytes [begin, end) of a view.
struct Span {
  uintptr_t begin, end;
};
Span span_of(const pulse_rows* x, int tokens, int64_t channels, int esz) {
  if (!x || !tokens) return Span{0, 0};
  const uintptr_t p = reinterpret_cast<uintptr_t>(x->ptr);
  return Span{p, p + ((uintptr_t)(tokens - 1) * x->token_stride + channels) * esz};
}
bool meet(Span a, Span b) { return a.begin < b.end && b.begin < a.end; }

// Two views with rows of `row` bytes, `step` bytes apart, share no byte: their
// spans are apart, or they are columns of the same rows that do not touch.
bool apart(Span a, int64_t step_a, int64_t row_a, Span b, int64_t step_b, int64_t row_b) {
  if (!meet(a, b)) return true;
  if (step_a != step_b || step_a <= 0) return false;
  const int64_t d = ((int64_t)(b.begin - a.begin) % step_a + step_a) % step_a;
  return d >= row_a && d + row_b <= step_a;
}

struct View {
  const pulse_rows* x;
  const char* name;
  int tokens;
  int64_t channels;
  int esz;
};
bool same(const View& a, const View& b) {
  return a.x->ptr == b.x->ptr && a.esz == b.esz &&
         (a.tokens <= 1 || a.x->token_stride == b.x->token_stride);
}
// `out` does not overlap `in`, unless `alias` and it is the same view
pulse_status check_apart(const View& out, const View& in, bool alias) {
  if (!out.x || !in.x || !out.tokens || !in.tokens) return PULSE_OK;
  if (alias && same(out, in)) return PULSE_OK;
  const auto step = [](const View& v) {
    return v.tokens > 1 ? v.x->token_stride * v.esz : INT64_C(0);
  };
  if (!apart(span_of(out.x, out.tokens, out.channels, out.esz), step(out),
             out.channels * out.esz, span_of(in.x, in.tokens, in.channels, in.esz), step(in),
             in.channels * in.esz))
    return ofail(PULSE_E_INVALID_ARG, "%s overlaps %s", out.name, in.name);
  return PULSE_OK;
}

// ---- norms ---------------------------------------------------------------------

pulse_status check_norm(const pulse_norm_desc* d) {
  if (!d) return ofail(PULSE_E_INVALID_ARG, "desc is NULL");
  if (d->channels < 8 || d->channels > 8192 || d->channels % 8)
    return ofail(PULSE_E_SHAPE, "channels must be a multiple of 8 in [8, 8192]");
  if (d->docs < 1 || d->docs > 1 << 20) return ofail(PULSE_E_SHAPE, "docs must be in [1, 2^20]");
  for (int k : {d->pre, d->post})
    if (k != PULSE_NORM_NONE && k != PULSE_NORM_LAYER && k != PULSE_NORM_RMS)
      return ofail(PULSE_E_INVALID_ARG, "pre and post must be PULSE_NORM_NONE, _LAYER or _RMS");
  if (d->branch != 0 && d->branch != 1) return ofail(PULSE_E_INVALID_ARG, "branch must be 0 or 1");
  if (!d->branch && (d->post || !d->pre))
    return ofail(PULSE_E_INVALID_ARG, "without a branch there is a norm before and none after");
  if (!(d->eps >= 0.f) || !std::isfinite(d->eps))
    return ofail(PULSE_E_INVALID_ARG, "eps must be finite and >= 0");
  if (!std::isfinite(d->residual_scale))
    return ofail(PULSE_E_INVALID_ARG, "residual_scale must be finite");
  if (!a_dtype(d->dtype) || (d->stream_dtype != PULSE_F32 && d->stream_dtype != d->dtype))
    return ofail(PULSE_E_INVALID_ARG,
                 "dtype must be PULSE_F32 or PULSE_BF16, and stream_dtype PULSE_F32 or the same");
  return PULSE_OK;
}

pulse_status check_vector(const void* p, const char* name, bool may) {
  if (!p) return PULSE_OK;
  if (!may) return ofail(PULSE_E_INVALID_ARG, "%s is given, but the joint has no use for it", name);
  if (!aligned(p, 16)) return ofail(PULSE_E_INVALID_ARG, "%s is not 16-byte aligned", name);
  return PULSE_OK;
}

pulse_status check_cond(const float* p, int64_t stride, const char* name, bool may, int docs) {
  OCHK(check_vector(p, name, may));
  if (!p || docs == 1) return PULSE_OK;
  if (stride < 0 || stride > INT64_C(1) << 40 || stride % 4)
    return ofail(PULSE_E_INVALID_ARG,
                 "%s has a stride that is not a multiple of 4 in [0, 2^40]", name);
  return PULSE_OK;
}

pulse_status check_params(const pulse_norm_desc* d, const pulse_norm_params* p) {
  if (!p) return ofail(PULSE_E_INVALID_ARG, "params is NULL");
  if (!p->offsets && d->docs != 1)
    return ofail(PULSE_E_INVALID_ARG, "offsets is NULL and docs is not 1");
  if (!aligned(p->offsets, 4)) return ofail(PULSE_E_INVALID_ARG, "offsets is not 4-byte aligned");
  OCHK(check_cond(p->gate, p->gate_stride, "gate", d->branch, d->docs));
  OCHK(check_cond(p->scale, p->scale_stride, "scale", d->pre, d->docs));
  OCHK(check_cond(p->shift, p->shift_stride, "shift", d->pre, d->docs));
  OCHK(check_vector(p->weight, "weight", d->pre));
  OCHK(check_vector(p->bias, "bias", d->pre));
  OCHK(check_vector(p->post_weight, "post_weight", d->post));
  return PULSE_OK;
}

// What a joint applies, and its gradients, as views (those that are not there have
// no rows).
struct ParamViews {
  pulse_rows r[7];
  View v[7];
  ParamViews(const pulse_norm_desc* d, const pulse_norm_params* p) {
    const int docs = d->docs;
    const int64_t C = d->channels;
    set(0, p->offsets, 0, "offsets", 1, (int64_t)docs + 1);
    set(1, p->gate, p->gate_stride, "gate", docs, C);
    set(2, p->scale, p->scale_stride, "scale", docs, C);
    set(3, p->shift, p->shift_stride, "shift", docs, C);
    set(4, p->weight, 0, "weight", 1, C);
    set(5, p->bias, 0, "bias", 1, C);
    set(6, p->post_weight, 0, "post_weight", 1, C);
  }
  ParamViews(const pulse_norm_desc* d, const pulse_norm_grads* g) {
    const int64_t C = d->channels, many = C * d->docs;
    set(0, g->dgate, 0, "dgate", 1, many);
    set(1, g->dscale, 0, "dscale", 1, many);
    set(2, g->dshift, 0, "dshift", 1, many);
    set(3, g->dweight, 0, "dweight", 1, C);
    set(4, g->dbias, 0, "dbias", 1, C);
    set(5, g->dpost_weight, 0, "dpost_weight", 1, C);
    set(6, nullptr, 0, "", 0, 0);
  }
  ParamViews(const ParamViews&) = delete;
  void set(int i, const void* p, int64_t stride, const char* name, int rows, int64_t channels) {
    r[i] = pulse_rows{const_cast<void*>(p), stride};
    v[i] = View{&r[i], name, p ? rows : 0, channels, 4};
  }
};

pulse_status check_apart(const View& out, const ParamViews& in) {
  for (const View& v : in.v) OCHK(check_apart(out, v, false));
  return PULSE_OK;
}

NormArgs norm_args(const pulse_norm_desc* d, int tokens, const pulse_norm_params* p) {
  NormArgs a{};
  a.tokens = tokens, a.C = d->channels, a.docs = d->docs;
  a.pre = d->pre, a.post = d->post, a.branch = d->branch;
  a.dtype = d->dtype, a.stream_dtype = d->stream_dtype;
  a.eps = d->eps, a.r = d->residual_scale;
  a.off = p->offsets;
  a.gate = p->gate, a.scale = p->scale, a.shift = p->shift;
  a.gate_t = p->gate_stride, a.scale_t = p->scale_stride, a.shift_t = p->shift_stride;
  a.weight = p->weight, a.bias = p->bias, a.post_weight = p->post_weight;
  return a;
}

// ---- kept rows ------------------------------------------------------------------

pulse_status check_keep(const pulse_keep_desc* d) {
  if (!d) return ofail(PULSE_E_INVALID_ARG, "desc is NULL");
  if (d->channels < 8 || d->channels > 65536 || d->channels % 8)
    return ofail(PULSE_E_SHAPE, "channels must be a multiple of 8 in [8, 65536]");
  if (d->act < PULSE_ACT_NONE || d->act > PULSE_ACT_SILU)
    return ofail(PULSE_E_INVALID_ARG, "act must be PULSE_ACT_NONE, _GELU or _SILU");
  if (!a_dtype(d->dtype))
    return ofail(PULSE_E_INVALID_ARG, "dtype must be PULSE_F32 or PULSE_BF16");
  return PULSE_OK;
}

pulse_status check_kept(const pulse_keep_desc* d, int tokens, const void* kept, size_t bytes,
                        const char* name) {
  if (tokens == 0) return PULSE_OK;
  if (!kept) return ofail(PULSE_E_INVALID_ARG, "%s is NULL", name);
  if (!aligned(kept, 16)) return ofail(PULSE_E_INVALID_ARG, "%s is not 16-byte aligned", name);
  if (bytes < keep_bytes(d->channels, tokens))
    return ofail(PULSE_E_INVALID_ARG, "%s has %zu bytes, needs %zu", name, bytes,
                 keep_bytes(d->channels, tokens));
  return PULSE_OK;
}

// kept rows as a view of one row of bytes
pulse_rows flat(const void* p) { return pulse_rows{const_cast<void*>(p), 0}; }

struct Flat {
  pulse_rows r;
  View v;
  Flat(const void* p, size_t bytes, const char* name) : r(flat(p)) {
    // a span in units of 16 bytes, rounded up: kept rows are aligned to as much
    v = View{&r, name, p && bytes ? 1 : 0, (int64_t)((bytes + 15) / 16), 16};
  }
  Flat(const Flat&) = delete;
};

KeepArgs keep_args(const pulse_keep_desc* d, int tokens, const void* kept) {
  KeepArgs a{};
  a.tokens = tokens, a.C = d->channels, a.act = d->act, a.dtype = d->dtype;
  a.kept = const_cast<void*>(kept);
  return a;
}

// ---- 8-bit linear layers ----------------------------------------------------------

pulse_status check_lin8(const pulse_lin8_desc* d) {
  if (!d) return ofail(PULSE_E_INVALID_ARG, "desc is NULL");
  for (int n : {d->inputs, d->outputs})
    if (n < 8 || n > 65536 || n % 8)
      return ofail(PULSE_E_SHAPE, "inputs and outputs must be multiples of 8 in [8, 65536]");
  if (d->act < PULSE_ACT_NONE || d->act > PULSE_ACT_SILU)
    return ofail(PULSE_E_INVALID_ARG, "act must be PULSE_ACT_NONE, _GELU or _SILU");
  if (d->dtype != PULSE_BF16) return ofail(PULSE_E_INVALID_ARG, "dtype must be PULSE_BF16");
  return PULSE_OK;
}

pulse_status check_lin8_tokens(const pulse_lin8_desc* d, int tokens) {
  OCHK(check_tokens(tokens));
  if ((int64_t)tokens * d->outputs > INT64_C(1) << 38)
    return ofail(PULSE_E_SHAPE, "tokens * outputs must be at most 2^38");
  return PULSE_OK;
}

pulse_status check_weights(const pulse_lin8_desc* d, const void* weights, size_t bytes) {
  const size_t need = lin8_weight_bytes(d->inputs, d->outputs);
  if (!weights) return ofail(PULSE_E_INVALID_ARG, "weights is NULL");
  if (!aligned(weights, 256)) return ofail(PULSE_E_INVALID_ARG, "weights is not 256-byte aligned");
  if (bytes < need)
    return ofail(PULSE_E_INVALID_ARG, "weights has %zu bytes, needs %zu", bytes, need);
  return PULSE_OK;
}

}  // namespace

extern "C" {

pulse_status pulse_norm_sizes(const pulse_norm_desc* desc, int32_t tokens,
                              size_t* backward_bytes) {
  OCHK(check_norm(desc));
  OCHK(check_tokens(tokens));
  if (!backward_bytes) return ofail(PULSE_E_INVALID_ARG, "backward_bytes is NULL");
  *backward_bytes = norm_bwd_bytes(*desc, tokens);
  return PULSE_OK;
}

pulse_status pulse_norm_forward(const pulse_norm_desc* desc, int32_t tokens, const pulse_rows* x,
                                const pulse_rows* y, const pulse_norm_params* params,
                                const pulse_rows* h, const pulse_rows* u, void* stream) {
  OCHK(check_norm(desc));
  OCHK(check_tokens(tokens));
  OCHK(check_params(desc, params));
  const int C = desc->channels, es = size_of(desc->stream_dtype), eb = size_of(desc->dtype);
  NormArgs a = norm_args(desc, tokens, params);
  OCHK(check_rows(x, "x", tokens, C, es, false));
  a.x = x->ptr, a.xt = x->token_stride;
  const View vx{x, "x", tokens, C, es};
  View vy{nullptr, "y", tokens, C, eb}, vh{nullptr, "h", tokens, C, es};
  if (desc->branch) {
    OCHK(check_rows(y, "y", tokens, C, eb, false));
    OCHK(check_rows(h, "h", tokens, C, es, true));
    a.y = y->ptr, a.yt = y->token_stride;
    a.h = h->ptr, a.ht = h->token_stride;
    vy.x = y, vh.x = h;
    OCHK(check_apart(vh, vx, true));
    OCHK(check_apart(vh, vy, false));
  }
  if (desc->pre) {
    OCHK(check_rows(u, "u", tokens, C, eb, true));
    a.u = u->ptr, a.ut = u->token_stride;
    const View vu{u, "u", tokens, C, eb};
    OCHK(check_apart(vu, vx, false));
    OCHK(check_apart(vu, vy, true));
    OCHK(check_apart(vu, vh, false));
    OCHK(check_apart(vu, ParamViews(desc, params)));
  }
  OCHK(check_apart(vh, ParamViews(desc, params)));
  return launched(launch_norm_fwd(a, static_cast<hipStream_t>(stream)), "norm forward");
}

pulse_status pulse_norm_backward(const pulse_norm_desc* desc, int32_t tokens, const pulse_rows* du,
                                 const pulse_rows* dh, const pulse_rows* h, const pulse_rows* y,
                                 const pulse_norm_params* params, const pulse_rows* dx,
                                 const pulse_rows* dy, const pulse_norm_grads* grads,
                                 void* workspace, size_t workspace_bytes, void* stream) {
  OCHK(check_norm(desc));
  OCHK(check_tokens(tokens));
  OCHK(check_params(desc, params));
  if (!grads) return ofail(PULSE_E_INVALID_ARG, "grads is NULL");
  const int C = desc->channels, es = size_of(desc->stream_dtype), eb = size_of(desc->dtype);
  OCHK(check_vector(grads->dgate, "dgate", desc->branch));
  OCHK(check_vector(grads->dscale, "dscale", desc->pre));
  OCHK(check_vector(grads->dshift, "dshift", desc->pre));
  OCHK(check_vector(grads->dweight, "dweight", desc->pre));
  OCHK(check_vector(grads->dbias, "dbias", desc->pre));
  OCHK(check_vector(grads->dpost_weight, "dpost_weight", desc->post));
  NormArgs a = norm_args(desc, tokens, params);
  View vdu{nullptr, "du", tokens, C, eb}, vdh{nullptr, "dh", tokens, C, es};
  View vh{nullptr, "h", tokens, C, es}, vy{nullptr, "y", tokens, C, eb};
  View vdx{nullptr, "dx", tokens, C, es}, vdy{nullptr, "dy", tokens, C, eb};
  if (desc->pre) {
    OCHK(check_rows(du, "du", tokens, C, eb, false));
    OCHK(check_rows(h, "h", tokens, C, es, false));
    a.du = du->ptr, a.dut = du->token_stride;
    a.h = h->ptr, a.ht = h->token_stride;
    vdu.x = du, vh.x = h;
  }
  if (dh) {
    OCHK(check_rows(dh, "dh", tokens, C, es, false));
    a.dh = dh->ptr, a.dht = dh->token_stride;
    vdh.x = dh;
  }
  if (desc->branch) {
    OCHK(check_rows(y, "y", tokens, C, eb, false));
    OCHK(check_rows(dy, "dy", tokens, C, eb, true));
    a.y = y->ptr, a.yt = y->token_stride;
    a.dy = dy->ptr, a.dyt = dy->token_stride;
    vy.x = y, vdy.x = dy;
  }
  if (dx) {
    OCHK(check_rows(dx, "dx", tokens, C, es, true));
    a.dx = dx->ptr, a.dxt = dx->token_stride;
    vdx.x = dx;
    OCHK(check_apart(vdx, vdh, true));
    OCHK(check_apart(vdx, vdu, false));
    OCHK(check_apart(vdx, vh, false));
    OCHK(check_apart(vdx, vy, false));
    OCHK(check_apart(vdx, vdy, false));
  }
  OCHK(check_apart(vdy, vdu, true));
  OCHK(check_apart(vdy, vy, true));
  OCHK(check_apart(vdy, vdh, false));
  OCHK(check_apart(vdy, vh, false));
  OCHK(check_ws(workspace, workspace_bytes, norm_bwd_bytes(*desc, tokens)));
  const ParamViews in(desc, params), out(desc, grads);
  OCHK(check_apart(vdx, in));
  OCHK(check_apart(vdy, in));
  for (int i = 0; i < 7; ++i) {
    OCHK(check_apart(out.v[i], in));
    for (const View* v : {&vdu, &vdh, &vh, &vy, &vdx, &vdy})
      OCHK(check_apart(out.v[i], *v, false));
    for (int j = 0; j < i; ++j) OCHK(check_apart(out.v[i], out.v[j], false));
  }
  return launched(launch_norm_bwd(a, *grads, static_cast<float*>(workspace),
                                  static_cast<hipStream_t>(stream)),
                  "norm backward");
}

pulse_status pulse_keep_sizes(const pulse_keep_desc* desc, int32_t tokens, size_t* bytes) {
  OCHK(check_keep(desc));
  OCHK(check_tokens(tokens));
  if (!bytes) return ofail(PULSE_E_INVALID_ARG, "bytes is NULL");
  *bytes = keep_bytes(desc->channels, tokens);
  return PULSE_OK;
}

pulse_status pulse_keep_save(const pulse_keep_desc* desc, int32_t tokens, const pulse_rows* x,
                             const pulse_rows* a, void* kept, size_t kept_bytes, void* stream) {
  OCHK(check_keep(desc));
  OCHK(check_tokens(tokens));
  const int C = desc->channels, esz = size_of(desc->dtype);
  OCHK(check_rows(x, "x", tokens, C, esz, false));
  OCHK(check_kept(desc, tokens, kept, kept_bytes, "kept"));
  const View vx{x, "x", tokens, C, esz};
  const Flat fk(kept, tokens ? keep_bytes(C, tokens) : 0, "kept");
  OCHK(check_apart(fk.v, vx, false));
  KeepArgs k = keep_args(desc, tokens, kept);
  k.x = x->ptr, k.xt = x->token_stride;
  if (a) {
    if (!desc->act) return ofail(PULSE_E_INVALID_ARG, "a is given, and there is no act");
    OCHK(check_rows(a, "a", tokens, C, esz, true));
    const View va{a, "a", tokens, C, esz};
    OCHK(check_apart(va, vx, true));
    OCHK(check_apart(va, fk.v, false));
    k.y = a->ptr, k.yt = a->token_stride;
  }
  return launched(launch_keep_save(k, static_cast<hipStream_t>(stream)), "keep save");
}

pulse_status pulse_keep_load(const pulse_keep_desc* desc, int32_t tokens, const void* kept,
                             size_t kept_bytes, const pulse_rows* x, void* stream) {
  OCHK(check_keep(desc));
  OCHK(check_tokens(tokens));
  const int C = desc->channels, esz = size_of(desc->dtype);
  OCHK(check_kept(desc, tokens, kept, kept_bytes, "kept"));
  OCHK(check_rows(x, "x", tokens, C, esz, true));
  const Flat fk(kept, tokens ? keep_bytes(C, tokens) : 0, "kept");
  OCHK(check_apart(View{x, "x", tokens, C, esz}, fk.v, false));
  KeepArgs k = keep_args(desc, tokens, kept);
  k.y = x->ptr, k.yt = x->token_stride;
  return launched(launch_keep_load(k, static_cast<hipStream_t>(stream)), "keep load");
}

pulse_status pulse_keep_backward(const pulse_keep_desc* desc, int32_t tokens, const pulse_rows* da,
                                 const void* kept, size_t kept_bytes, const pulse_rows* dx,
                                 void* a_kept, size_t a_kept_bytes, void* stream) {
  OCHK(check_keep(desc));
  OCHK(check_tokens(tokens));
  if (!desc->act) return ofail(PULSE_E_INVALID_ARG, "there is no act to go back through");
  const int C = desc->channels, esz = size_of(desc->dtype);
  const size_t bytes = tokens ? keep_bytes(C, tokens) : 0;
  OCHK(check_rows(da, "da", tokens, C, esz, false));
  OCHK(check_kept(desc, tokens, kept, kept_bytes, "kept"));
  OCHK(check_rows(dx, "dx", tokens, C, esz, true));
  const View vda{da, "da", tokens, C, esz}, vdx{dx, "dx", tokens, C, esz};
  const Flat fk(kept, bytes, "kept"), fa(a_kept, a_kept ? bytes : 0, "a_kept");
  if (a_kept) OCHK(check_kept(desc, tokens, a_kept, a_kept_bytes, "a_kept"));
  OCHK(check_apart(vdx, vda, true));
  OCHK(check_apart(vdx, fk.v, false));
  OCHK(check_apart(vdx, fa.v, false));
  OCHK(check_apart(fa.v, vda, false));
  OCHK(check_apart(fa.v, fk.v, false));
  KeepArgs k = keep_args(desc, tokens, kept);
  k.x = da->ptr, k.xt = da->token_stride;
  k.y = dx->ptr, k.yt = dx->token_stride;
  k.a_kept = a_kept;
  return launched(launch_keep_back(k, static_cast<hipStream_t>(stream)), "keep backward");
}

static pulse_status check_outputs(int outputs) {
  if (outputs < 8 || outputs > 65536 || outputs % 8)
    return ofail(PULSE_E_SHAPE, "outputs must be a multiple of 8 in [8, 65536]");
  return PULSE_OK;
}

pulse_status pulse_keep_wgrad_sizes(const pulse_keep_desc* desc, int32_t tokens, int32_t outputs,
                                    size_t* workspace_bytes) {
  OCHK(check_keep(desc));
  OCHK(check_tokens(tokens));
  OCHK(check_outputs(outputs));
  if (!workspace_bytes) return ofail(PULSE_E_INVALID_ARG, "workspace_bytes is NULL");
  *workspace_bytes = kgrad_bytes(tokens, desc->channels, outputs);
  return PULSE_OK;
}

pulse_status pulse_keep_wgrad(const pulse_keep_desc* desc, int32_t tokens, int32_t outputs,
                              const pulse_rows* dy, const void* kept, size_t kept_bytes, float* dw,
                              float* db, int32_t accumulate, void* workspace,
                              size_t workspace_bytes, void* stream) {
  OCHK(check_keep(desc));
  OCHK(check_tokens(tokens));
  OCHK(check_outputs(outputs));
  OCHK(check_rows(dy, "dy", tokens, outputs, 2, false));
  OCHK(check_kept(desc, tokens, kept, kept_bytes, "kept"));
  if (!dw) return ofail(PULSE_E_INVALID_ARG, "dw is NULL");
  if (!aligned(dw, 16) || !aligned(db, 16))
    return ofail(PULSE_E_INVALID_ARG, "dw or db is not 16-byte aligned");
  if (accumulate != 0 && accumulate != 1)
    return ofail(PULSE_E_INVALID_ARG, "accumulate must be 0 or 1");
  const View vdy{dy, "dy", tokens, outputs, 2};
  const Flat fk(kept, tokens ? keep_bytes(desc->channels, tokens) : 0, "kept");
  const Flat fw(dw, (size_t)outputs * desc->channels * 4, "dw"), fb(db, (size_t)outputs * 4, "db");
  for (const Flat* out : {&fw, &fb}) {
    OCHK(check_apart(out->v, vdy, false));
    OCHK(check_apart(out->v, fk.v, false));
  }
  OCHK(check_apart(fb.v, fw.v, false));
  OCHK(check_ws(workspace, workspace_bytes, kgrad_bytes(tokens, desc->channels, outputs)));
  KgradArgs k{};
  k.tokens = tokens, k.C = desc->channels, k.N = outputs;
  k.dy = dy->ptr, k.dyt = dy->token_stride;
  k.kept = kept;
  k.dw = dw, k.db = db, k.accumulate = accumulate;
  k.ws = static_cast<float*>(workspace);
  return launched(launch_kgrad(k, static_cast<hipStream_t>(stream)), "kept weight gradient");
}

pulse_status pulse_lin8_sizes(const pulse_lin8_desc* desc, int32_t tokens, size_t* weight_bytes,
                              size_t* workspace_bytes) {
  OCHK(check_lin8(desc));
  OCHK(check_lin8_tokens(desc, tokens));
  if (weight_bytes) *weight_bytes = lin8_weight_bytes(desc->inputs, desc->outputs);
  if (workspace_bytes) *workspace_bytes = lin8_ws_bytes(tokens, desc->inputs, desc->outputs);
  return PULSE_OK;
}

pulse_status pulse_lin8_pack(const pulse_lin8_desc* desc, const void* w, int32_t w_dtype,
                             void* weights, size_t weight_bytes, void* stream) {
  OCHK(check_lin8(desc));
  if (!a_dtype(w_dtype))
    return ofail(PULSE_E_INVALID_ARG, "w_dtype must be PULSE_F32 or PULSE_BF16");
  if (!w || !aligned(w, 16)) return ofail(PULSE_E_INVALID_ARG, "w is NULL or not 16-byte aligned");
  OCHK(check_weights(desc, weights, weight_bytes));
  return launched(launch_lin8_pack(desc->inputs, desc->outputs, w, w_dtype, weights,
                                   static_cast<hipStream_t>(stream)),
                  "linear layer's layout");
}

pulse_status pulse_lin8_forward(const pulse_lin8_desc* desc, int32_t tokens, const pulse_rows* x,
                                const void* weights, size_t weight_bytes, const float* bias,
                                const pulse_rows* y, void* workspace, size_t workspace_bytes,
                                void* stream) {
  OCHK(check_lin8(desc));
  OCHK(check_lin8_tokens(desc, tokens));
  OCHK(check_rows(x, "x", tokens, desc->inputs, 2, false));
  OCHK(check_rows(y, "y", tokens, desc->outputs, 2, true));
  OCHK(check_apart(View{y, "y", tokens, desc->outputs, 2}, View{x, "x", tokens, desc->inputs, 2},
                   false));
  OCHK(check_weights(desc, weights, weight_bytes));
  if (!aligned(bias, 16)) return ofail(PULSE_E_INVALID_ARG, "bias is not 16-byte aligned");
  OCHK(check_ws(workspace, workspace_bytes, lin8_ws_bytes(tokens, desc->inputs, desc->outputs)));
  Lin8Args a{};
  a.tokens = tokens, a.K = desc->inputs, a.N = desc->outputs, a.act = desc->act;
  a.x = x->ptr, a.xt = x->token_stride;
  a.weights = weights, a.bias = bias;
  a.y = y->ptr, a.yt = y->token_stride;
  a.ws = workspace;
  return launched(launch_lin8(a, static_cast<hipStream_t>(stream)), "8-bit linear layer");
}

}  // extern "C"
