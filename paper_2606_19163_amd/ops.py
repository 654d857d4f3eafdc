"""ctypes binding of the packed-sequence operators (``include/pulse_ops.h``).

Images and clips of several resolutions lie one after another in one sequence,
a document each.  :class:`Mask` says which keys every query row attends,
:class:`Rope` turns query and key heads by their positions, :class:`Attn` is
attention under such a mask, forward and backward, and :class:`GradClip` the
global gradient norm with clipping.

Argument marshalling only: every step runs in the library's HIP kernels, and
loading fails loudly when the library has not been built.  Tensors are
``[tokens, heads, head_dim]`` with the last axis contiguous; the other two may
be strided (the heads inside a projection's output, or head-major storage).
Gradients come from the ``backward`` methods; autograd sees none of this, so a
call refuses inputs that require a gradient where torch records one.  Work is
enqueued on ``stream`` (default: torch's current one), and what a call allocates
belongs to that stream.  An object may be used from several: the caller orders
them, and the memory that an object holds is kept until all are done with it.
"""

from __future__ import annotations

import bisect
import ctypes
import math

import torch

from .stage import BF16, F32, E_INVALID_ARG, PulseError, _check, lib as _lib

__all__ = ["Rope", "Mask", "Attn", "Saved", "GradClip", "rope_freqs", "grid_positions", "MaskRow"]

_i32 = ctypes.c_int32
_i64 = ctypes.c_int64
_vp = ctypes.c_void_p
_szp = ctypes.POINTER(ctypes.c_size_t)
_PAIRS = {"adjacent": 0, "halves": 1}


class Heads(ctypes.Structure):
    _fields_ = [("ptr", _vp), ("token_stride", _i64), ("head_stride", _i64)]


class RopeDesc(ctypes.Structure):
    _fields_ = [("heads", _i32), ("head_dim", _i32), ("axes", _i32), ("axis_dim", _i32 * 4),
                ("pairs", _i32), ("dtype", ctypes.c_int)]


class MaskRow(ctypes.Structure):
    _fields_ = [("lo", _i32), ("hi", _i32), ("pos", _i32), ("doc", _i32)]


class MaskDesc(ctypes.Structure):
    _fields_ = [("queries", _i32), ("keys", _i32), ("docs", _i32), ("causal", _i32)]


class AttnDesc(ctypes.Structure):
    _fields_ = [("queries", _i32), ("keys", _i32), ("heads", _i32), ("kv_heads", _i32),
                ("head_dim", _i32), ("scale", ctypes.c_float), ("cap", ctypes.c_float),
                ("dtype", ctypes.c_int)]


class ClipTensor(ctypes.Structure):
    _fields_ = [("grad", _vp), ("out", _vp), ("n", _i64), ("dtype", ctypes.c_int)]


# torch.cuda.current_stream() builds an object that only its handle is read from
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream",
                      lambda dev: torch.cuda.current_stream(dev).cuda_stream)

_bound = None


def lib():
    global _bound
    if _bound is None:
        L = _lib()
        st, hp, f = ctypes.c_int, ctypes.POINTER(Heads), ctypes.c_float
        L.pulse_rope.argtypes = [ctypes.POINTER(RopeDesc), _i32, _i32, hp, _vp, _vp, hp, _vp]
        L.pulse_rope.restype = st
        md = ctypes.POINTER(MaskDesc)
        L.pulse_mask_sizes.argtypes = [md, _szp]
        L.pulse_mask_sizes.restype = st
        L.pulse_mask_build.argtypes = [md, _vp, _vp, _vp, _vp, ctypes.c_size_t, _vp]
        L.pulse_mask_build.restype = st
        L.pulse_mask_from_rows.argtypes = [md, _vp, _vp, ctypes.c_size_t, _vp]
        L.pulse_mask_from_rows.restype = st
        ad = ctypes.POINTER(AttnDesc)
        L.pulse_attn_sizes.argtypes = [ad, _szp, _szp]
        L.pulse_attn_sizes.restype = st
        L.pulse_attn_forward.argtypes = [ad, hp, hp, hp, _vp, _vp, hp, _vp, _vp, _vp,
                                         ctypes.c_size_t, _vp]
        L.pulse_attn_forward.restype = st
        L.pulse_attn_backward.argtypes = [ad, hp, hp, hp, hp, hp, _vp, _vp, _vp, _vp, hp, hp, hp,
                                          _vp, ctypes.c_size_t, _vp]
        L.pulse_attn_backward.restype = st
        L.pulse_clip_create.argtypes = [ctypes.POINTER(ClipTensor), _i32, ctypes.POINTER(_vp)]
        L.pulse_clip_create.restype = st
        L.pulse_clip_destroy.argtypes = [_vp]
        L.pulse_clip_destroy.restype = None
        L.pulse_clip_sizes.argtypes = [_vp, _szp]
        L.pulse_clip_sizes.restype = st
        L.pulse_clip_bind.argtypes = [_vp, _vp, ctypes.c_size_t, _vp]
        L.pulse_clip_bind.restype = st
        L.pulse_clip_run.argtypes = [_vp, f, f, _vp, _vp]
        L.pulse_clip_run.restype = st
        _bound = L
    return _bound


def _bad(msg):
    raise PulseError(E_INVALID_ARG, msg)


def _dtype(dt):
    if dt == torch.bfloat16:
        return BF16
    if dt == torch.float32:
        return F32
    _bad(f"dtype must be torch.bfloat16 or torch.float32, not {dt}")


def _heads(t, name, shape, dtype, dev):
    """The view [tokens, heads, dim] `t` of GPU `dev`, where the call runs."""
    if t.dtype is not dtype or t.shape != shape:
        _bad(f"{name} is {t.dtype} {tuple(t.shape)}, expected {dtype} {tuple(shape)}")
    s0, s1, s2 = t.stride()
    if s2 != 1 and shape[2] != 1:
        _bad(f"{name}: the channels of a head must be contiguous")
    if t.get_device() != dev:
        _bad(f"{name} is on {t.device}, not on the current GPU")
    # the stride of an axis of one element is never used
    return Heads(t.data_ptr(), s0 if shape[0] > 1 else 0, s1 if shape[1] > 1 else 0)


def _flat(t, name, n, dtype, dev):
    """Pointer of a contiguous tensor of n elements (None stays NULL)."""
    if t is None:
        return None
    if t.dtype is not dtype or t.numel() != n or not t.is_contiguous():
        _bad(f"{name} must be contiguous {dtype} with {n} elements, not {t.dtype} "
             f"{tuple(t.shape)}")
    if t.get_device() != dev:
        _bad(f"{name} is on {t.device}, not on the current GPU")
    return t.data_ptr()


def _by_hand(*inputs):
    """Refuse inputs, (name, tensor) each, whose gradients the caller expects
    from autograd."""
    for name, t in inputs:
        if t is not None and t.requires_grad:
            _bad(f"{name} requires a gradient, which autograd would not get: call this under "
                 "torch.no_grad() and use backward")


_grad_on = torch.is_grad_enabled


def _here():
    """The current GPU and the handle of its current stream.  A call given a
    `stream` makes it current and calls itself, so that what it allocates
    belongs to the stream it runs on."""
    dev = torch.cuda.current_device()
    return dev, _raw_stream(dev)


def _home(t):
    """The stream that the allocator thinks `t` is used on."""
    return _raw_stream(t.get_device()) if t.is_cuda else None


def _used_on(t, dev):
    """`t` is used on another stream than its own, the current one: its memory
    is not handed on before that is done."""
    t.record_stream(torch.cuda.current_stream(dev))


def rope_freqs(axis_dim, base=10000.0, device="cuda"):
    """freq[p] = base^(-2 i / n) for pair i of an axis of n channels, the axes
    one after another (fp32)."""
    parts = [base ** (-torch.arange(0, n, 2, dtype=torch.float64) / max(n, 1)) for n in axis_dim]
    return torch.cat(parts).float().to(device)


def grid_positions(shapes, device="cuda"):
    """Positions [tokens, axes] of documents whose tokens are grids (time,
    height, width or any other number of axes) in row-major order."""
    out = [torch.cartesian_prod(*[torch.arange(n) for n in s]).reshape(-1, len(s)) for s in shapes]
    return torch.cat(out).float().to(device)


class Rope:
    """Rotary positions of ``heads`` heads; ``axis_dim``: channels per axis."""

    def __init__(self, heads, head_dim, axis_dim, pairs="adjacent", dtype=None):
        self.dtype = torch.bfloat16 if dtype is None else dtype
        if pairs not in _PAIRS:
            _bad(f"pairs must be one of {sorted(_PAIRS)}")
        if not 1 <= len(axis_dim) <= 4:
            _bad("one to four axes")
        self.heads, self.dim, self.axes = heads, head_dim, len(axis_dim)
        self.half = sum(axis_dim) // 2
        self.desc = RopeDesc(heads, head_dim, len(axis_dim), (_i32 * 4)(*axis_dim), _PAIRS[pairs],
                             _dtype(self.dtype))
        # no tokens: only the descriptor is checked
        none = Heads(None, 0, 0)
        _check(lib().pulse_rope(ctypes.byref(self.desc), 0, 0, ctypes.byref(none), None, None,
                                ctypes.byref(none), None))

    def _run(self, x, pos, freq, out, backward, stream):
        n = x.shape[0]
        shape = (n, self.heads, self.dim)
        if stream is not None:
            with torch.cuda.stream(stream):
                return self._run(x, pos, freq, out, backward, None)
        dev, s = _here()
        if out is None:
            out = torch.empty(shape, dtype=self.dtype, device=x.device)
        hx = _heads(x, "x", shape, self.dtype, dev)
        hy = _heads(out, "out", shape, self.dtype, dev)
        _check(lib().pulse_rope(
            self.desc, n, backward, hx, _flat(pos, "pos", n * self.axes, torch.float32, dev),
            _flat(freq, "freq", self.half, torch.float32, dev), hy, s))
        return out

    def forward(self, x, pos, freq, out=None, stream=None):
        """x turned by its positions; ``out`` may be x."""
        if _grad_on() and (x.requires_grad or pos.requires_grad or freq.requires_grad):
            _by_hand(("x", x), ("pos", pos), ("freq", freq))
        return self._run(x, pos, freq, out, 0, stream)

    def backward(self, dout, pos, freq, out=None, stream=None):
        """The gradient of ``forward``'s input from that of its output."""
        if dout.requires_grad and _grad_on():
            _by_hand(("dout", dout))
        return self._run(dout, pos, freq, out, 1, stream)


class Mask:
    """Which of ``keys`` keys each of ``queries`` rows attends.  Beside the
    rows lies a table over them that attention reads, so :class:`Attn` takes
    a mask only once ``build`` or ``from_rows`` has filled both: after writing
    into ``rows``, call ``from_rows(mask.rows)``.  Both overwrite the mask in
    place: with several batches between forward and backward, each needs a
    mask of its own."""

    def __init__(self, queries, keys=None, docs=0, causal=False, device="cuda"):
        self.queries, self.keys = queries, queries if keys is None else keys
        self.docs = docs
        self.desc = MaskDesc(queries, self.keys, docs, 1 if causal else 0)
        n = ctypes.c_size_t()
        _check(lib().pulse_mask_sizes(ctypes.byref(self.desc), ctypes.byref(n)))
        self.bytes = n.value
        self.buffer = torch.empty(max(n.value // 4, 4), dtype=torch.int32, device=device)
        self.ptr, self.home = self.buffer.data_ptr(), _home(self.buffer)
        #: [queries, 4]: lo, hi, pos, doc of every row
        self.rows = self.buffer[:4 * queries].view(queries, 4)
        self.inference = self.buffer.is_inference()
        self.stamp, self.serial = None, 0

    def _stamp(self):
        """Changes with every torch operation that writes the rows."""
        return 0 if self.inference else self.buffer._version

    def _built(self):
        self.stamp = self._stamp()
        self.serial += 1

    def check(self):
        """Refuse a mask that was not built, or written since."""
        if self.stamp != self._stamp() and self.queries:
            if self.stamp is None:
                _bad("the mask was not built: call build or from_rows first")
            _bad("the mask's rows were written since it was built: call from_rows")

    def build(self, offsets, key_offsets=None, prefix=None, stream=None):
        """From int32 ``offsets`` [docs + 1] on the GPU; returns ``rows``."""
        if stream is not None:
            with torch.cuda.stream(stream):
                return self.build(offsets, key_offsets, prefix)
        dev, s = _here()
        if self.buffer.get_device() != dev:
            _bad(f"the mask is on {self.buffer.device}, not on the current GPU")
        if s != self.home:
            _used_on(self.buffer, dev)
        _check(lib().pulse_mask_build(
            self.desc, _flat(offsets, "offsets", self.docs + 1, torch.int32, dev),
            _flat(key_offsets, "key_offsets", self.docs + 1, torch.int32, dev),
            _flat(prefix, "prefix", self.docs, torch.int32, dev), self.ptr, self.bytes, s))
        self._built()
        return self.rows

    def from_rows(self, rows, stream=None):
        """From the caller's int32 [queries, 4] (it may be ``self.rows``)."""
        if stream is not None:
            with torch.cuda.stream(stream):
                return self.from_rows(rows)
        dev, s = _here()
        if self.buffer.get_device() != dev:
            _bad(f"the mask is on {self.buffer.device}, not on the current GPU")
        if s != self.home:
            _used_on(self.buffer, dev)
        _check(lib().pulse_mask_from_rows(
            self.desc, _flat(rows, "rows", 4 * self.queries, torch.int32, dev), self.ptr,
            self.bytes, s))
        self._built()
        return self.rows


class Saved:
    """What a forward leaves for its backward beside the output: the scores'
    log sum exp (``lse``, fp32 [heads, queries]), what the rounding of the
    output left out, and which mask it ran under."""

    __slots__ = ("buffer", "shape", "lse_ptr", "low_ptr", "home", "mask", "serial")

    def __init__(self, heads, queries, head_dim, device, home=None):
        n = -(-heads * queries // 4) * 4  # the second part is 16-byte aligned
        self.buffer = torch.empty(n + heads * queries * head_dim // 2, dtype=torch.float32,
                                  device=device)
        self.shape = (heads, queries, head_dim)
        self.lse_ptr = self.buffer.data_ptr()
        self.low_ptr = self.lse_ptr + 4 * n
        self.home = _home(self.buffer) if home is None else home
        self.mask, self.serial = None, 0

    @property
    def lse(self):
        h, t, _ = self.shape
        return self.buffer[:h * t].view(h, t)


class Attn:
    """Attention of ``queries`` rows and ``heads`` heads under a mask (bf16)."""

    def __init__(self, queries, heads, head_dim, keys=None, kv_heads=None, scale=None, cap=0.0):
        self.queries, self.keys = queries, queries if keys is None else keys
        self.heads, self.kv, self.dim = heads, heads if kv_heads is None else kv_heads, head_dim
        scale = 1.0 / math.sqrt(head_dim) if scale is None else scale
        self.desc = AttnDesc(queries, self.keys, heads, self.kv, head_dim, scale, cap, BF16)
        f, b = ctypes.c_size_t(), ctypes.c_size_t()
        _check(lib().pulse_attn_sizes(ctypes.byref(self.desc), ctypes.byref(f), ctypes.byref(b)))
        self.fwd_bytes, self.bwd_bytes = f.value, b.value
        self.qs = (queries, heads, head_dim)
        self.ks = (self.keys, self.kv, head_dim)

    def _mask(self, mask, dev, s):
        if mask.queries != self.queries or mask.keys != self.keys:
            _bad(f"the mask is of {mask.queries} rows and {mask.keys} keys")
        if mask.inference or mask.stamp != mask.buffer._version:
            mask.check()
        if mask.buffer.get_device() != dev:
            _bad(f"the mask is on {mask.buffer.device}, not on the current GPU")
        if s != mask.home:
            _used_on(mask.buffer, dev)
        return mask.ptr

    def forward(self, q, k, v, mask, slopes=None, out=None, saved=None, stream=None, keep=True):
        """(o, saved): o [queries, heads, head_dim] and what the backward needs
        beside it (into ``saved`` of an earlier call, if given).  Without
        ``keep`` nothing is kept for a backward and saved is None."""
        bf = torch.bfloat16
        if _grad_on() and (q.requires_grad or k.requires_grad or v.requires_grad or
                           slopes is not None and slopes.requires_grad):
            _by_hand(("q", q), ("k", k), ("v", v), ("slopes", slopes))
        if saved is not None and not keep:
            _bad("saved is given, and nothing is to be kept")
        if stream is not None:
            with torch.cuda.stream(stream):
                return self.forward(q, k, v, mask, slopes, out, saved, None, keep)
        dev, s = _here()
        if out is None:
            out = torch.empty(self.qs, dtype=bf, device=q.device)
        lse = None
        if not keep:
            lse = torch.empty((self.heads, self.queries), dtype=torch.float32, device=q.device)
        elif saved is None:
            saved = Saved(self.heads, self.queries, self.dim, q.device, s)
        ws = None
        if self.fwd_bytes:
            ws = torch.empty(self.fwd_bytes, dtype=torch.uint8, device=q.device)
        _check(lib().pulse_attn_forward(
            self.desc, _heads(q, "q", self.qs, bf, dev), _heads(k, "k", self.ks, bf, dev),
            _heads(v, "v", self.ks, bf, dev), self._mask(mask, dev, s),
            _flat(slopes, "slopes", self.heads, torch.float32, dev),
            _heads(out, "out", self.qs, bf, dev),
            *(self._saved(saved, dev, s) if keep else (lse.data_ptr(), None)),
            ws.data_ptr() if ws is not None else None, self.fwd_bytes, s))
        if keep:
            saved.mask, saved.serial = mask, mask.serial
        return out, saved

    def _saved(self, saved, dev, s):
        if saved.shape != (self.heads, self.queries, self.dim):
            _bad(f"saved is of heads, queries and head_dim {saved.shape}")
        if saved.buffer.get_device() != dev:
            _bad(f"saved is on {saved.buffer.device}, not on the current GPU")
        if s != saved.home:
            _used_on(saved.buffer, dev)
        return saved.lse_ptr, saved.low_ptr

    def backward(self, dout, q, k, v, o, saved, mask, slopes=None, out=None, stream=None):
        """(dq, dk, dv), written into the tensors of ``out`` if given."""
        bf = torch.bfloat16
        if dout.requires_grad and _grad_on():
            _by_hand(("dout", dout))
        if saved.mask is None:
            _bad("saved is of no forward")
        if saved.mask is mask and saved.serial != mask.serial:
            _bad("the mask was built again since this forward: batches in flight need one each")
        if stream is not None:
            with torch.cuda.stream(stream):
                return self.backward(dout, q, k, v, o, saved, mask, slopes, out)
        dev, s = _here()
        if out is None:
            out = [torch.empty(n, dtype=bf, device=q.device)
                   for n in (self.qs, self.ks, self.ks)]
        dq, dk, dv = out
        ws = None
        if self.bwd_bytes:
            ws = torch.empty(self.bwd_bytes, dtype=torch.uint8, device=q.device)
        _check(lib().pulse_attn_backward(
            self.desc, _heads(dout, "dout", self.qs, bf, dev), _heads(q, "q", self.qs, bf, dev),
            _heads(k, "k", self.ks, bf, dev), _heads(v, "v", self.ks, bf, dev),
            _heads(o, "o", self.qs, bf, dev), *self._saved(saved, dev, s),
            self._mask(mask, dev, s),
            _flat(slopes, "slopes", self.heads, torch.float32, dev),
            _heads(dq, "dq", self.qs, bf, dev), _heads(dk, "dk", self.ks, bf, dev),
            _heads(dv, "dv", self.ks, bf, dev),
            ws.data_ptr() if ws is not None else None, self.bwd_bytes, s))
        return dq, dk, dv


def _clashes(grads, outs):
    """(i, j) of an output i that overlaps output j or gradient j, but for a
    gradient that is its own output; else None.  Spans are (begin, end)."""
    order = sorted((b, e, i) for i, (b, e) in enumerate(outs) if e > b)
    for x, y in zip(order, order[1:]):
        if y[0] < x[1]:
            return x[2], y[2]
    begins = [b for b, _, _ in order]  # disjoint from here on
    for j, (b, e) in enumerate(grads):
        at = max(bisect.bisect_right(begins, b) - 1, 0)
        while e > b and at < len(order) and order[at][0] < e:
            if order[at][1] > b and not (order[at][2] == j and order[at][:2] == (b, e)):
                return order[at][2], j
            at += 1
    return None


def _span(t):
    return t.data_ptr(), t.data_ptr() + t.numel() * t.element_size()


class GradClip:
    """The global norm of ``grads`` (contiguous, fp32 or bf16) and their
    clipping, in place or into ``outs``.  The tensors' addresses are taken
    once, so they must stay where they are from step to step.  No output may
    overlap another, or another tensor's gradient."""

    def __init__(self, grads, outs=None):
        self.h = _vp()
        grads = list(grads)
        outs = grads if outs is None else list(outs)
        if len(grads) != len(outs):
            _bad(f"{len(grads)} gradients and {len(outs)} outputs")
        if not all(t.is_cuda for t in grads + outs):
            _bad("a gradient or an output is not on a GPU")
        dev = torch.cuda.current_device() if grads else -1
        arr = (ClipTensor * max(len(grads), 1))()
        for i, (g, o) in enumerate(zip(grads, outs)):
            if g.dtype != o.dtype or g.numel() != o.numel():
                _bad(f"gradient {i} and its output differ in type or size")
            if not g.is_contiguous() or not o.is_contiguous():
                _bad(f"gradient {i} or its output is not contiguous")
            if g.get_device() != dev or o.get_device() != dev:
                _bad(f"gradient {i} or its output is not on the current GPU")
            arr[i] = ClipTensor(g.data_ptr(), o.data_ptr(), g.numel(), _dtype(g.dtype))
        clash = _clashes([_span(g) for g in grads], [_span(o) for o in outs])
        if clash:
            _bad(f"output {clash[0]} overlaps output or gradient {clash[1]}")
        self.grads, self.outs = grads, outs
        self.device = grads[0].device if grads else "cuda"
        _check(lib().pulse_clip_create(arr, len(grads), ctypes.byref(self.h)))
        n = ctypes.c_size_t()
        _check(lib().pulse_clip_sizes(self.h, ctypes.byref(n)))
        self.workspace = torch.empty(n.value, dtype=torch.uint8, device=self.device)
        self.home = _home(self.workspace)
        s = torch.cuda.current_stream()
        _check(lib().pulse_clip_bind(self.h, self.workspace.data_ptr(), n.value, s.cuda_stream))
        s.synchronize()  # the table is there whichever stream the first run is on

    def __del__(self):
        try:
            if self.h:
                lib().pulse_clip_destroy(self.h)
                self.h = _vp()
        except Exception:
            pass

    def run(self, max_norm, eps=1e-6, norm=None, stream=None):
        """Clip to ``max_norm``; returns the norm before it, fp32 [1].  Calls
        share one workspace: order the streams that they run on."""
        if stream is not None:
            with torch.cuda.stream(stream):
                return self.run(max_norm, eps, norm)
        dev, s = _here()
        if s != self.home:
            _used_on(self.workspace, dev)
        if norm is None:
            norm = torch.empty(1, dtype=torch.float32, device=self.device)
        _check(lib().pulse_clip_run(self.h, max_norm, eps,
                                    _flat(norm, "norm", 1, torch.float32, dev), s))
        return norm
