"""ctypes binding of the packed-sequence operators (``include/pulse_ops.h``).

Images and clips of several resolutions lie one after another in one sequence,
a document each.  :class:`Mask` says which keys every query row attends,
:class:`Rope` turns query and key heads by their positions, :class:`Attn` is
attention under such a mask, forward and backward, and :class:`GradClip` the
global gradient norm with clipping.  Around the attention, :class:`Norm` is the
joint between two halves of a block (gate, residual, norms, the documents'
scales and shifts), :class:`Checkpoint` keeps activations in 8 bits until the
backward pass and computes gradients from them, and :class:`Linear8` is a linear
layer in 8-bit integers for sampling.

Argument marshalling only: every step runs in the library's HIP kernels, and
loading fails loudly when the library has not been built.  Tensors are
``[tokens, heads, head_dim]`` with the last axis contiguous; the other two may
be strided (the heads inside a projection's output, or head-major storage), or
``[tokens, channels]`` with strided rows.
Gradients come from the ``backward`` methods; autograd sees none of this, so a
call refuses inputs that require a gradient where torch records one.  Work is
enqueued on ``stream`` (default: torch's current one), and what a call allocates
belongs to that stream.  An object may be used from several: the caller orders
them, and the memory that an object holds is kept until all are done with it.
Copies (copy, deepcopy, pickle) have memory of their own; a :class:`GradClip`,
which knows its gradients by address, refuses to be copied.
"""

from __future__ import annotations

import bisect
import copy
import ctypes
import math
import struct

import torch

from .stage import BF16, F32, E_INVALID_ARG, PulseError, _check, lib as _lib

__all__ = ["Rope", "Mask", "Attn", "Saved", "GradClip", "Norm", "Checkpoint", "Kept", "Linear8",
           "rope_freqs", "grid_positions", "MaskRow"]

_i32 = ctypes.c_int32
_i64 = ctypes.c_int64
_vp = ctypes.c_void_p
_szp = ctypes.POINTER(ctypes.c_size_t)
_PAIRS = {"adjacent": 0, "halves": 1}
_NORMS = {None: 0, "layer": 1, "rms": 2}
_ACTS = {None: 0, "gelu": 1, "silu": 2}


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


class Rows(ctypes.Structure):
    _fields_ = [("ptr", _vp), ("token_stride", _i64)]


class NormDesc(ctypes.Structure):
    _fields_ = [("channels", _i32), ("docs", _i32), ("pre", _i32), ("post", _i32),
                ("branch", _i32), ("eps", ctypes.c_float), ("residual_scale", ctypes.c_float),
                ("dtype", _i32), ("stream_dtype", _i32)]


class NormParams(ctypes.Structure):
    _fields_ = [("offsets", _vp), ("gate", _vp), ("scale", _vp), ("shift", _vp),
                ("gate_stride", _i64), ("scale_stride", _i64), ("shift_stride", _i64),
                ("weight", _vp), ("bias", _vp), ("post_weight", _vp)]


class NormGrads(ctypes.Structure):
    _fields_ = [("dgate", _vp), ("dscale", _vp), ("dshift", _vp), ("dweight", _vp),
                ("dbias", _vp), ("dpost_weight", _vp)]


class KeepDesc(ctypes.Structure):
    _fields_ = [("channels", _i32), ("act", _i32), ("dtype", _i32)]


class Lin8Desc(ctypes.Structure):
    _fields_ = [("inputs", _i32), ("outputs", _i32), ("act", _i32), ("dtype", _i32)]


# torch.cuda.current_stream() builds an object that only its handle is read from
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream",
                      lambda dev: torch.cuda.current_stream(dev).cuda_stream)

_bound = None


def lib():
    global _bound, _fast
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
        rp, sz, nd = ctypes.POINTER(Rows), ctypes.c_size_t, ctypes.POINTER(NormDesc)
        pp, gp = ctypes.POINTER(NormParams), ctypes.POINTER(NormGrads)
        kd, ld = ctypes.POINTER(KeepDesc), ctypes.POINTER(Lin8Desc)
        fast = {}
        for name, args in (
                ("norm_sizes", [nd, _i32, _szp]),
                ("norm_forward", [nd, _i32, rp, rp, pp, rp, rp, _vp]),
                ("norm_backward", [nd, _i32, rp, rp, rp, rp, pp, rp, rp, gp, _vp, sz, _vp]),
                ("keep_sizes", [kd, _i32, _szp]),
                ("keep_save", [kd, _i32, rp, rp, _vp, sz, _vp]),
                ("keep_load", [kd, _i32, _vp, sz, rp, _vp]),
                ("keep_backward", [kd, _i32, rp, _vp, sz, rp, _vp, sz, _vp]),
                ("keep_wgrad_sizes", [kd, _i32, _i32, _szp]),
                ("keep_wgrad", [kd, _i32, _i32, rp, _vp, sz, _vp, _vp, _i32, _vp, sz, _vp]),
                ("lin8_sizes", [ld, _i32, _szp, _szp]),
                ("lin8_pack", [ld, _vp, _i32, _vp, sz, _vp]),
                ("lin8_forward", [ld, _i32, rp, _vp, sz, _vp, rp, _vp, sz, _vp])):
            fn = getattr(L, "pulse_" + name)
            fn.argtypes, fn.restype = args, st
            # the same entry for structures that come as bytes: packing takes a third
            # of the time of building one
            fn = L["pulse_" + name]
            fn.argtypes = [a if a in (_i32, sz, _szp) else _vp for a in args]
            fn.restype = st
            fast[name] = fn
        # whole, and before any object can be made: another thread may be here too
        _fast = fast
        _bound = L
    return _bound


_fast = {}
_NORM_GRADS = [k for k, _ in NormGrads._fields_]
_pack_rows = struct.Struct("=qq").pack
_pack_params = struct.Struct("=qqqqqqqqqq").pack
_pack_grads = struct.Struct("=qqqqqq").pack


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


def _rows(t, name, shape, dtype, dev):
    """The view [tokens, channels] `t` of GPU `dev`, where the call runs, as the
    bytes of a Rows."""
    if t.dtype is not dtype or t.shape != shape:
        _bad(f"{name} is {t.dtype} {tuple(t.shape)}, expected {dtype} {tuple(shape)}")
    s0, s1 = t.stride()
    if s1 != 1:
        _bad(f"{name}: the channels of a row must be contiguous")
    if t.get_device() != dev:
        _bad(f"{name} is on {t.device}, not on the current GPU")
    return _pack_rows(t.data_ptr(), s0 if shape[0] > 1 else 0)


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


_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)


def _here():
    """The current GPU and the handle of its current stream.  A call given a
    `stream` makes it current and calls itself, so that what it allocates
    belongs to the stream it runs on."""
    dev = _device()
    return dev, _raw_stream(dev)


def _home(t):
    """The stream that the allocator thinks `t` is used on."""
    return _raw_stream(t.get_device()) if t.is_cuda else None


def _used_on(t, dev):
    """`t` is used on another stream than its own, the current one: its memory
    is not handed on before that is done."""
    t.record_stream(torch.cuda.current_stream(dev))


class _Owner:
    """An object that holds GPU memory (``_memory``, names of its tensors) and what
    its calls look up there once: addresses, and the stream the memory is from.
    Every copy, a shallow or an unpickled one too, has memory of its own and looks
    these up again (``_locate``)."""

    __slots__ = ()
    _memory, _found = (), ("ptr", "home")

    def __copy__(self):
        return copy.deepcopy(self)

    def __getstate__(self):
        for t in (getattr(self, k) for k in self._memory):
            # the copy reads it on the current stream
            if t.is_cuda and _raw_stream(t.get_device()) != self.home:
                _used_on(t, t.get_device())
        names = {*getattr(self, "__dict__", ()), *self.__slots__}
        return {k: getattr(self, k) for k in names if k not in self._found}

    def __setstate__(self, state):
        for k, v in state.items():
            setattr(self, k, v)
        self._locate()


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


class Mask(_Owner):
    """Which of ``keys`` keys each of ``queries`` rows attends.  Beside the
    rows lies a table over them that attention reads, so :class:`Attn` takes
    a mask only once ``build`` or ``from_rows`` has filled both: after writing
    into ``rows``, call ``from_rows(mask.rows)``.  Both overwrite the mask in
    place: with several batches between forward and backward, each needs a
    mask of its own."""

    _memory, _found = ("buffer",), ("ptr", "home", "rows", "inference")

    def __init__(self, queries, keys=None, docs=0, causal=False, device="cuda"):
        self.queries, self.keys = queries, queries if keys is None else keys
        self.docs = docs
        self.desc = MaskDesc(queries, self.keys, docs, 1 if causal else 0)
        n = ctypes.c_size_t()
        _check(lib().pulse_mask_sizes(ctypes.byref(self.desc), ctypes.byref(n)))
        self.bytes = n.value
        self.buffer = torch.empty(max(n.value // 4, 4), dtype=torch.int32, device=device)
        self.stamp, self.serial = None, 0
        self._locate()

    def _locate(self):
        self.ptr, self.home = self.buffer.data_ptr(), _home(self.buffer)
        #: [queries, 4]: lo, hi, pos, doc of every row
        self.rows = self.buffer[:4 * self.queries].view(self.queries, 4)
        self.inference = self.buffer.is_inference()

    def __getstate__(self):
        # the stamp is of this buffer's version: whether it holds is what a copy keeps
        stamp = self.stamp if self.stamp is None else self.stamp == self._stamp()
        return {**super().__getstate__(), "stamp": stamp}

    def __setstate__(self, state):
        super().__setstate__(state)
        if self.stamp is not None:
            self.stamp = self._stamp() if self.stamp else -1

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


class Saved(_Owner):
    """What a forward leaves for its backward beside the output: the scores'
    log sum exp (``lse``, fp32 [heads, queries]), what the rounding of the
    output left out, and which mask it ran under."""

    __slots__ = ("buffer", "shape", "lse_ptr", "low_ptr", "home", "mask", "serial")
    _memory, _found = ("buffer",), ("lse_ptr", "low_ptr", "home")

    def __init__(self, heads, queries, head_dim, device, home=None):
        n = -(-heads * queries // 4) * 4  # the second part is 16-byte aligned
        self.buffer = torch.empty(n + heads * queries * head_dim // 2, dtype=torch.float32,
                                  device=device)
        self.shape = (heads, queries, head_dim)
        self.mask, self.serial = None, 0
        self._locate(home)

    def _locate(self, home=None):
        heads, queries, _ = self.shape
        self.lse_ptr = self.buffer.data_ptr()
        self.low_ptr = self.lse_ptr + 4 * (-(-heads * queries // 4) * 4)
        self.home = _home(self.buffer) if home is None else home

    def __deepcopy__(self, memo):
        # it ran under that mask still, but where the mask is copied along
        new, state = Saved.__new__(Saved), self.__getstate__()
        memo[id(self)], mask = new, state.pop("mask")
        new.__setstate__({**copy.deepcopy(state, memo), "mask": memo.get(id(mask), mask)})
        return new

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

    def __reduce_ex__(self, protocol):
        # the handle is destroyed once, and its table names these very tensors
        _bad("a GradClip cannot be copied: make one of the copied gradients")

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


def _choice(v, among, name):
    if v not in among:
        _bad(f"{name} must be one of {sorted(map(str, among))}, not {v!r}")
    return among[v]


def _bytes_at(n, device):
    return torch.empty(n, dtype=torch.uint8, device=device)


class Norm:
    """The joint between two halves of a transformer block:

        h = x + residual_scale * gate[doc] * Post(y)
        u = Pre(h) * (1 + scale[doc]) + shift[doc]

    with the residual stream x and h (``stream_dtype``), the last half's output y
    and the next half's input u (``dtype``).  ``pre`` and ``post`` are "layer",
    "rms" or None: the norm before the next half (None: the joint only adds, and
    there is no u) and after the last one (None: y itself).  Without ``branch``
    there is no y, and h is x.  Documents are rows [offsets[d], offsets[d + 1]) of
    int32 ``offsets`` [docs + 1]; rows from the last offset on are padding, where h
    = x and u = 0 and which no sum sees.  Without offsets all rows are the one
    document's.  ``gate``, ``scale`` and ``shift`` are fp32 [docs, channels] (rows
    may be strided), ``weight``, ``bias`` and ``post_weight`` fp32 [channels];
    each may be left out."""

    def __init__(self, channels, docs=1, pre="layer", post=None, branch=True, eps=1e-6,
                 residual_scale=1.0, dtype=None, stream_dtype=None):
        self.dtype = torch.bfloat16 if dtype is None else dtype
        self.stream_dtype = self.dtype if stream_dtype is None else stream_dtype
        self.channels, self.docs, self.branch = channels, docs, bool(branch)
        self.pre, self.post = pre, post
        self.desc = NormDesc(channels, docs, _choice(pre, _NORMS, "pre"),
                             _choice(post, _NORMS, "post"), 1 if branch else 0, eps,
                             residual_scale, _dtype(self.dtype), _dtype(self.stream_dtype))
        n = ctypes.c_size_t()
        _check(lib().pulse_norm_sizes(self.desc, 0, n))
        # its bytes, and no address: a copy of the object has its own
        self.packed, self.sizes = bytes(self.desc), {0: n.value}
        self.cond_shape = (docs, channels)

    def _cond(self, t, name, dev):
        if t is None:
            return 0, 0
        s0, s1 = t.stride() if t.dim() == 2 else (0, 0)
        if t.dtype is not torch.float32 or t.shape != self.cond_shape or s1 != 1:
            _bad(f"{name} must be fp32 {list(self.cond_shape)} with contiguous rows, not "
                 f"{t.dtype} {tuple(t.shape)}")
        if t.get_device() != dev:
            _bad(f"{name} is on {t.device}, not on the current GPU")
        return t.data_ptr(), s0

    def _params(self, offsets, gate, scale, shift, weight, bias, post_weight, dev):
        """The bytes of a NormParams."""
        (g, gs), (s, ss), (f, fs) = (self._cond(gate, "gate", dev), self._cond(scale, "scale", dev),
                                     self._cond(shift, "shift", dev))
        c, f32 = self.channels, torch.float32
        return _pack_params(
            _flat(offsets, "offsets", self.docs + 1, torch.int32, dev) or 0, g, s, f, gs, ss, fs,
            0 if weight is None else _flat(weight, "weight", c, f32, dev),
            0 if bias is None else _flat(bias, "bias", c, f32, dev),
            0 if post_weight is None else _flat(post_weight, "post_weight", c, f32, dev))

    def _branch(self, y):
        if (y is not None) != self.branch:
            _bad("y is missing" if self.branch else "y is given, and the joint has no branch")

    def forward(self, x, y=None, offsets=None, gate=None, scale=None, shift=None, weight=None,
                bias=None, post_weight=None, out=None, stream=None):
        """(h, u), written into the tensors of ``out`` if given (h may be x's own
        memory, u may be y's; the backward passes of this joint and of the one
        before it read y and x).  h is x without a branch, u is None without
        ``pre``."""
        if _grad_on() and (x.requires_grad or y is not None and y.requires_grad or
                           gate is not None and gate.requires_grad or
                           scale is not None and scale.requires_grad or
                           shift is not None and shift.requires_grad or
                           weight is not None and weight.requires_grad or
                           bias is not None and bias.requires_grad or
                           post_weight is not None and post_weight.requires_grad):
            _by_hand(("x", x), ("y", y), ("gate", gate), ("scale", scale), ("shift", shift),
                     ("weight", weight), ("bias", bias), ("post_weight", post_weight))
        if stream is not None:
            with torch.cuda.stream(stream):
                return self.forward(x, y, offsets, gate, scale, shift, weight, bias, post_weight,
                                    out)
        self._branch(y)
        dev, s = _here()
        shape = (x.shape[0], self.channels)
        h, u = (None, None) if out is None else out
        if not self.branch:
            h = x
        elif h is None:
            h = torch.empty(shape, dtype=self.stream_dtype, device=x.device)
        if self.pre is None:
            u = None
        elif u is None:
            u = torch.empty(shape, dtype=self.dtype, device=x.device)
        _check(_fast["norm_forward"](
            self.packed, shape[0], _rows(x, "x", shape, self.stream_dtype, dev),
            _rows(y, "y", shape, self.dtype, dev) if self.branch else None,
            self._params(offsets, gate, scale, shift, weight, bias, post_weight, dev),
            _rows(h, "h", shape, self.stream_dtype, dev) if self.branch else None,
            None if u is None else _rows(u, "u", shape, self.dtype, dev), s))
        return h, u

    def backward(self, du, h, dh=None, y=None, offsets=None, gate=None, scale=None, shift=None,
                 weight=None, bias=None, post_weight=None, out=None, stream=None):
        """Gradients as a dict: dx, dy (with a branch), and of each parameter that
        is given (dgate, dscale, dshift, dweight, dbias, dpost_weight; fp32).  du is
        the gradient of u, dh that of h as the next joint sees it (None: 0), h the
        forward's (x without a branch).  ``out``: a dict of tensors to write into; dx
        may be dh's own memory, dy may be du's or y's.  Without ``pre`` du and h are
        None."""
        if _grad_on():
            _by_hand(("du", du), ("dh", dh), ("h", h), ("y", y))
        if stream is not None:
            with torch.cuda.stream(stream):
                return self.backward(du, h, dh, y, offsets, gate, scale, shift, weight, bias,
                                     post_weight, out)
        self._branch(y)
        if self.pre is not None and (du is None or h is None):
            _bad("du or h is missing")
        if self.pre is None and (du is not None or h is not None):
            _bad("du or h is given, and the joint has no norm before the next half")
        at = next((t for t in (du, dh, y) if t is not None), None)
        if at is None:
            _bad("no gradient is given")
        dev, s = _here()
        n, c, st, dt = at.shape[0], self.channels, self.stream_dtype, self.dtype
        shape, device = (n, c), at.device
        given = {} if out is None else {k: v for k, v in out.items() if v is not None}
        conds = [k for k, t in (("dgate", gate), ("dscale", scale), ("dshift", shift))
                 if t is not None]
        vectors = [k for k, t in (("dweight", weight), ("dbias", bias),
                                  ("dpost_weight", post_weight)) if t is not None]
        res = {"dx": given.pop("dx", None)}
        if res["dx"] is None:
            res["dx"] = torch.empty(shape, dtype=st, device=device)
        if self.branch:
            res["dy"] = given.pop("dy", None)
            if res["dy"] is None:
                res["dy"] = torch.empty(shape, dtype=dt, device=device)
        ptr = dict.fromkeys(_NORM_GRADS, 0)
        for names, size in ((conds, self.cond_shape), (vectors, (c,))):
            new, many = [], size[0] * c if len(size) == 2 else c
            for k in names:
                if k in given:
                    res[k] = given.pop(k)
                    ptr[k] = _flat(res[k], k, many, torch.float32, dev)
                else:
                    res[k] = None
                    new.append(k)
            if new:  # one allocation
                buf = torch.empty((len(new), *size), dtype=torch.float32, device=device)
                base = buf.data_ptr()
                for i, (k, t) in enumerate(zip(new, buf.unbind(0))):
                    res[k], ptr[k] = t, base + 4 * many * i
        if given:
            _bad(f"out has {sorted(given)[0]}, which this call does not compute")
        need = self.sizes.get(n)
        if need is None:
            b = ctypes.c_size_t()
            _check(lib().pulse_norm_sizes(self.desc, n, b))
            need = self.sizes[n] = b.value
        ws = _bytes_at(need, device)
        _check(_fast["norm_backward"](
            self.packed, n, None if du is None else _rows(du, "du", shape, dt, dev),
            None if dh is None else _rows(dh, "dh", shape, st, dev),
            None if h is None else _rows(h, "h", shape, st, dev),
            _rows(y, "y", shape, dt, dev) if self.branch else None,
            self._params(offsets, gate, scale, shift, weight, bias, post_weight, dev),
            _rows(res["dx"], "dx", shape, st, dev),
            _rows(res["dy"], "dy", shape, dt, dev) if self.branch else None,
            _pack_grads(*ptr.values()), ws.data_ptr(), need, s))
        return res


class Kept(_Owner):
    """Rows of ``channels`` channels in 8 bits: what :class:`Checkpoint` keeps."""

    __slots__ = ("tokens", "channels", "bytes", "buffer", "ptr", "home", "full")
    _memory = ("buffer",)

    def __init__(self, tokens, channels, device="cuda"):
        n = ctypes.c_size_t()
        _check(lib().pulse_keep_sizes(KeepDesc(channels, 0, BF16), tokens, n))
        self.tokens, self.channels, self.bytes = tokens, channels, n.value
        self.buffer, self.full = _bytes_at(max(n.value, 16), device), False
        self._locate()

    def _locate(self):
        self.ptr, self.home = self.buffer.data_ptr(), _home(self.buffer)


class Checkpoint:
    """Activations of ``channels`` channels kept in 8 bits until the backward
    pass.  Groups of 32 channels share a power of two; a kept value is a whole
    number of at most 127 times it, which bf16 holds exactly.  ``act`` ("gelu" or
    "silu"): the activation function that follows x, for :meth:`forward` and
    :meth:`backward`; x and its function's value and gradient are ``dtype``."""

    def __init__(self, channels, act=None, dtype=None):
        self.dtype = torch.bfloat16 if dtype is None else dtype
        self.channels, self.act = channels, act
        self.desc = KeepDesc(channels, _choice(act, _ACTS, "act"), _dtype(self.dtype))
        self.packed, self.sizes = bytes(self.desc), {}
        _check(lib().pulse_keep_sizes(self.desc, 0, ctypes.c_size_t()))

    def buffer(self, tokens, device="cuda"):
        """Room for the kept rows of ``tokens`` tokens."""
        return Kept(tokens, self.channels, device)

    def _kept(self, kept, name, tokens, dev, s, read):
        if kept.channels != self.channels or tokens is not None and kept.tokens != tokens:
            _bad(f"{name} is of {kept.tokens} tokens and {kept.channels} channels")
        if read and not kept.full:
            _bad(f"{name} holds nothing yet")
        if kept.buffer.get_device() != dev:
            _bad(f"{name} is on {kept.buffer.device}, not on the current GPU")
        if s != kept.home:
            _used_on(kept.buffer, dev)
        return kept.ptr, kept.bytes

    def save(self, x, out=None, kept=None, stream=None):
        """Keep x (into ``kept`` of an earlier call, if given), and write act(x)
        into ``out``, if given (it may be x); returns what is kept."""
        if x.requires_grad and _grad_on():
            _by_hand(("x", x))
        if stream is not None:
            with torch.cuda.stream(stream):
                return self.save(x, out, kept)
        dev, s = _here()
        n = x.shape[0]
        shape = (n, self.channels)
        if kept is None:
            kept = Kept(n, self.channels, x.device)
        _check(_fast["keep_save"](
            self.packed, n, _rows(x, "x", shape, self.dtype, dev),
            None if out is None else _rows(out, "out", shape, self.dtype, dev),
            *self._kept(kept, "kept", n, dev, s, False), s))
        kept.full = True
        return kept

    def forward(self, x, out=None, kept=None, stream=None):
        """(act(x), kept)."""
        if self.act is None:
            _bad("there is no act: use save")
        if stream is not None:
            with torch.cuda.stream(stream):
                return self.forward(x, out, kept)
        if out is None:
            out = torch.empty((x.shape[0], self.channels), dtype=self.dtype, device=x.device)
        return out, self.save(x, out, kept)

    def load(self, kept, out=None, stream=None):
        """x as kept."""
        if stream is not None:
            with torch.cuda.stream(stream):
                return self.load(kept, out)
        dev, s = _here()
        shape = (kept.tokens, self.channels)
        at = self._kept(kept, "kept", None, dev, s, True)
        if out is None:
            out = torch.empty(shape, dtype=self.dtype, device=kept.buffer.device)
        _check(_fast["keep_load"](self.packed, kept.tokens, *at,
                                  _rows(out, "out", shape, self.dtype, dev), s))
        return out

    def backward(self, da, kept, out=None, again=None, stream=None):
        """The gradient of x from that of act(x), at x as kept (``out`` may be
        da).  ``again``: receives act(x) of x as kept, in 8 bits, for the next
        layer's weight gradient."""
        if da.requires_grad and _grad_on():
            _by_hand(("da", da))
        if stream is not None:
            with torch.cuda.stream(stream):
                return self.backward(da, kept, out, again)
        dev, s = _here()
        n = da.shape[0]
        shape = (n, self.channels)
        if out is None:
            out = torch.empty(shape, dtype=self.dtype, device=da.device)
        _check(_fast["keep_backward"](
            self.packed, n, _rows(da, "da", shape, self.dtype, dev),
            *self._kept(kept, "kept", n, dev, s, True),
            _rows(out, "out", shape, self.dtype, dev),
            *((None, 0) if again is None else self._kept(again, "again", n, dev, s, False)), s))
        if again is not None:
            again.full = True
        return out

    def weight_grad(self, dy, kept, out=None, bias_out=None, accumulate=False, stream=None):
        """dw [outputs, channels] = dy^T x of x as kept (no act is applied), fp32,
        for a linear layer whose output's gradient is dy (bf16 [tokens, outputs]);
        ``bias_out`` receives dy's sums over tokens.  ``accumulate``: add to what
        ``out`` and ``bias_out`` hold."""
        if dy.requires_grad and _grad_on():
            _by_hand(("dy", dy))
        if stream is not None:
            with torch.cuda.stream(stream):
                return self.weight_grad(dy, kept, out, bias_out, accumulate)
        if dy.dim() != 2:
            _bad(f"dy is {tuple(dy.shape)}, expected [tokens, outputs]")
        dev, s = _here()
        n, m = dy.shape
        f32 = torch.float32
        if out is None:
            if accumulate:
                _bad("there is nothing to add to: out is None")
            out = torch.empty((m, self.channels), dtype=f32, device=dy.device)
        if out.shape != (m, self.channels):
            _bad(f"out is {tuple(out.shape)}, expected {(m, self.channels)}")
        need = self.sizes.get((n, m))
        if need is None:
            b = ctypes.c_size_t()
            _check(lib().pulse_keep_wgrad_sizes(self.desc, n, m, b))
            need = self.sizes[n, m] = b.value
        ws = _bytes_at(need, dy.device)
        _check(_fast["keep_wgrad"](
            self.packed, n, m, _rows(dy, "dy", (n, m), torch.bfloat16, dev),
            *self._kept(kept, "kept", n, dev, s, True),
            _flat(out, "out", m * self.channels, f32, dev),
            _flat(bias_out, "bias_out", m, f32, dev), 1 if accumulate else 0, ws.data_ptr(), need,
            s))
        return out


_SAME = object()  # Linear8.update: the bias stays


class Linear8(_Owner):
    """y = act(x W^T + bias) in 8-bit integers, for sampling: W (fp32 or bf16
    [outputs, inputs]) is laid out once, with a scale for each output channel; a
    call lays out x (bf16 [tokens, inputs]) with a scale for each token, and
    integer sums are exact.  ``bias``: fp32 [outputs], copied.  After the weights
    change, call :meth:`update`."""

    _memory, _found = ("weights", "bias"), ("ptr", "bias_ptr", "home")

    def __init__(self, weight, bias=None, act=None):
        if weight.dim() != 2:
            _bad(f"weight is {tuple(weight.shape)}, expected [outputs, inputs]")
        self.outputs, self.inputs = weight.shape
        self.desc = Lin8Desc(self.inputs, self.outputs, _choice(act, _ACTS, "act"), BF16)
        n = ctypes.c_size_t()
        _check(lib().pulse_lin8_sizes(self.desc, 0, n, None))
        self.packed, self.bytes, self.sizes = bytes(self.desc), n.value, {}
        self.weights = _bytes_at(n.value, weight.device)
        self.bias = torch.empty(self.outputs, dtype=torch.float32, device=weight.device)
        self.biased = False
        self._locate()
        self.update(weight, bias)

    def _locate(self):
        self.ptr, self.home = self.weights.data_ptr(), _home(self.weights)
        self.bias_ptr = self.bias.data_ptr() if self.biased else None

    def update(self, weight, bias=_SAME, stream=None):
        """Lay out other weights of the same shape, in place, and copy another
        ``bias``, if one is given: without it the layer keeps the one that it has,
        and with None it has none from then on.  Captured calls take the new weights
        too, and those captured with a bias the new bias (0 for none)."""
        same = bias is _SAME
        if same:
            bias = None
        if _grad_on():
            _by_hand(("weight", weight), ("bias", bias))
        if stream is not None:
            with torch.cuda.stream(stream):
                return self.update(weight, _SAME if same else bias)
        dev, s = _here()
        if tuple(weight.shape) != (self.outputs, self.inputs):
            _bad(f"weight is {tuple(weight.shape)}, expected {(self.outputs, self.inputs)}")
        at = _flat(weight, "weight", self.outputs * self.inputs, weight.dtype, dev)
        _flat(bias, "bias", self.outputs, torch.float32, dev)
        _check(lib().pulse_lin8_pack(self.desc, at, _dtype(weight.dtype), self._weights(dev, s),
                                     self.bytes, s))
        if same:
            return
        if bias is not None:
            self.bias.copy_(bias)
        elif self.biased:
            self.bias.zero_()
        self.biased = bias is not None
        self.bias_ptr = self.bias.data_ptr() if self.biased else None

    def _weights(self, dev, s):
        if self.weights.get_device() != dev:
            _bad(f"the weights are on {self.weights.device}, not on the current GPU")
        if s != self.home:
            _used_on(self.weights, dev)
            _used_on(self.bias, dev)
        return self.ptr

    def forward(self, x, out=None, stream=None):
        """y (bf16 [tokens, outputs])."""
        bf = torch.bfloat16
        if x.requires_grad and _grad_on():
            _by_hand(("x", x))
        if stream is not None:
            with torch.cuda.stream(stream):
                return self.forward(x, out)
        dev, s = _here()
        n = x.shape[0]
        if out is None:
            out = torch.empty((n, self.outputs), dtype=bf, device=x.device)
        need = self.sizes.get(n)
        if need is None:
            b = ctypes.c_size_t()
            _check(lib().pulse_lin8_sizes(self.desc, n, None, b))
            need = self.sizes[n] = b.value
        ws = _bytes_at(need, x.device) if need else None
        _check(_fast["lin8_forward"](
            self.packed, n, _rows(x, "x", (n, self.inputs), bf, dev), self._weights(dev, s),
            self.bytes, self.bias_ptr, _rows(out, "out", (n, self.outputs), bf, dev),
            ws.data_ptr() if need else None, need, s))
        return out
