"""The operators of a decode step, on the GPU: rotary positions (and their gradient), appending keys and values to a
paged cache, and attention of a batch over a shared prefix and each sequence's own tokens.  And those of prompts: attention
of packed sequences (and its gradient), attention of chunks of new tokens over a paged cache, and copies of pages.

They are the kernels whose tile graphs the simulator takes, run on the machine itself.  Functions named like the C ABI
in include/gts_serving.h marshal its descriptors; the ones below them take torch tensors:

    rotary = Rotary(128, base=10000.0, layout="half")          # frequencies, once
    cache = PagedCache.empty(n_pages, page_size, kv_heads, 128, torch.bfloat16)
    q = append_kv(q, k, v, positions, slots, rotary, cache)    # one step's new tokens
    out, lse = prefix_attention(q, cache, prefix_pages, prefix_len, page_table, lens)

    out, lse = prompt_attention(q, k, v, starts)               # packed sequences, with gradients
    out, lse = chunk_attention(q, starts, cache, page_table, lens)
    copy_pages(cache, src, dst, tokens)

Tensors are on one CUDA device, the current one, with a contiguous innermost dimension and any other strides.  Work is
enqueued on ``stream`` (default: torch's current stream); outputs and workspaces that a call allocates belong to that
stream.  There is no CPU fallback.
"""
from __future__ import annotations

import ctypes
import math
import struct

import numpy as np
import torch
from torch.autograd import forward_ad

from . import gts
from .gts import GtsError

GTS_BF16, GTS_F16, GTS_F32 = 0, 1, 2
GTS_ROTARY_HALF, GTS_ROTARY_INTERLEAVED = 0, 1

EXPORTS = ("gts_rope", "gts_append_kv", "gts_prefix_attention", "gts_prompt_attention", "gts_prompt_attention_grad",
           "gts_chunk_attention", "gts_copy_pages", "gts_attention_workspace_bytes", "gts_prompt_workspace_bytes",
           "gts_prompt_grad_workspace_bytes", "gts_chunk_workspace_bytes")

_DTYPES = {torch.bfloat16: GTS_BF16, torch.float16: GTS_F16, torch.float32: GTS_F32}
_LAYOUTS = {"half": GTS_ROTARY_HALF, "interleaved": GTS_ROTARY_INTERLEAVED}

_vp, _u32, _i32, _i64, _f32, _sz = (ctypes.c_void_p, ctypes.c_uint32, ctypes.c_int32, ctypes.c_int64, ctypes.c_float,
                                    ctypes.c_size_t)


class HeadsDesc(ctypes.Structure):
    _fields_ = [("data", _vp), ("token_stride", _i64), ("head_stride", _i64)]


class CacheDesc(ctypes.Structure):
    _fields_ = [("k", _vp), ("v", _vp),
                ("k_page_stride", _i64), ("k_token_stride", _i64), ("k_head_stride", _i64),
                ("v_page_stride", _i64), ("v_token_stride", _i64), ("v_head_stride", _i64),
                ("n_pages", _u32), ("page_size", _u32), ("kv_heads", _u32), ("head_dim", _u32), ("dtype", _i32)]


class RotaryDesc(ctypes.Structure):
    _fields_ = [("units", _vp), ("rot_dim", _u32), ("layout", _i32), ("factor", _f32), ("transposed", _u32)]


class RopeDesc(ctypes.Structure):
    _fields_ = [("n_tokens", _u32), ("q_heads", _u32), ("kv_heads", _u32), ("head_dim", _u32), ("dtype", _i32),
                ("positions", _vp), ("rotary", RotaryDesc), ("q", HeadsDesc), ("k", HeadsDesc), ("q_out", HeadsDesc),
                ("k_out", HeadsDesc)]


class AppendDesc(ctypes.Structure):
    _fields_ = [("n_tokens", _u32), ("q_heads", _u32), ("positions", _vp), ("slots", _vp), ("rotary", RotaryDesc),
                ("q", HeadsDesc), ("k", HeadsDesc), ("v", HeadsDesc), ("q_out", HeadsDesc), ("cache", CacheDesc),
                ("d_status", _vp)]


class AttentionDesc(ctypes.Structure):
    _fields_ = [("n_seqs", _u32), ("n_new", _u32), ("q_heads", _u32), ("scale", _f32),
                ("q", _vp), ("q_seq_stride", _i64), ("q_token_stride", _i64), ("q_head_stride", _i64),
                ("out", _vp), ("out_seq_stride", _i64), ("out_token_stride", _i64), ("out_head_stride", _i64),
                ("lse", _vp), ("cache", CacheDesc), ("prefix_pages", _vp), ("prefix_len", _u32), ("page_table", _vp),
                ("max_pages", _u32), ("lens", _vp), ("workspace", _vp), ("workspace_bytes", _sz), ("d_status", _vp)]


class PromptDesc(ctypes.Structure):
    _fields_ = [("n_seqs", _u32), ("n_tokens", _u32), ("q_heads", _u32), ("kv_heads", _u32), ("head_dim", _u32), ("dtype", _i32),
                ("causal", _u32), ("zero_rest", _u32), ("scale", _f32), ("starts", _vp), ("q", HeadsDesc), ("k", HeadsDesc),
                ("v", HeadsDesc), ("out", HeadsDesc), ("low", HeadsDesc), ("lse", _vp), ("workspace", _vp), ("workspace_bytes", _sz), ("d_status", _vp)]


class PromptGradDesc(ctypes.Structure):
    _fields_ = [("forward", PromptDesc), ("dout", HeadsDesc), ("dlse", _vp), ("dq", HeadsDesc), ("dk", HeadsDesc), ("dv", HeadsDesc)]


class ChunkDesc(ctypes.Structure):
    _fields_ = [("n_seqs", _u32), ("n_tokens", _u32), ("q_heads", _u32), ("zero_rest", _u32), ("scale", _f32), ("starts", _vp),
                ("q", HeadsDesc), ("out", HeadsDesc), ("lse", _vp), ("cache", CacheDesc), ("page_table", _vp), ("max_pages", _u32),
                ("lens", _vp), ("workspace", _vp), ("workspace_bytes", _sz), ("d_status", _vp)]


class CopyPagesDesc(ctypes.Structure):
    _fields_ = [("n_copies", _u32), ("src", _vp), ("dst", _vp), ("tokens", _vp), ("cache", CacheDesc), ("into", CacheDesc),
                ("d_status", _vp)]


# The same layouts as format strings: the torch entry points pack a descriptor in one go, which takes a fifth of the time of
# filling the structures above (about 2 against 10 us a call).
_HEADS_FORMAT, _ROTARY_FORMAT, _CACHE_FORMAT = "Pqq", "PIifI", "PPqqqqqqIIIIi4x"
_ROPE = struct.Struct("@IIIIiP" + _ROTARY_FORMAT + 4 * _HEADS_FORMAT)
_APPEND = struct.Struct("@IIPP" + _ROTARY_FORMAT + 4 * _HEADS_FORMAT + _CACHE_FORMAT + "P")
_ATTENTION = struct.Struct("@IIIf" + 2 * "Pqqq" + "P" + _CACHE_FORMAT + "PI4xPI4xPPNP")
_PROMPT_FORMAT = "IIIIIiIIf4xP" + 5 * _HEADS_FORMAT + "PPNP"
_PROMPT = struct.Struct("@" + _PROMPT_FORMAT)
_PROMPT_GRAD = struct.Struct("@" + _PROMPT_FORMAT + _HEADS_FORMAT + "P" + 3 * _HEADS_FORMAT)
_CHUNK = struct.Struct("@IIIIf4xP" + 2 * _HEADS_FORMAT + "P" + _CACHE_FORMAT + "PI4xPPNP")
_COPY_PAGES = struct.Struct("@I4xPPP" + 2 * _CACHE_FORMAT + "P")

_lib = None


def _load():
    global _lib
    if _lib is None:
        lib = gts.load()
        for name in EXPORTS:
            f = getattr(lib, name)
            f.argtypes, f.restype = ([_vp], _sz) if name.endswith("_bytes") else ([_vp, _vp], _i32)
        _lib = lib
    return _lib


# ---------------------------------------------------------------- raw ABI (same names)
def gts_rope(desc: RopeDesc, stream: int = 0):
    gts._check(_load().gts_rope(ctypes.byref(desc), stream))


def gts_append_kv(desc: AppendDesc, stream: int = 0):
    gts._check(_load().gts_append_kv(ctypes.byref(desc), stream))


def gts_prefix_attention(desc: AttentionDesc, stream: int = 0):
    gts._check(_load().gts_prefix_attention(ctypes.byref(desc), stream))


def gts_attention_workspace_bytes(desc: AttentionDesc) -> int:
    return int(_load().gts_attention_workspace_bytes(ctypes.byref(desc)))


def gts_prompt_attention(desc: PromptDesc, stream: int = 0):
    gts._check(_load().gts_prompt_attention(ctypes.byref(desc), stream))


def gts_prompt_workspace_bytes(desc: PromptDesc) -> int:
    return int(_load().gts_prompt_workspace_bytes(ctypes.byref(desc)))


def gts_prompt_attention_grad(desc: PromptGradDesc, stream: int = 0):
    gts._check(_load().gts_prompt_attention_grad(ctypes.byref(desc), stream))


def gts_prompt_grad_workspace_bytes(desc: PromptGradDesc) -> int:
    return int(_load().gts_prompt_grad_workspace_bytes(ctypes.byref(desc)))


def gts_chunk_attention(desc: ChunkDesc, stream: int = 0):
    gts._check(_load().gts_chunk_attention(ctypes.byref(desc), stream))


def gts_chunk_workspace_bytes(desc: ChunkDesc) -> int:
    return int(_load().gts_chunk_workspace_bytes(ctypes.byref(desc)))


def gts_copy_pages(desc: CopyPagesDesc, stream: int = 0):
    gts._check(_load().gts_copy_pages(ctypes.byref(desc), stream))


# ---------------------------------------------------------------- torch tensors
def _refuse(msg):
    raise GtsError(gts.GTS_ERR_INVALID_ARG, msg)


def _tensor(t, name, dims, dtype=None, device=None):
    """Shape and strides of a tensor with a contiguous innermost dimension on a CUDA device (or of a type, on a device)."""
    shape = t.shape
    if len(shape) != dims:
        _refuse(f"{name}: {dims} dimensions wanted, got {len(shape)}")
    if device is None:
        if not t.is_cuda:
            _refuse(f"{name} is not on a CUDA device")
    elif t.device != device or t.dtype != dtype:
        _refuse(f"{name}: {dtype} on {device} wanted, got {t.dtype} on {t.device}")
    strides = t.stride()
    if strides[-1] != 1 and shape[-1] > 1:
        _refuse(f"{name}: the innermost dimension must be contiguous")
    return shape, strides


def _index(t, name, shape, dtype, device):
    """The address of a contiguous index tensor of the given shape (None: any extent)."""
    if t.dtype != dtype or t.device != device:
        _refuse(f"{name}: {dtype} on {device} wanted, got {t.dtype} on {t.device}")
    got = t.shape
    if got != shape and (len(got) != len(shape) or any(w is not None and w != n for w, n in zip(shape, got))) or \
            not t.is_contiguous():
        _refuse(f"{name}: contiguous {list(shape)} wanted, got {list(got)}")
    return t.data_ptr()


def _status(t, device):
    return 0 if t is None else _index(t, "status", (1,), torch.int32, device)


# (the same as torch.cuda's functions, without their checks for a first use of CUDA: a CUDA tensor exists here)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)


def _handle(stream, device):
    """The stream's handle, for tensors that have to be on the current device."""
    index = device.index
    if index != _current_device():
        _refuse(f"tensors are on {device}, the current device is cuda:{_current_device()}")
    if stream is not None:
        return stream.cuda_stream
    return _raw_stream(index) if _raw_stream is not None else torch.cuda.current_stream().cuda_stream


def _empty(shape, dtype, device, stream):
    """Memory that belongs to the stream the call runs on."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=device)


def _output(out, name, shape, dtype, device, stream):
    """(tensor, strides)"""
    if out is None:
        out = torch.empty(shape, dtype=dtype, device=device) if stream is None else _empty(shape, dtype, device, stream)
        return out, out.stride()
    got, strides = _tensor(out, name, len(shape), dtype, device)
    if got != shape:
        _refuse(f"{name}: {list(shape)} wanted, got {list(got)}")
    return out, strides


class _Fixed:
    """Attributes are set once, by the constructor: a descriptor made from them stays true."""

    def __setattr__(self, name, value):
        _refuse(f"{type(self).__name__}.{name} cannot be set: make a new {type(self).__name__}")

    def __delattr__(self, name):
        self.__setattr__(name, None)


class Rotary(_Fixed):
    """The rotation of a model's heads: the frequencies of its pairs, held on the device in turns a position.

    Pair i of ``rot_dim / 2`` turns by ``base ** (-2 i / rot_dim)`` radians a position.  ``layout``: "half" pairs the
    values i and i + rot_dim / 2, "interleaved" 2 i and 2 i + 1; values after ``rot_dim`` (default: the whole head) are
    left as they are.  ``scaling`` stretches positions for contexts longer than those of training:

    * ``{"kind": "linear", "factor": s}``: every frequency divided by s;
    * ``{"kind": "ntk", "factor": s}``: the base times ``s ** (rot_dim / (rot_dim - 2))``, which divides the lowest
      frequency by s and keeps the highest;
    * ``{"kind": "by_parts", "factor": s, "original_len": L, "low": a, "high": b}``: frequencies of fewer than a
      turns in L positions divided by s, those of more than b kept, between them a blend that is linear in the turns
      (a model whose blend is linear in the pair's index has other frequencies); rotated values times ``magnitude``
      (default ``0.1 ln s + 1``).
    """

    def __init__(self, head_dim, rot_dim=None, base=10000.0, layout="half", scaling=None, device="cuda"):
        rot_dim = head_dim if rot_dim is None else rot_dim
        if rot_dim % 2 or not 0 <= rot_dim <= head_dim:
            _refuse(f"rot_dim must be even and at most head_dim, got {rot_dim} of {head_dim}")
        if layout not in _LAYOUTS:
            _refuse(f"unknown rotary layout {layout!r}")
        if not base > 0:
            _refuse("base must be positive")
        theta, factor = self._frequencies(rot_dim, base, scaling)
        units = [round(float(t) / (2 * math.pi) * 2.0 ** 64) % 2 ** 64 for t in theta]
        units = torch.from_numpy(np.array(units, np.uint64).view(np.int64)).to(device)
        vars(self).update(head_dim=head_dim, rot_dim=rot_dim, layout=layout, theta=theta, factor=factor, units=units,
                          device=units.device)
        self._describe()

    def _describe(self):
        at = _index(self.units, "units", (self.rot_dim // 2,), torch.int64, self.device)
        vars(self).update(_at=at, _values=[(at, self.rot_dim, _LAYOUTS[self.layout], self.factor, t) for t in (0, 1)])

    def _descriptor(self, transposed):
        """The rotation's part of a call's descriptor; made again where the frequencies have moved (a copy of this object)."""
        if self.units.data_ptr() != self._at:
            self._describe()
        return self._values[transposed]

    @staticmethod
    def _frequencies(rot_dim, base, scaling):
        """Radians a position of each pair, in 64 bits, and the factor of the rotated values."""
        i = np.arange(rot_dim // 2, dtype=np.float64)
        if scaling is None:
            return base ** (-2.0 * i / max(rot_dim, 1)), 1.0
        scaling = dict(scaling)
        kind, s = scaling.pop("kind", None), float(scaling.pop("factor", 0.0))
        if not s > 0:
            _refuse("scaling needs a positive factor")
        if kind == "ntk" and rot_dim > 2:
            base = base * s ** (rot_dim / (rot_dim - 2))
        theta, magnitude = base ** (-2.0 * i / max(rot_dim, 1)), 1.0
        if kind == "linear":
            theta = theta / s
        elif kind == "by_parts":
            length = scaling.pop("original_len", None)
            low, high = float(scaling.pop("low", 1.0)), float(scaling.pop("high", 32.0))
            if not length or not high > low:
                _refuse("by_parts scaling needs original_len and low < high")
            keep = np.clip((length * theta / (2 * math.pi) - low) / (high - low), 0.0, 1.0)
            theta = theta * keep + theta / s * (1.0 - keep)
            magnitude = float(scaling.pop("magnitude", 0.1 * math.log(s) + 1.0))
        elif kind != "ntk":
            _refuse(f"unknown scaling {kind!r}")
        if scaling:
            _refuse(f"unknown scaling entries {sorted(scaling)}")
        return theta, magnitude


class PagedCache(_Fixed):
    """Keys and values in pages: two [pages, page_size, kv_heads, head_dim] tensors of any outer strides.  Other tensors (a
    larger cache) take another PagedCache."""

    def __init__(self, k, v):
        vars(self).update(k=k, v=v)
        self._describe()

    def _describe(self):
        k, v = self.k, self.v
        _tensor(k, "k cache", 4)
        _tensor(v, "v cache", 4, k.dtype, k.device)
        if k.shape != v.shape:
            _refuse(f"k and v caches differ: {list(k.shape)}, {list(v.shape)}")
        if k.dtype not in _DTYPES:
            _refuse(f"cache: bfloat16, float16 or float32 wanted, got {k.dtype}")
        n_pages, page_size, kv_heads, head_dim = k.shape
        if page_size < 1:
            _refuse("page_size must be positive")
        vars(self).update(dtype=k.dtype, device=k.device, n_pages=n_pages, page_size=page_size, kv_heads=kv_heads, head_dim=head_dim,
                          _values=(k.data_ptr(), v.data_ptr(), *k.stride()[:3], *v.stride()[:3], *k.shape, _DTYPES[k.dtype]))

    def _descriptor(self):
        """The cache's part of a call's descriptor; made again where its tensors have moved (given other memory in place, or
        copied with this object)."""
        if self.k.data_ptr() != self._values[0] or self.v.data_ptr() != self._values[1]:
            self._describe()
        return self._values

    @classmethod
    def empty(cls, n_pages, page_size, kv_heads, head_dim, dtype, order="tokens", device="cuda"):
        """``order``: "tokens" keeps the heads of a token together, "heads" the tokens of a head."""
        if order not in ("tokens", "heads"):
            _refuse(f"unknown order {order!r}")

        def one():
            if order == "tokens":
                return torch.empty((n_pages, page_size, kv_heads, head_dim), dtype=dtype, device=device)
            return torch.empty((n_pages, kv_heads, page_size, head_dim), dtype=dtype, device=device).transpose(1, 2)
        return cls(one(), one())


def _rope_call(q, k, positions, rotary, transposed, out_q, out_k, stream):
    shape, qs = _tensor(q, "q", 3)
    device, dtype = q.device, q.dtype
    handle = _handle(stream, device)
    dt = _DTYPES.get(dtype)
    if dt is None:
        _refuse(f"q: bfloat16, float16 or float32 wanted, got {q.dtype}")
    T, heads, dim = shape
    if dim != rotary.head_dim or rotary.device != device:
        _refuse(f"q has heads of {dim} on {device}, the rotary is of {rotary.head_dim} on {rotary.device}")
    pos = _index(positions, "positions", (T,), torch.int32, device)
    kh, kp, kop, ks, kos = 0, 0, 0, (0, 0), (0, 0)
    if k is not None:
        kshape, ks = _tensor(k, "k", 3, dtype, device)
        kh = kshape[1]
        if kshape[0] != T or kshape[2] != dim:
            _refuse(f"k: [{T}, kv_heads, {dim}] wanted, got {list(kshape)}")
        out_k, kos = _output(out_k, "out_k", kshape, dtype, device, stream)
        if kh:
            kp, kop = k.data_ptr(), out_k.data_ptr()
    else:
        out_k = None
    out_q, qos = _output(out_q, "out_q", shape, dtype, device, stream)
    if T and (heads or kh):
        gts._check((_lib or _load()).gts_rope(_ROPE.pack(
            T, heads, kh, dim, dt, pos, *rotary._descriptor(transposed), q.data_ptr(), qs[0], qs[1], kp, ks[0], ks[1],
            out_q.data_ptr(), qos[0], qos[1], kop, kos[0], kos[1]), handle))
    return out_q, out_k


class _Rope(torch.autograd.Function):
    """The rotation of each pair, or its transpose.  Either is linear, so its gradient is the other one and its tangent is itself,
    through this function again: derivatives of any order are."""

    @staticmethod
    def forward(q, k, positions, rotary, transposed):
        return _rope_call(q, k, positions, rotary, transposed, None, None, None)

    @staticmethod
    def setup_context(ctx, inputs, output):
        _, _, positions, ctx.rotary, ctx.transposed = inputs
        ctx.save_for_backward(positions)
        ctx.save_for_forward(positions)

    @staticmethod
    def backward(ctx, dq, dk):
        want_q, want_k = ctx.needs_input_grad[:2]
        x = [_inner(t) for t, want in ((dq, want_q), (dk, want_k)) if want]
        got = list(_Rope.apply(x[0], x[1] if len(x) > 1 else None, ctx.saved_tensors[0], ctx.rotary, 1 - ctx.transposed))
        return got.pop(0) if want_q else None, got.pop(0) if want_k else None, None, None, None

    @staticmethod
    def jvp(ctx, tq, tk, *_):
        return _Rope.apply(_inner(tq), _inner(tk), ctx.saved_tensors[0], ctx.rotary, ctx.transposed)


def _inner(t):
    return t if t is None or t.stride(-1) == 1 else t.contiguous()


def _differentiated(t):
    """Whether a gradient or a tangent goes through t."""
    return t is not None and (t.requires_grad and torch.is_grad_enabled() or
                              getattr(forward_ad, "_current_level", 0) >= 0 and forward_ad.unpack_dual(t).tangent is not None)


def _rope(q, k, positions, rotary, transposed, out_q, out_k, stream):
    if _differentiated(q) or _differentiated(k):
        if out_q is not None or out_k is not None or stream is not None:
            _refuse("rope: gradients need the call's own outputs and the current stream")
        return _Rope.apply(q, k, positions, rotary, transposed)
    return _rope_call(q, k, positions, rotary, transposed, out_q, out_k, stream)


def rope(q, k, positions, rotary, out_q=None, out_k=None, stream=None):
    """q [tokens, heads, head_dim] and k [tokens, kv_heads, head_dim] (or None) rotated to ``positions`` [tokens] int32:
    (q', k').  ``out_q`` / ``out_k`` may be q and k themselves.  With outputs and stream left to the call, gradients (of any
    order) and tangents flow through it."""
    return _rope(q, k, positions, rotary, 0, out_q, out_k, stream)


def rope_grad(dq, dk, positions, rotary, out_dq=None, out_dk=None, stream=None):
    """The gradients of q and k from those of ``rope``'s results: the transposed rotation.  Differentiable like ``rope``."""
    return _rope(dq, dk, positions, rotary, 1, out_dq, out_dk, stream)


def append_kv(q, k, v, positions, slots, rotary, cache, out_q=None, status=None, stream=None):
    """Rotates q and k of every token to its position, writes k and v to the cache, returns the rotated q (no gradients).

    q [tokens, heads, head_dim], k and v [tokens, kv_heads, head_dim], positions [tokens] int32; slots [tokens] int64,
    page * page_size + index within the page, no two alike; a negative one is a padding row, of which nothing is
    written to the cache.  A slot beyond the cache writes nothing and stores GTS_ERR_INVALID_PARAMS to ``status``
    (int32 [1] on the device), where given."""
    cache_values = cache._descriptor()
    dtype, device = cache.dtype, cache.device
    shape, qs = _tensor(q, "q", 3, dtype, device)
    handle = _handle(stream, device)
    T, heads, dim = shape
    if dim != cache.head_dim or dim != rotary.head_dim or rotary.device != device:
        _refuse(f"heads of {dim} (q), {cache.head_dim} (cache) and {rotary.head_dim} (rotary, on {rotary.device})")
    (kshape, ks), (vshape, vs) = _tensor(k, "k", 3, dtype, device), _tensor(v, "v", 3, dtype, device)
    if kshape != (T, cache.kv_heads, dim) or vshape != kshape:
        _refuse(f"k and v: {[T, cache.kv_heads, dim]} wanted, got {list(kshape)} and {list(vshape)}")
    pos = _index(positions, "positions", (T,), torch.int32, device)
    at = _index(slots, "slots", (T,), torch.int64, device)
    st = _status(status, device)
    out_q, qos = _output(out_q, "out_q", shape, dtype, device, stream)
    if T:
        gts._check((_lib or _load()).gts_append_kv(_APPEND.pack(
            T, heads, pos, at, *rotary._descriptor(0), q.data_ptr(), qs[0], qs[1], k.data_ptr(), ks[0], ks[1], v.data_ptr(),
            vs[0], vs[1], out_q.data_ptr(), qos[0], qos[1], *cache_values, st), handle))
    return out_q


def _workspace_bytes(shape, cache_values, prefix_len, max_pages):
    return int(_load().gts_attention_workspace_bytes(_ATTENTION.pack(
        *shape[:3], 1.0, 0, 0, 0, 0, 0, 0, 0, 0, 0, *cache_values, 0, prefix_len, 0, max_pages, 0, 0, 0, 0)))


def attention_workspace(cache, q, prefix_len, page_table, stream=None):
    """A workspace for ``prefix_attention`` calls of this shape; calls that may run at the same time need one each."""
    need = _workspace_bytes(q.shape, cache._descriptor(), prefix_len, page_table.shape[1])
    return _empty(max(need, 16), torch.uint8, q.device, stream)


def prefix_attention(q, cache, prefix_pages, prefix_len, page_table, lens, scale=None, out=None, lse=None,
                     workspace=None, status=None, stream=None):
    """Attention of q [seqs, new, heads, head_dim] over a shared prefix and each sequence's own tokens: (out, lse), without
    gradients.

    The prefix is the first ``prefix_len`` tokens of the pages in ``prefix_pages`` (int32); sequence b's own tokens are
    the first ``lens[b]`` (int32) of the pages in ``page_table[b]`` (int32 [seqs, max_pages]; entries past its length
    are not looked at).  They include the ``new`` newest, whose keys are in the cache already: query i sees the whole
    prefix and its sequence's tokens up to its own.  ``scale``: of the products (default 1 / sqrt(head_dim)).  A query
    that sees nothing gets zeros and lse = -inf (float32 [seqs, new, heads]).  A page number or a length out of range
    is not followed and stores GTS_ERR_INVALID_PARAMS to ``status`` (int32 [1] on the device), where given.  A kernel whose
    waits run out (after two seconds) stores GTS_ERR_STEP_LIMIT there, and rows that miss a part are NaN."""
    cache_values = cache._descriptor()
    dtype, device = cache.dtype, cache.device
    shape, qs = _tensor(q, "q", 4, dtype, device)
    handle = _handle(stream, device)
    B, new, heads, dim = shape
    if dim != cache.head_dim:
        _refuse(f"heads of {dim} (q) and {cache.head_dim} (cache)")
    if not 0 <= prefix_len <= 1 << 30:
        _refuse(f"prefix_len out of range: {prefix_len}")
    prefix_at = _index(prefix_pages, "prefix_pages", (None,), torch.int32, device)
    if prefix_pages.shape[0] * cache.page_size < prefix_len:
        _refuse(f"{prefix_pages.shape[0]} prefix pages of {cache.page_size} hold no {prefix_len} tokens")
    table_at = _index(page_table, "page_table", (B, None), torch.int32, device)
    max_pages = page_table.shape[1]
    lens_at = _index(lens, "lens", (B,), torch.int32, device)
    st = _status(status, device)
    out, os = _output(out, "out", shape, dtype, device, stream)
    if lse is None:
        lse = _empty((B, new, heads), torch.float32, device, stream)
        lse_at = lse.data_ptr()
    else:
        lse_at = _index(lse, "lse", (B, new, heads), torch.float32, device)
    if workspace is None:
        workspace = _empty(max(_workspace_bytes(shape, cache_values, prefix_len, max_pages), 16), torch.uint8, device, stream)
    elif workspace.device != device or not workspace.is_contiguous():
        _refuse(f"workspace: contiguous on {device} wanted")
    if B and new:
        gts._check((_lib or _load()).gts_prefix_attention(_ATTENTION.pack(
            B, new, heads, 1.0 / math.sqrt(dim) if scale is None else scale, q.data_ptr(), qs[0], qs[1], qs[2],
            out.data_ptr(), os[0], os[1], os[2], lse_at, *cache_values, prefix_at, prefix_len, table_at, max_pages, lens_at,
            workspace.data_ptr(), workspace.nbytes, st), handle))
    return out, lse


# ---------------------------------------------------------------- prompts
def _heads(t, strides):
    return t.data_ptr(), strides[0], strides[1]


def _workspace(workspace, need, device, stream):
    if workspace is None:
        return _empty(max(need, 16), torch.uint8, device, stream)
    if workspace.device != device or not workspace.is_contiguous():
        _refuse(f"workspace: contiguous on {device} wanted")
    return workspace


def _prompt_shape(q, k, v, starts):
    """(values of the descriptor up to dtype, strides of q, k and v, device, address of starts)"""
    shape, qs = _tensor(q, "q", 3)
    device, dtype = q.device, q.dtype
    dt = _DTYPES.get(dtype)
    if dt is None or dt == GTS_F32:
        _refuse(f"q: bfloat16 or float16 wanted, got {dtype}")
    T, heads, dim = shape
    (kshape, ks), (vshape, vs) = _tensor(k, "k", 3, dtype, device), _tensor(v, "v", 3, dtype, device)
    if kshape[0] != T or kshape[2] != dim or vshape != kshape:
        _refuse(f"k and v: [{T}, kv_heads, {dim}] wanted, got {list(kshape)} and {list(vshape)}")
    return (_sequences(starts), T, heads, kshape[1], dim, dt), qs, ks, vs, device, _index(starts, "starts", (None,), torch.int32, device)


def _sequences(starts):
    if starts.dim() != 1 or starts.shape[0] < 1:
        _refuse(f"starts: one dimension of sequences + 1 wanted, got {list(starts.shape)}")
    return starts.shape[0] - 1


def _scale(scale, dim):
    if scale is None:
        return 1.0 / math.sqrt(dim)
    scale = float(scale)
    if not 0.0 < scale < 3e38:
        _refuse(f"scale must be positive, got {scale}")
    return scale


_NO_HEADS = (0, 0, 0)


def prompt_workspace(q, k, starts, stream=None):
    """A workspace for ``prompt_attention`` calls of this shape; calls that may run at the same time need one each, and one that a
    captured call was given lives as long as the graph."""
    T, heads, dim = q.shape
    need = _load().gts_prompt_workspace_bytes(_PROMPT.pack(
        _sequences(starts), T, heads, k.shape[1], dim, _DTYPES.get(q.dtype, -1), 0, 0, 1.0, 0, *(5 * _NO_HEADS), 0, 0, 0, 0))
    return _empty(max(int(need), 16), torch.uint8, q.device, stream)


def _prompt_call(q, k, v, starts, causal, scale, out, lse, low, workspace, status, stream):
    shape, qs, ks, vs, device, starts_at = _prompt_shape(q, k, v, starts)
    handle = _handle(stream, device)
    T, heads = shape[1:3]
    scale, st, zero = _scale(scale, shape[4]), _status(status, device), (out is None) + 2 * (lse is None)
    out, os = _output(out, "out", q.shape, q.dtype, device, stream)
    if lse is None:
        lse = _empty((T, heads), torch.float32, device, stream)
    lse_at = _index(lse, "lse", (T, heads), torch.float32, device)
    low_at = _low(low, q, device)
    lib = _lib or _load()
    if workspace is None:
        workspace = _workspace(None, lib.gts_prompt_workspace_bytes(_PROMPT.pack(*shape, 0, 0, 1.0, 0, *(5 * _NO_HEADS), 0, 0, 0, 0)), device,
                               stream)
    else:
        _workspace(workspace, 0, device, stream)
    if T:
        gts._check(lib.gts_prompt_attention(_PROMPT.pack(
            *shape, bool(causal), zero, scale, starts_at, *_heads(q, qs), *_heads(k, ks), *_heads(v, vs), *_heads(out, os), *low_at,
            lse_at, workspace.data_ptr(), workspace.nbytes, st), handle))
    return out, lse


def _low(low, q, device):
    if low is None:
        return _NO_HEADS
    shape, strides = _tensor(low, "low", 3, q.dtype, device)
    if shape != q.shape:
        _refuse(f"low: {list(q.shape)} wanted, got {list(shape)}")
    return _heads(low, strides)


class _Prompt(torch.autograd.Function):
    # (forward with a context: the form with setup_context takes 25 us more of the host's time a call)
    @staticmethod
    def forward(ctx, q, k, v, starts, causal, scale, status):
        low = torch.empty(q.shape, dtype=q.dtype, device=q.device)
        out, lse = _prompt_call(q, k, v, starts, causal, scale, None, None, low, None, status, None)
        ctx.causal, ctx.scale, ctx.status = causal, scale, status
        ctx.set_materialize_grads(False)
        ctx.save_for_backward(q, k, v, starts, out, lse, low)
        return out, lse

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dout, dlse):
        q, k, v, starts, out, lse, low = ctx.saved_tensors
        if dout is None and dlse is None:
            return (None,) * 7
        dout = torch.zeros_like(out) if dout is None else _inner(dout)
        dlse = None if dlse is None else dlse.contiguous()
        got = prompt_attention_grad(dout, q, k, v, out, lse, starts, causal=ctx.causal, scale=ctx.scale, dlse=dlse, low=low, status=ctx.status)
        return *(g if want else None for g, want in zip(got, ctx.needs_input_grad)), None, None, None, None


def prompt_attention(q, k, v, starts, causal=True, scale=None, out=None, lse=None, low=None, workspace=None, status=None, stream=None):
    """Attention of packed sequences over themselves: (out, lse).

    q [tokens, heads, head_dim], k and v [tokens, kv_heads, head_dim], bfloat16 or float16, heads of 64 or 128; sequence b's tokens
    are the rows ``starts[b]`` .. ``starts[b + 1] - 1`` (int32 [seqs + 1], rising, on the device).  A query sees its sequence's keys
    up to its own (``causal``) or all of them; ``scale``: of the products, positive (default 1 / sqrt(head_dim)).  lse (float32
    [tokens, heads]) is the logarithm of the sum of exponentials; ``low``, a tensor like out, gets what rounding took from out, for
    ``prompt_attention_grad``.  Rows of no sequence get zeros and lse = -inf, and so does a row whose visible scores are all -inf; rows of no
    sequence of a given ``out`` or ``lse`` are left as they are.  A row that sees a score of +inf or NaN is NaN.  Results may not
    overlap what the call reads.  Starts out of range are clamped and store GTS_ERR_INVALID_PARAMS to ``status`` (int32 [1]
    on the device), where given.  A kernel whose waits run out (after two seconds) stores GTS_ERR_STEP_LIMIT there, and its rows are NaN.

    With outputs, workspace and stream left to the call, gradients flow from out and lse to q, k and v (once; torch.func does not go through).
    The graph holds q, k, v, out, lse and ``low``, which is as large as out.  A backward pass that is
    captured into a graph while another graph of the same leaves lives wants that one made on the capturing stream: torch ties
    a leaf's gradient to the stream of its first use."""
    if _differentiated(q) or _differentiated(k) or _differentiated(v):
        if out is not None or lse is not None or low is not None or workspace is not None or stream is not None:
            _refuse("prompt_attention: gradients need the call's own outputs and workspace and the current stream")
        return _Prompt.apply(q, k, v, starts, causal, scale, status)
    return _prompt_call(q, k, v, starts, causal, scale, out, lse, low, workspace, status, stream)


def prompt_attention_grad(dout, q, k, v, out, lse, starts, causal=True, scale=None, dlse=None, low=None, out_dq=None, out_dk=None,
                          out_dv=None, workspace=None, status=None, stream=None):
    """The gradients (dq, dk, dv) of ``prompt_attention`` from those of its results (``dlse`` [tokens, heads] float32, default none);
    ``out``, ``lse`` and ``low`` are what it gave (without ``low`` dq and dk are 4 to 10% less exact).  Every sum has one order, so
    results repeat bit for bit.  float16: what is summed for dq and dk is held to 2^-39 of 2 max |dout_i| max |v_j| + max |dlse_i| (norms
    of rows, over the call).  Rows of no sequence get zeros; those of a given output are left as they are.  Results may not overlap
    what the call reads.  ``workspace``: of gts_prompt_grad_workspace_bytes, by default the call's own."""
    shape, qs, ks, vs, device, starts_at = _prompt_shape(q, k, v, starts)
    handle = _handle(stream, device)
    T, heads = shape[1:3]
    scale, st = _scale(scale, shape[4]), _status(status, device)
    (oshape, os), (dshape, ds) = _tensor(out, "out", 3, q.dtype, device), _tensor(dout, "dout", 3, q.dtype, device)
    if oshape != q.shape or dshape != q.shape:
        _refuse(f"out and dout: {list(q.shape)} wanted, got {list(oshape)} and {list(dshape)}")
    lse_at = _index(lse, "lse", (T, heads), torch.float32, device)
    dlse_at = 0 if dlse is None else _index(dlse, "dlse", (T, heads), torch.float32, device)
    low_at = _low(low, q, device)
    zero = (out_dq is None) + 2 * (out_dk is None) + 4 * (out_dv is None)
    dq, dqs = _output(out_dq, "out_dq", q.shape, q.dtype, device, stream)
    dk, dks = _output(out_dk, "out_dk", k.shape, q.dtype, device, stream)
    dv, dvs = _output(out_dv, "out_dv", v.shape, q.dtype, device, stream)
    lib = _lib or _load()

    def pack(work_at, work_bytes):
        return _PROMPT_GRAD.pack(
            *shape, bool(causal), zero, scale, starts_at, *_heads(q, qs), *_heads(k, ks), *_heads(v, vs), *_heads(out, os), *low_at,
            lse_at, work_at, work_bytes, st, *_heads(dout, ds), dlse_at, *_heads(dq, dqs), *_heads(dk, dks), *_heads(dv, dvs))
    if workspace is None:
        workspace = _workspace(None, lib.gts_prompt_grad_workspace_bytes(pack(0, 0)), device, stream)
    else:
        _workspace(workspace, 0, device, stream)
    if T:
        gts._check(lib.gts_prompt_attention_grad(pack(workspace.data_ptr(), workspace.nbytes), handle))
    return dq, dk, dv


def _chunk_bytes(shape, cache_values, max_pages):
    return int(_load().gts_chunk_workspace_bytes(_CHUNK.pack(*shape, 0, 1.0, 0, *(2 * _NO_HEADS), 0, *cache_values, 0, max_pages, 0, 0, 0, 0)))


def chunk_workspace(q, starts, cache, page_table, stream=None):
    """A workspace for ``chunk_attention`` calls of this shape; calls that may run at the same time need one each, and one that a
    captured call was given lives as long as the graph."""
    need = _chunk_bytes((_sequences(starts), *q.shape[:2]), cache._descriptor(), page_table.shape[1])
    return _empty(max(need, 16), torch.uint8, q.device, stream)


def chunk_attention(q, starts, cache, page_table, lens, scale=None, out=None, lse=None, workspace=None, status=None, stream=None):
    """Attention of chunks of new tokens over a paged cache: (out, lse), without gradients.

    q [tokens, heads, head_dim] holds the new tokens of all sequences, packed: those of sequence b are the rows ``starts[b]`` ..
    ``starts[b + 1] - 1`` (int32 [seqs + 1], rising).  Their keys and values are in the cache already, as the newest of the
    sequence's first ``lens[b]`` tokens (int32; a negative length is none) of the pages in ``page_table[b]`` (int32 [seqs, max_pages];
    entries past its length are not looked at): each query sees the tokens up to its own.  A query that sees nothing gets zeros and lse = -inf; so do rows
    of no sequence, but those of a given ``out`` or ``lse`` are left as they are.  Types, scale, status and heads as in
    ``prompt_attention``; a page number out of range or a length beyond the table is not followed.  ``prefix_attention`` does the same for a few tokens of each
    sequence, and shares a prefix."""
    cache_values = cache._descriptor()
    dtype, device = cache.dtype, cache.device
    shape, qs = _tensor(q, "q", 3, dtype, device)
    handle = _handle(stream, device)
    T, heads, dim = shape
    if dim != cache.head_dim:
        _refuse(f"heads of {dim} (q) and {cache.head_dim} (cache)")
    n = _sequences(starts)
    starts_at = _index(starts, "starts", (None,), torch.int32, device)
    table_at = _index(page_table, "page_table", (n, None), torch.int32, device)
    max_pages = page_table.shape[1]
    lens_at = _index(lens, "lens", (n,), torch.int32, device)
    scale, st, zero = _scale(scale, dim), _status(status, device), (out is None) + 2 * (lse is None)
    out, os = _output(out, "out", shape, dtype, device, stream)
    if lse is None:
        lse = _empty((T, heads), torch.float32, device, stream)
    lse_at = _index(lse, "lse", (T, heads), torch.float32, device)
    if workspace is None:
        workspace = _workspace(None, _chunk_bytes((n, T, heads), cache_values, max_pages), device, stream)
    else:
        _workspace(workspace, 0, device, stream)
    if T:
        gts._check((_lib or _load()).gts_chunk_attention(_CHUNK.pack(
            n, T, heads, zero, scale, starts_at, *_heads(q, qs), *_heads(out, os), lse_at, *cache_values, table_at, max_pages,
            lens_at, workspace.data_ptr(), workspace.nbytes, st), handle))
    return out, lse


def copy_pages(cache, src, dst, tokens=None, into=None, status=None, stream=None):
    """Copies the pages ``src`` of a cache, keys and values, to its pages ``dst`` (int32, one of each a copy), or to those of the cache
    ``into`` (of the same page size, heads and type, in any order).

    ``tokens`` (int32): how many tokens of each page, from its first (default: all).  A negative page copies nothing.  So a sequence that
    forks shares its full pages and copies the one that is being filled; a cache is compacted by moving pages to free ones.  A page may
    be copied to several others, but one that is written twice, or read and written, in a call holds unspecified values.  A page
    number beyond the cache copies nothing and stores GTS_ERR_INVALID_PARAMS to ``status`` (int32 [1] on the device), where given."""
    into = cache if into is None else into
    if into.dtype != cache.dtype or into.device != cache.device:
        _refuse(f"into: a cache of {cache.dtype} on {cache.device} wanted, got {into.dtype} on {into.device}")
    device = cache.device
    handle = _handle(stream, device)
    src_at = _index(src, "src", (None,), torch.int32, device)
    n = src.shape[0]
    dst_at = _index(dst, "dst", (n,), torch.int32, device)
    tokens_at = 0 if tokens is None else _index(tokens, "tokens", (n,), torch.int32, device)
    gts._check((_lib or _load()).gts_copy_pages(_COPY_PAGES.pack(
        n, src_at, dst_at, tokens_at, *cache._descriptor(), *into._descriptor(), _status(status, device)), handle))
