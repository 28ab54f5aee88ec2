"""The operators of a decode step, on the GPU: rotary positions (and their gradient), appending keys and values to a
paged cache, and attention of a batch over a shared prefix and each sequence's own tokens.

They are the kernels whose tile graphs the simulator takes, run on the machine itself.  Functions named like the C ABI
in include/gts_serving.h marshal its descriptors; the ones below them take torch tensors:

    rotary = Rotary(128, base=10000.0, layout="half")          # frequencies, once
    cache = PagedCache.empty(n_pages, page_size, kv_heads, 128, torch.bfloat16)
    q = append_kv(q, k, v, positions, slots, rotary, cache)    # one step's new tokens
    out, lse = prefix_attention(q, cache, prefix_pages, prefix_len, page_table, lens)

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

EXPORTS = ("gts_rope", "gts_append_kv", "gts_prefix_attention", "gts_attention_workspace_bytes")

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


# The same layouts as format strings: the torch entry points pack a descriptor in one go, which takes a fifth of the time of
# filling the structures above (about 2 against 10 us a call).
_HEADS_FORMAT, _ROTARY_FORMAT, _CACHE_FORMAT = "Pqq", "PIifI", "PPqqqqqqIIIIi4x"
_ROPE = struct.Struct("@IIIIiP" + _ROTARY_FORMAT + 4 * _HEADS_FORMAT)
_APPEND = struct.Struct("@IIPP" + _ROTARY_FORMAT + 4 * _HEADS_FORMAT + _CACHE_FORMAT + "P")
_ATTENTION = struct.Struct("@IIIf" + 2 * "Pqqq" + "P" + _CACHE_FORMAT + "PI4xPI4xPPNP")

_lib = None


def _load():
    global _lib
    if _lib is None:
        lib = gts.load()
        for name in EXPORTS[:3]:
            f = getattr(lib, name)
            f.argtypes, f.restype = [_vp, _vp], _i32
        lib.gts_attention_workspace_bytes.argtypes, lib.gts_attention_workspace_bytes.restype = [_vp], _sz
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
