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

import numpy as np
import torch

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


def _tensor(t, name, dims, dtype=None, like=None):
    if t.dim() != dims:
        _refuse(f"{name}: {dims} dimensions wanted, got {t.dim()}")
    if not t.is_cuda:
        _refuse(f"{name} is not on a CUDA device")
    if like is not None and (t.dtype != like.dtype or t.device != like.device):
        _refuse(f"{name}: {like.dtype} on {like.device} wanted, got {t.dtype} on {t.device}")
    if dtype is not None and t.dtype != dtype:
        _refuse(f"{name}: {dtype} wanted, got {t.dtype}")
    if t.stride(-1) != 1 and t.shape[-1] > 1:
        _refuse(f"{name}: the innermost dimension must be contiguous")
    return t


def _index(t, name, shape, dtype, device):
    """A contiguous index tensor of the given shape (None: any extent)."""
    if t.dtype != dtype or t.device != device:
        _refuse(f"{name}: {dtype} on {device} wanted, got {t.dtype} on {t.device}")
    if t.dim() != len(shape) or any(w is not None and w != n for w, n in zip(shape, t.shape)) or not t.is_contiguous():
        _refuse(f"{name}: contiguous {list(shape)} wanted, got {list(t.shape)}")
    return t


def _status(t, device):
    if t is None:
        return None
    return _index(t, "status", (1,), torch.int32, device).data_ptr()


def _on(stream):
    """(context in which outputs are allocated, stream handle)"""
    if stream is None:
        return gts._null(), torch.cuda.current_stream().cuda_stream
    return torch.cuda.stream(stream), stream.cuda_stream


def _check_device(t):
    if t.device.index != torch.cuda.current_device():
        _refuse(f"tensors are on {t.device}, the current device is cuda:{torch.cuda.current_device()}")


def _heads(t):
    if t is None:
        return HeadsDesc()
    s = t.stride()
    return HeadsDesc(t.data_ptr(), s[0], s[1])


class Rotary:
    """The rotation of a model's heads: the frequencies of its pairs, held on the device in turns a position.

    Pair i of ``rot_dim / 2`` turns by ``base ** (-2 i / rot_dim)`` radians a position.  ``layout``: "half" pairs the
    values i and i + rot_dim / 2, "interleaved" 2 i and 2 i + 1; values after ``rot_dim`` (default: the whole head) are
    left as they are.  ``scaling`` stretches positions for contexts longer than those of training:

    * ``{"kind": "linear", "factor": s}``: every frequency divided by s;
    * ``{"kind": "ntk", "factor": s}``: the base times ``s ** (rot_dim / (rot_dim - 2))``, which divides the lowest
      frequency by s and keeps the highest;
    * ``{"kind": "by_parts", "factor": s, "original_len": L, "low": a, "high": b}``: frequencies of fewer than a
      turns in L positions divided by s, those of more than b kept, a linear blend between; rotated values times
      ``magnitude`` (default ``0.1 ln s + 1``).
    """

    def __init__(self, head_dim, rot_dim=None, base=10000.0, layout="half", scaling=None, device="cuda"):
        rot_dim = head_dim if rot_dim is None else rot_dim
        if rot_dim % 2 or not 0 <= rot_dim <= head_dim:
            _refuse(f"rot_dim must be even and at most head_dim, got {rot_dim} of {head_dim}")
        if layout not in _LAYOUTS:
            _refuse(f"unknown rotary layout {layout!r}")
        if not base > 0:
            _refuse("base must be positive")
        self.head_dim, self.rot_dim, self.layout = head_dim, rot_dim, layout
        self.theta, self.factor = self._frequencies(rot_dim, base, scaling)
        units = [round(float(t) / (2 * math.pi) * 2.0 ** 64) % 2 ** 64 for t in self.theta]
        self.units = torch.from_numpy(np.array(units, np.uint64).view(np.int64)).to(device)
        self._descs = [RotaryDesc(self.units.data_ptr() if units else None, rot_dim, _LAYOUTS[layout], self.factor, t)
                       for t in (0, 1)]

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


class PagedCache:
    """Keys and values in pages: two [pages, page_size, kv_heads, head_dim] tensors of any outer strides."""

    def __init__(self, k, v):
        _tensor(k, "k cache", 4)
        _tensor(v, "v cache", 4, like=k)
        if k.shape != v.shape:
            _refuse(f"k and v caches differ: {list(k.shape)}, {list(v.shape)}")
        if k.dtype not in _DTYPES:
            _refuse(f"cache: bfloat16, float16 or float32 wanted, got {k.dtype}")
        self.k, self.v = k, v
        self.n_pages, self.page_size, self.kv_heads, self.head_dim = k.shape
        if self.page_size < 1:
            _refuse("page_size must be positive")
        self.desc = CacheDesc(k.data_ptr(), v.data_ptr(), *k.stride()[:3], *v.stride()[:3], *k.shape, _DTYPES[k.dtype])

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
    _tensor(q, "q", 3)
    _check_device(q)
    dt = _DTYPES.get(q.dtype)
    if dt is None:
        _refuse(f"q: bfloat16, float16 or float32 wanted, got {q.dtype}")
    T, heads, dim = q.shape
    if dim != rotary.head_dim:
        _refuse(f"q has heads of {dim}, the rotary of {rotary.head_dim}")
    _index(positions, "positions", (T,), torch.int32, q.device)
    if k is not None:
        _tensor(k, "k", 3, like=q)
        if k.shape[0] != T or k.shape[2] != dim:
            _refuse(f"k: [{T}, kv_heads, {dim}] wanted, got {list(k.shape)}")
    ctx, handle = _on(stream)
    with ctx:
        out_q = torch.empty((T, heads, dim), dtype=q.dtype, device=q.device) if out_q is None else \
            _same_shape(out_q, q, "out_q")
        if k is not None:
            out_k = torch.empty(k.shape, dtype=q.dtype, device=q.device) if out_k is None else \
                _same_shape(out_k, k, "out_k")
    kh = 0 if k is None else k.shape[1]
    if T and (heads or kh):
        gts_rope(RopeDesc(T, heads, kh, dim, dt, positions.data_ptr(), rotary._descs[transposed], _heads(q),
                          _heads(k if kh else None), _heads(out_q), _heads(out_k if kh else None)), handle)
    return out_q, out_k if k is not None else None


def _same_shape(out, t, name):
    _tensor(out, name, t.dim(), like=t)
    if out.shape != t.shape:
        _refuse(f"{name}: {list(t.shape)} wanted, got {list(out.shape)}")
    return out


class _Rope(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, positions, rotary):
        ctx.save_for_backward(positions)
        ctx.rotary = rotary
        return _rope_call(q, k, positions, rotary, 0, None, None, None)

    @staticmethod
    def backward(ctx, dq, dk):
        dq, dk = rope_grad(_inner(dq), _inner(dk), ctx.saved_tensors[0], ctx.rotary)
        return dq, dk, None, None


def _inner(t):
    return t if t is None or t.stride(-1) == 1 else t.contiguous()


def rope(q, k, positions, rotary, out_q=None, out_k=None, stream=None):
    """q [tokens, heads, head_dim] and k [tokens, kv_heads, head_dim] (or None) rotated to ``positions`` [tokens] int32:
    (q', k').  ``out_q`` / ``out_k`` may be q and k themselves.  With outputs and stream left to the call, gradients
    flow through it."""
    if torch.is_grad_enabled() and (q.requires_grad or (k is not None and k.requires_grad)):
        if out_q is not None or out_k is not None or stream is not None:
            _refuse("rope: gradients need the call's own outputs and the current stream")
        return _Rope.apply(q, k, positions, rotary)
    return _rope_call(q, k, positions, rotary, 0, out_q, out_k, stream)


def rope_grad(dq, dk, positions, rotary, out_dq=None, out_dk=None, stream=None):
    """The gradients of q and k from those of ``rope``'s results: the transposed rotation."""
    return _rope_call(dq, dk, positions, rotary, 1, out_dq, out_dk, stream)


def append_kv(q, k, v, positions, slots, rotary, cache, out_q=None, status=None, stream=None):
    """Rotates q and k of every token to its position, writes k and v to the cache, returns the rotated q.

    q [tokens, heads, head_dim], k and v [tokens, kv_heads, head_dim], positions [tokens] int32; slots [tokens] int64,
    page * page_size + index within the page, no two alike; a negative one is a padding row, of which nothing is
    written to the cache.  A slot beyond the cache writes nothing and stores GTS_ERR_INVALID_PARAMS to ``status``
    (int32 [1] on the device), where given."""
    _tensor(q, "q", 3, like=cache.k)
    _check_device(q)
    T, heads, dim = q.shape
    if dim != cache.head_dim or dim != rotary.head_dim:
        _refuse(f"heads of {dim} (q), {cache.head_dim} (cache) and {rotary.head_dim} (rotary)")
    for t, name in ((k, "k"), (v, "v")):
        _tensor(t, name, 3, like=q)
        if t.shape != (T, cache.kv_heads, dim):
            _refuse(f"{name}: {[T, cache.kv_heads, dim]} wanted, got {list(t.shape)}")
    _index(positions, "positions", (T,), torch.int32, q.device)
    _index(slots, "slots", (T,), torch.int64, q.device)
    ctx, handle = _on(stream)
    with ctx:
        out_q = torch.empty((T, heads, dim), dtype=q.dtype, device=q.device) if out_q is None else \
            _same_shape(out_q, q, "out_q")
    st = _status(status, q.device)
    if T:
        gts_append_kv(AppendDesc(T, heads, positions.data_ptr(), slots.data_ptr(), rotary._descs[0], _heads(q),
                                 _heads(k), _heads(v), _heads(out_q), cache.desc, st), handle)
    return out_q


def _attention_shape(q, cache, prefix_len, max_pages, scale=1.0):
    B, new, heads, _ = q.shape
    d = AttentionDesc(B, new, heads, scale)
    d.cache, d.prefix_len, d.max_pages = cache.desc, prefix_len, max_pages
    return d


def attention_workspace(cache, q, prefix_len, page_table, stream=None):
    """A workspace for ``prefix_attention`` calls of this shape (and of this prefix or a shorter one); calls that may
    run at the same time need one each."""
    need = gts_attention_workspace_bytes(_attention_shape(q, cache, prefix_len, page_table.shape[1]))
    with _on(stream)[0]:
        return torch.empty(max(need, 16), dtype=torch.uint8, device=q.device)


def prefix_attention(q, cache, prefix_pages, prefix_len, page_table, lens, scale=None, out=None, lse=None,
                     workspace=None, status=None, stream=None):
    """Attention of q [seqs, new, heads, head_dim] over a shared prefix and each sequence's own tokens: (out, lse).

    The prefix is the first ``prefix_len`` tokens of the pages in ``prefix_pages`` (int32); sequence b's own tokens are
    the first ``lens[b]`` (int32) of the pages in ``page_table[b]`` (int32 [seqs, max_pages]; entries past its length
    are not looked at).  They include the ``new`` newest, whose keys are in the cache already: query i sees the whole
    prefix and its sequence's tokens up to its own.  ``scale``: of the products (default 1 / sqrt(head_dim)).  A query
    that sees nothing gets zeros and lse = -inf (float32 [seqs, new, heads]).  A page number or a length out of range
    is not followed and stores GTS_ERR_INVALID_PARAMS to ``status`` (int32 [1] on the device), where given."""
    _tensor(q, "q", 4, like=cache.k)
    _check_device(q)
    B, new, heads, dim = q.shape
    if dim != cache.head_dim:
        _refuse(f"heads of {dim} (q) and {cache.head_dim} (cache)")
    if not 0 <= prefix_len <= 1 << 30:
        _refuse(f"prefix_len out of range: {prefix_len}")
    dev = q.device
    _index(prefix_pages, "prefix_pages", (None,), torch.int32, dev)
    if prefix_pages.shape[0] * cache.page_size < prefix_len:
        _refuse(f"{prefix_pages.shape[0]} prefix pages of {cache.page_size} hold no {prefix_len} tokens")
    _index(page_table, "page_table", (B, None), torch.int32, dev)
    _index(lens, "lens", (B,), torch.int32, dev)
    d = _attention_shape(q, cache, prefix_len, page_table.shape[1], 1.0 / math.sqrt(dim) if scale is None else scale)
    ctx, handle = _on(stream)
    with ctx:
        out = torch.empty((B, new, heads, dim), dtype=q.dtype, device=dev) if out is None else _same_shape(out, q, "out")
        if lse is None:
            lse = torch.empty((B, new, heads), dtype=torch.float32, device=dev)
        else:
            _index(lse, "lse", (B, new, heads), torch.float32, dev)
        if workspace is None:
            workspace = torch.empty(max(gts_attention_workspace_bytes(d), 16), dtype=torch.uint8, device=dev)
    s, o = q.stride(), out.stride()
    d.q, d.q_seq_stride, d.q_token_stride, d.q_head_stride = q.data_ptr(), s[0], s[1], s[2]
    d.out, d.out_seq_stride, d.out_token_stride, d.out_head_stride = out.data_ptr(), o[0], o[1], o[2]
    d.lse, d.prefix_pages, d.page_table, d.lens = (lse.data_ptr(), prefix_pages.data_ptr(), page_table.data_ptr(),
                                                   lens.data_ptr())
    d.workspace, d.workspace_bytes = workspace.data_ptr(), workspace.numel() * workspace.element_size()
    d.d_status = _status(status, dev)
    if B and new:
        gts_prefix_attention(d, handle)
    return out, lse
