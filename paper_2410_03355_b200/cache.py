"""Binding of the cache operators of include/lantern.h: rotary positions, the paged 8-bit cache of keys and values, attention to it.

Like binding.py it marshals arguments and does nothing else; there is no CPU path.  Calls in their usual form (outputs and workspace
given, no stream argument, tensors on the current device) go to the library natively, all others through ctypes.
"""
from __future__ import annotations

import contextlib
import ctypes
from typing import Optional, Sequence

import torch

from . import binding
from .binding import BF16, F32, LanternError, _ptr, _stream_ptr, load_library

MAX_AXES = 4
ST_BAD_BLOCK, ST_BAD_LENGTH, ST_BAD_PATH = 128, 256, 512


class _CacheStruct(ctypes.Structure):
    _fields_ = [("k_code", ctypes.c_void_p), ("v_code", ctypes.c_void_p), ("k_scale", ctypes.c_void_p), ("v_scale", ctypes.c_void_p),
                ("pages", ctypes.c_int32), ("heads", ctypes.c_int32), ("page_tokens", ctypes.c_int32), ("head_dim", ctypes.c_int32)]


class _RotationStruct(ctypes.Structure):
    _fields_ = [("inv_freq", ctypes.c_void_p), ("positions", ctypes.c_void_p), ("axes", ctypes.c_int32), ("interleaved", ctypes.c_int32),
                ("section", ctypes.c_int32 * MAX_AXES)]


_Strides = ctypes.c_int64 * 3


def declare(lib):
    """Argument types of the operators' entry points; returns them in the order that the native part of the binding takes them in."""
    vp, i32, f32, sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_float, ctypes.c_size_t
    lib.lantern_rotary.argtypes = [vp, vp, i32, i32, i32, i32, i32, vp, vp, vp, i32, vp]
    lib.lantern_cache_append.argtypes = [vp, vp, i32, i32, i32, vp, vp, vp, vp, i32, vp, vp, vp, vp, vp]
    lib.lantern_cache_attention_workspace_bytes.restype = sz
    lib.lantern_cache_attention_workspace_bytes.argtypes = [i32, i32, i32, i32, vp, i32]
    lib.lantern_cache_attention.argtypes = [vp, vp, i32, i32, i32, i32, vp, vp, vp, i32, vp, vp, vp, vp, f32, vp, vp, sz, vp]
    lib.lantern_cache_keep.argtypes = [vp, vp, i32, vp, vp, vp, i32, i32, vp, vp, vp]
    lib.lantern_cache_read.argtypes = [vp, vp, i32, vp, vp, i32, i32, i32, vp, vp, vp, vp]
    operators = (lib.lantern_rotary, lib.lantern_cache_append, lib.lantern_cache_attention, lib.lantern_cache_keep, lib.lantern_cache_read)
    for f in operators:
        f.restype = i32
    return operators


def _dtype(t: torch.Tensor, name: str) -> int:
    if t.dtype == torch.bfloat16:
        return BF16
    if t.dtype == torch.float32:
        return F32
    raise ValueError(f"{name} must be float32 or bfloat16")


def _rows(t: torch.Tensor, name: str):
    """Pointer and strides of a row tensor [B, R, heads, D]: the last axis is contiguous, the others may have any stride."""
    if t.dim() != 4:
        raise ValueError(f"{name} must be [B, R, heads, D]")
    if not t.is_cuda:
        raise ValueError(f"{name} must be a CUDA tensor (the library has no CPU path)")
    if t.stride(3) != 1 and t.shape[3] > 1 and t.numel():
        raise ValueError(f"{name}: the components of a head must lie side by side")
    return t.data_ptr(), _Strides(t.stride(0), t.stride(1), t.stride(2))


def _index(t: Optional[torch.Tensor], shape, device, name: str):
    """Pointer of an int32 tensor of that shape, or None."""
    if t is None:
        return None
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} must be {list(shape)}, got {list(t.shape)}")
    if t.device != device:
        raise ValueError(f"{name} must be on {device}")
    return _ptr(t, torch.int32, name)


class _Fixed:
    """An object whose tensors are those it was made of: the library is given their addresses, so that none may be put in another's place."""
    __slots__ = ()

    def __setattr__(self, name, value):
        if hasattr(self, "_device"):   # (set last)
            raise AttributeError(f"{type(self).__name__}.{name} is fixed: make another {type(self).__name__}")
        object.__setattr__(self, name, value)


class KVCache(_Fixed):
    """A paged cache of one layer's keys and values in 8 bits: codes k, v [pages, heads, page_tokens, head_dim] float8_e4m3fn, and a
    scale for each page and head, k_scale, v_scale [pages, heads] float32 (see lantern_cache in include/lantern.h)."""
    __slots__ = ("k", "v", "k_scale", "v_scale", "pages", "heads", "page_tokens", "head_dim", "device", "_struct", "_at", "_device")

    def __init__(self, k: torch.Tensor, v: torch.Tensor, k_scale: torch.Tensor, v_scale: torch.Tensor):
        if k.dim() != 4 or k.shape != v.shape:
            raise ValueError("k and v must both be [pages, heads, page_tokens, head_dim]")
        self.pages, self.heads, self.page_tokens, self.head_dim = (int(n) for n in k.shape)
        self.device = k.device
        for name, t, shape, dtype in (("k", k, k.shape, torch.float8_e4m3fn), ("v", v, k.shape, torch.float8_e4m3fn),
                                      ("k_scale", k_scale, k.shape[:2], torch.float32), ("v_scale", v_scale, k.shape[:2], torch.float32)):
            if t.shape != shape:
                raise ValueError(f"{name} must be {list(shape)}, got {list(t.shape)}")
            if t.device != self.device:
                raise ValueError(f"{name} must be on {self.device}")
            _ptr(t, dtype, name)
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        self._struct = _CacheStruct(k.data_ptr(), v.data_ptr(), k_scale.data_ptr(), v_scale.data_ptr(), self.pages, self.heads,
                                    self.page_tokens, self.head_dim)
        self._at = ctypes.addressof(self._struct)
        self._device = k.get_device()

    @classmethod
    def empty(cls, pages: int, heads: int, page_tokens: int, head_dim: int, device="cuda") -> "KVCache":
        """A cache of blocks that hold nothing yet (all codes zero, scales one)."""
        code = [torch.zeros((pages, heads, page_tokens, head_dim), dtype=torch.uint8, device=device).view(torch.float8_e4m3fn) for _ in range(2)]
        return cls(*code, *(torch.ones((pages, heads), dtype=torch.float32, device=device) for _ in range(2)))


class Rotation(_Fixed):
    """Rotary frequencies: inv_freq [P] float32, the number of pairs of each axis, and which components make a pair -- (2j, 2j+1) if
    interleaved, else (j, j+P) (see lantern_rotation in include/lantern.h)."""
    __slots__ = ("inv_freq", "sections", "interleaved", "_struct", "_at", "_device")

    def __init__(self, inv_freq: torch.Tensor, sections: Sequence[int], *, interleaved: bool):
        sections = tuple(int(s) for s in sections)
        if not 1 <= len(sections) <= MAX_AXES or min(sections) < 0:
            raise ValueError(f"sections must be 1 to {MAX_AXES} counts")
        if inv_freq.dim() != 1 or inv_freq.shape[0] != sum(sections):
            raise ValueError("inv_freq must hold one frequency for each pair of the sections")
        _ptr(inv_freq, torch.float32, "inv_freq")
        self.inv_freq, self.sections, self.interleaved = inv_freq, sections, bool(interleaved)
        n = len(sections)
        self._struct = _RotationStruct(inv_freq.data_ptr(), None, n, int(interleaved), (ctypes.c_int32 * MAX_AXES)(*sections, *(0,) * (MAX_AXES - n)))
        self._at = ctypes.addressof(self._struct)
        self._device = inv_freq.get_device()

    def _bind(self, positions: torch.Tensor, B: int, R: int, device) -> _RotationStruct:
        if positions is None:
            raise ValueError("a rotation needs positions")
        if self.inv_freq.device != device:
            raise ValueError(f"inv_freq must be on {device}")
        out = _RotationStruct.from_buffer_copy(self._struct)
        out.positions = _index(positions, (len(self.sections), B, R), device, "positions")
        return out


def _allocating_on(stream: Optional[torch.cuda.Stream]):
    """What a call allocates belongs to the stream that it runs on (memory of another stream's pool may still be in use there)."""
    return contextlib.nullcontext() if stream is None else torch.cuda.stream(stream)


def _check(rc: int, where: str) -> None:
    if rc != 0:
        raise LanternError(rc, where)


class _Rotary(torch.autograd.Function):
    """The rotation within a graph of gradients: its transpose is the rotation back."""

    @staticmethod
    def forward(ctx, x, positions, rotation, inverse):
        if positions is None or rotation is None:
            raise ValueError("a rotation needs positions")
        ctx.save_for_backward(positions, rotation.inv_freq)   # (changes of them until then are noticed)
        ctx.rotation, ctx.inverse = rotation, inverse
        return rotary(x, positions, rotation, inverse=inverse)

    @staticmethod
    def backward(ctx, grad):
        positions, _ = ctx.saved_tensors
        if grad.stride(3) != 1:   # (a sum's gradient is one number expanded)
            grad = grad.contiguous()
        return rotary(grad, positions, ctx.rotation, inverse=not ctx.inverse), None, None, None


def rotary(x: torch.Tensor, positions: torch.Tensor, rotation: Rotation, *, inverse: bool = False, out: Optional[torch.Tensor] = None,
           stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """lantern_rotary: rows x [B, R, H, D] turned by positions [axes, B, R].  inverse=True turns back, which is also the gradient with
    respect to x of a gradient with respect to the result, and what backward() does where x requires a gradient (positions and frequencies
    have none).  out: a tensor like x, or x itself (no gradient goes through it: refused where one is asked for); allocated if not given."""
    inverse = bool(inverse)
    if torch.is_grad_enabled() and (x.requires_grad or out is not None and out.requires_grad):
        if out is not None:
            raise ValueError("out has no gradient: leave it out, or call under torch.no_grad()")
        with _allocating_on(stream):   # (its stream is the gradient's as well)
            return _Rotary.apply(x, positions, rotation, inverse)
    if out is None:
        with _allocating_on(stream):
            out = torch.empty(x.shape, dtype=x.dtype, device=x.device)
    if binding._call is not None and stream is None and rotation is not None:   # (loaded: the native part)
        rc = binding._call.rotary(x, positions, rotation._at, rotation._device, inverse, out)
        if rc is not None:
            if rc != 0:
                raise LanternError(rc, "lantern_rotary")
            return out
    lib = load_library()
    px, xs = _rows(x, "x")
    dtype = _dtype(x, "x")
    if out.shape != x.shape or out.dtype != x.dtype or out.device != x.device:
        raise ValueError("out must be like x")
    po, os_ = _rows(out, "out")
    if px == po and x.stride() != out.stride():
        raise ValueError("out may be x itself, but not another view of it")
    B, R, H, D = x.shape
    with torch.cuda.device(x.device):
        _check(lib.lantern_rotary(px, po, dtype, B, R, H, D, xs, os_, ctypes.byref(rotation._bind(positions, B, R, x.device)),
                                  int(inverse), _stream_ptr(stream)), "lantern_rotary")
    return out


def _table(cache: KVCache, table: torch.Tensor, B: int):
    if table.dim() != 2 or table.shape[0] != B:
        raise ValueError("table must be [B, blocks]")
    if table.device != cache.device:
        raise ValueError(f"table must be on {cache.device}")
    return _ptr(table, torch.int32, "table"), int(table.shape[1])


def cache_append(k: torch.Tensor, v: torch.Tensor, cache: KVCache, table: torch.Tensor, lengths: torch.Tensor, *,
                 counts: Optional[torch.Tensor] = None, positions: Optional[torch.Tensor] = None, rotation: Optional[Rotation] = None,
                 status: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None) -> None:
    """lantern_cache_append: rows k, v [B, R, heads, D] become tokens lengths[b], lengths[b] + 1, ... of their sequences; keys are turned by
    positions [axes, B, R] on the way if a rotation is given.  table [B, blocks], lengths [B], counts [B] (rows that there are; None = R)
    and status [B] (fault bits are OR-ed into it) are int32.  No gradient goes through the cache: rows that require one are taken as they are."""
    if binding._call is not None and stream is None:
        rc = binding._call.append(k, v, cache._at, cache._device, table, lengths, counts, positions, None if rotation is None else rotation._at,
                                  None if rotation is None else rotation._device, status)
        if rc is not None:
            return _check(rc, "lantern_cache_append")
    lib = load_library()
    pk, ks = _rows(k, "k")
    pv, vs = _rows(v, "v")
    dtype = _dtype(k, "k")
    B, R, H, D = k.shape
    if v.shape != k.shape or v.dtype != k.dtype:
        raise ValueError("k and v must have the same shape and type")
    if H != cache.heads or D != cache.head_dim:
        raise ValueError("k and v must have the cache's heads and components")
    dev = cache.device
    if k.device != dev or v.device != dev:
        raise ValueError(f"k and v must be on {dev}")
    if rotation is None and positions is not None:
        raise ValueError("positions without a rotation")
    pt, width = _table(cache, table, B)
    rot = None if rotation is None else ctypes.byref(rotation._bind(positions, B, R, dev))
    with torch.cuda.device(dev):
        _check(lib.lantern_cache_append(pk, pv, dtype, B, R, ks, vs, cache._at, pt, width, _index(lengths, (B,), dev, "lengths"),
                                        _index(counts, (B,), dev, "counts"), rot, _index(status, (B,), dev, "status"),
                                        _stream_ptr(stream)), "lantern_cache_append")


def cache_attention_workspace_bytes(B: int, R: int, q_heads: int, cache: KVCache, blocks: int, *, dtype: torch.dtype = torch.bfloat16) -> int:
    """lantern_cache_attention_workspace_bytes: scratch bytes of one cache_attention() call with a table of `blocks` columns."""
    return int(load_library().lantern_cache_attention_workspace_bytes(BF16 if dtype == torch.bfloat16 else F32, B, R, q_heads, cache._at, blocks))


def cache_attention(q: torch.Tensor, cache: KVCache, table: torch.Tensor, lengths: torch.Tensor, *, counts: Optional[torch.Tensor] = None,
                    starts: Optional[torch.Tensor] = None, tree_parents: Optional[torch.Tensor] = None, scale: Optional[float] = None,
                    out: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None, status: Optional[torch.Tensor] = None,
                    stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """lantern_cache_attention: queries [B, R, q_heads, D] of the rows that cache_append() has just put behind the sequences' `lengths`
    tokens, attending to the tokens from starts[b] (None: 0) on and to their own ancestors (tree_parents [B, R-1] as in verify(); None =
    a chain, i.e. causal).  scale: None = head_dim ** -0.5.  Rows that `counts` leaves out stay as they are in `out`.  The result has no
    gradient, also where q requires one."""
    if binding._call is not None and stream is None and out is not None and workspace is not None:
        rc = binding._call.attention(q, cache._at, cache._device, table, lengths, counts, starts, tree_parents, scale, out, workspace, status)
        if rc is not None:
            if rc != 0:
                raise LanternError(rc, "lantern_cache_attention")
            return out
    lib = load_library()
    pq, qs = _rows(q, "q")
    dtype = _dtype(q, "q")
    B, R, HQ, D = q.shape
    dev = cache.device
    if q.device != dev:
        raise ValueError(f"q must be on {dev}")
    if D != cache.head_dim or HQ % cache.heads:
        raise ValueError("q must have the cache's components and a multiple of its heads")
    if out is None:
        with _allocating_on(stream):
            out = (torch.empty if counts is None else torch.zeros)(q.shape, dtype=q.dtype, device=dev)
    elif out.shape != q.shape or out.device != dev:
        raise ValueError("out must have q's shape")
    pt, width = _table(cache, table, B)
    with torch.cuda.device(dev):
        if workspace is None:
            need = int(lib.lantern_cache_attention_workspace_bytes(dtype, B, R, HQ, cache._at, width))
            if need:
                with _allocating_on(stream):
                    workspace = torch.empty(need, dtype=torch.uint8, device=dev)
        elif workspace.device != dev:
            raise ValueError(f"workspace must be on {dev}")
        _check(lib.lantern_cache_attention(
            pq, _ptr(out, q.dtype, "out"), dtype, B, R, HQ, qs, cache._at, pt, width, _index(lengths, (B,), dev, "lengths"),
            _index(counts, (B,), dev, "counts"), _index(starts, (B,), dev, "starts"),
            _index(tree_parents, (B, max(R - 1, 0)), dev, "tree_parents"), D ** -0.5 if scale is None else float(scale),
            _index(status, (B,), dev, "status"), _ptr(workspace, torch.uint8, "workspace"),
            workspace.numel() if workspace is not None else 0, _stream_ptr(stream)), "lantern_cache_attention")
    return out


def cache_keep(cache: KVCache, table: torch.Tensor, lengths: torch.Tensor, accept_len: torch.Tensor, accept_path: torch.Tensor, *,
               out_lengths: Optional[torch.Tensor] = None, status: Optional[torch.Tensor] = None,
               stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """lantern_cache_keep: after verify(), moves the accepted path's tokens behind the root's and returns the sequences' new lengths (the
    root's and the path's tokens counted).  accept_len [B], accept_path [B, N] as verify() gives them."""
    if out_lengths is None:
        with _allocating_on(stream):
            out_lengths = torch.empty_like(lengths)
    if binding._call is not None and stream is None:
        rc = binding._call.keep(cache._at, cache._device, table, lengths, accept_len, accept_path, out_lengths, status)
        if rc is not None:
            if rc != 0:
                raise LanternError(rc, "lantern_cache_keep")
            return out_lengths
    lib = load_library()
    if accept_path.dim() != 2:
        raise ValueError("accept_path must be [B, N]")
    B, N = accept_path.shape
    dev = cache.device
    pt, width = _table(cache, table, B)
    pl = _index(lengths, (B,), dev, "lengths")
    with torch.cuda.device(dev):
        _check(lib.lantern_cache_keep(cache._at, pt, width, pl, _index(accept_len, (B,), dev, "accept_len"),
                                      _index(accept_path, (B, N), dev, "accept_path"), B, N, _index(out_lengths, (B,), dev, "out_lengths"),
                                      _index(status, (B,), dev, "status"), _stream_ptr(stream)), "lantern_cache_keep")
    return out_lengths


def cache_read(cache: KVCache, table: torch.Tensor, first: torch.Tensor, rows: int, *, counts: Optional[torch.Tensor] = None,
               dtype: torch.dtype = torch.bfloat16, out=None, status: Optional[torch.Tensor] = None,
               stream: Optional[torch.cuda.Stream] = None):
    """lantern_cache_read: the keys and values [B, rows, heads, D] of tokens first[b], first[b] + 1, ... in bf16 or fp32 (out: a pair of
    such tensors).  Rows that `counts` leaves out stay as they are in `out`."""
    if binding._call is not None and stream is None and out is not None:
        rc = binding._call.read(cache._at, cache._device, table, first, rows, counts, *out, status)
        if rc is not None:
            if rc != 0:
                raise LanternError(rc, "lantern_cache_read")
            return out
    lib = load_library()
    B, rows = int(table.shape[0]), int(rows)
    dev = cache.device
    shape = (B, rows, cache.heads, cache.head_dim)
    if out is None:
        with _allocating_on(stream):
            out = tuple((torch.empty if counts is None else torch.zeros)(shape, dtype=dtype, device=dev) for _ in range(2))
    k, v = out
    if tuple(k.shape) != shape or tuple(v.shape) != shape or k.dtype != v.dtype or k.device != dev or v.device != dev:
        raise ValueError(f"out must be two tensors {list(shape)} on {dev}")
    pt, width = _table(cache, table, B)
    with torch.cuda.device(dev):
        _check(lib.lantern_cache_read(cache._at, pt, width, _index(first, (B,), dev, "first"), _index(counts, (B,), dev, "counts"), B, rows,
                                      _dtype(k, "out"), _ptr(k, None, "out"), _ptr(v, None, "out"), _index(status, (B,), dev, "status"),
                                      _stream_ptr(stream)), "lantern_cache_read")
    return k, v
