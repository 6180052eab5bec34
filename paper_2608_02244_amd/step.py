"""The operators of a serving step: KV placement, norm and rotation of queries and
keys with the store into the cache, and attention over the paged cache.

Binding of ``fsched_kv_layout``, ``fsched_qk_norm_rope``, ``fsched_attend`` and
``fsched_attend_shared`` (``include/fsched.h`` says what each computes).  Every
array is a torch tensor on the GPU, the calls are enqueued on the current torch
stream (or ``stream``) and nothing is synchronised.

A cache is a pair of tensors [n_pages, kv_heads, page_size, head_dim]; a permuted
view (another order of page, head and slot in memory) does as well, as long as the
head dimension is contiguous.
"""
from __future__ import annotations

import ctypes
import functools
import struct

import torch

import paper_2608_02244_amd as _fs

_I32, _I64, _F32, _U32, _P = (ctypes.c_int32, ctypes.c_int64, ctypes.c_float, ctypes.c_uint32,
                              ctypes.c_void_p)
_DTYPES = {torch.bfloat16: 0, torch.float16: 1}
_INT32, _FLOAT32 = torch.int32, torch.float32


class KvCache(ctypes.Structure):
    _fields_ = [("k", _P), ("v", _P), ("k_stride", _I64 * 3), ("v_stride", _I64 * 3),
                ("n_pages", _I32), ("page_size", _I32), ("kv_heads", _I32), ("head_dim", _I32),
                ("dtype", _I32), ("reserved", _I32)]


class LayoutParams(ctypes.Structure):
    _fields_ = [(n, _I32) for n in ("n_req", "n_tok", "page_size", "table_width", "n_free",
                                    "first_pos")] + [("flags", _U32), ("reserved", _I32)]


class RopeParams(ctypes.Structure):
    _fields_ = [(n, _I32) for n in ("n_tok", "q_heads", "rot_dim", "n_pos", "interleaved")] + \
        [("eps", _F32), ("flags", _U32), ("reserved", _I32), ("qkv_stride", _I64),
         ("q_token_stride", _I64), ("q_head_stride", _I64)]


class AttnParams(ctypes.Structure):
    _fields_ = [(n, _I32) for n in ("n_req", "n_tok", "q_heads", "max_q", "table_width", "window",
                                    "n_sink", "prefix_len")] + \
        [("scale", _F32), ("flags", _U32), ("q_token_stride", _I64), ("q_head_stride", _I64),
         ("out_token_stride", _I64), ("out_head_stride", _I64)]


# The calls pack their parameter blocks directly: a ctypes structure built field by
# field costs more than the rest of a call.
_pack_cache = struct.Struct("=2Q6q6i").pack
_pack_layout = struct.Struct("=6iIi").pack
_pack_rope = struct.Struct("=5ifIi3q").pack
_pack_attn = struct.Struct("=8ifI4q").pack


def _stream(stream, device):
    return stream.cuda_stream if stream is not None else \
        torch._C._cuda_getCurrentRawStream(device.index)


def _call(name, *args):
    rc = getattr(_fs.lib(), name)(*args)
    if rc:
        raise _fs.FschedError(rc, name)


def _ints(name, x, shape):
    """Address of a contiguous int32 GPU tensor of the given shape."""
    if x.dtype is not _INT32 or not x.is_cuda or x.shape != shape or not x.is_contiguous():
        raise ValueError(f"{name} must be a contiguous int32 GPU tensor of shape {tuple(shape)}")
    return x.data_ptr()


def _rows(name, x, dim, dtype):
    """Strides of a ``dim``-dimensional GPU tensor whose last dimension is contiguous."""
    st = x.stride()
    if x.dim() != dim or x.dtype is not dtype or not x.is_cuda or \
            (st[-1] != 1 and x.shape[-1] > 1):
        raise ValueError(f"{name} must be a {dim}-dimensional {dtype} GPU tensor whose last "
                         "dimension is contiguous")
    return st


def _cache(k_cache, v_cache):
    """(parameter block, shape, element type) of a cache."""
    dtype = k_cache.dtype
    code = _DTYPES.get(dtype)
    if code is None:
        raise ValueError("the cache must be bfloat16 or float16")
    ks, vs = _rows("k_cache", k_cache, 4, dtype), _rows("v_cache", v_cache, 4, dtype)
    shape = k_cache.shape
    if shape != v_cache.shape:
        raise ValueError("k_cache and v_cache differ in shape")
    return _pack_cache(k_cache.data_ptr(), v_cache.data_ptr(), ks[0], ks[1], ks[2], vs[0], vs[1],
                       vs[2], shape[0], shape[2], shape[1], shape[3], code, 0), shape, dtype


def kv_layout(old_len, new_len, block_table, free_pages, *, page_size: int, n_tok: int,
              first_pos: int = 0, stream=None):
    """fsched_kv_layout: places for the step's new tokens.

    ``block_table`` [n_req, width] is updated in place.  Returns (slots [n_tok],
    positions [n_tok], q_start [n_req + 1], kv_len [n_req], used [2]), int32."""
    n = old_len.shape[0]
    table = block_table.shape
    if len(table) != 2 or table[0] != n:
        raise ValueError(f"block_table must be a contiguous int32 GPU tensor of shape ({n}, any)")
    args = (_ints("old_len", old_len, (n,)), _ints("new_len", new_len, (n,)),
            _ints("free_pages", free_pages, (free_pages.shape[0],)),
            _ints("block_table", block_table, table))
    # one allocation holds all results, each on a multiple of 16 bytes
    t, q, k = (max(0, n_tok) + 3) & ~3, (n + 4) & ~3, (n + 3) & ~3
    room = old_len.new_empty(2 * t + q + k + 4)
    m = max(0, n_tok)
    slots, _, positions, _, q_start, _, kv_len, _, used, _ = room.split_with_sizes(
        (m, t - m, m, t - m, n + 1, q - n - 1, n, k - n, 2, 2))
    at = room.data_ptr()
    _call("fsched_kv_layout",
          _pack_layout(n, n_tok, page_size, table[1], free_pages.shape[0], first_pos,
                       _fs.F_DEVICE_PTRS, 0),
          *args, at, at + 4 * t, at + 8 * t, at + 8 * t + 4 * q, at + 8 * t + 4 * (q + k),
          _stream(stream, room.device))
    return slots, positions, q_start, kv_len, used


def qk_norm_rope(qkv, positions, slots, cos_sin, k_cache, v_cache, q_weight=None, k_weight=None,
                 *, eps: float = 1e-6, interleaved: bool = False, out=None, stream=None):
    """fsched_qk_norm_rope: ``qkv`` [n_tok, q_heads + 2 kv_heads, head_dim] to the
    rotated queries [n_tok, q_heads, head_dim] (``out``, made if None), keys and
    values put into the caches at ``slots`` (None: nowhere).  ``cos_sin`` [n_pos,
    rot_dim] f32 (None: no rotation, ``positions`` may be None)."""
    cache, shape, dt = _cache(k_cache, v_cache)
    dim = shape[3]
    st = _rows("qkv", qkv, 3, dt)
    n, heads, qkv_dim = qkv.shape
    q_heads = heads - 2 * shape[1]
    if q_heads < 1 or qkv_dim != dim or st[1] != dim:
        raise ValueError("qkv must be [n_tok, q_heads + 2 kv_heads, head_dim] with heads "
                         "head_dim apart")
    rot = n_pos = 0
    if cos_sin is not None:
        if cos_sin.dtype is not _FLOAT32 or not cos_sin.is_cuda or cos_sin.dim() != 2 or \
                not cos_sin.is_contiguous():
            raise ValueError("cos_sin must be a contiguous float32 GPU tensor [n_pos, rot_dim]")
        n_pos, rot = cos_sin.shape
        if positions is None:
            raise ValueError("a rotation needs positions")
    for name, w in (("q_weight", q_weight), ("k_weight", k_weight)):
        if w is not None:
            _rows(name, w, 1, dt)
            if w.shape[0] != dim:
                raise ValueError(f"{name} must have head_dim elements")
    if out is None:
        out = qkv.new_empty((n, q_heads, dim))
    os = _rows("out", out, 3, dt)
    if out.shape != (n, q_heads, dim):
        raise ValueError(f"out must have shape {(n, q_heads, dim)}")
    _call("fsched_qk_norm_rope",
          _pack_rope(n, q_heads, rot, n_pos, bool(interleaved), eps, _fs.F_DEVICE_PTRS, 0, st[0],
                     os[0], os[1]),
          cache, qkv.data_ptr(),
          None if positions is None else _ints("positions", positions, (n,)),
          None if slots is None else _ints("slots", slots, (n,)),
          None if cos_sin is None else cos_sin.data_ptr(),
          None if q_weight is None else q_weight.data_ptr(),
          None if k_weight is None else k_weight.data_ptr(), out.data_ptr(),
          _stream(stream, out.device))
    return out


@functools.lru_cache(maxsize=4096)
def _workspace_bytes(device, n_tok, n_req, q_heads, kv_heads, head_dim, page_size, table_width,
                     max_q, prefix_len, window, n_sink):
    """What fsched_attend_workspace answers for a shape on the current device."""
    c = KvCache(n_pages=0, page_size=page_size, kv_heads=kv_heads, head_dim=head_dim)
    p = AttnParams(n_req=n_req, n_tok=n_tok, q_heads=q_heads, max_q=max_q,
                   table_width=table_width, window=window, n_sink=n_sink, prefix_len=prefix_len,
                   scale=1.0, flags=_fs.F_DEVICE_PTRS)
    size = _I64(0)
    _call("fsched_attend_workspace", ctypes.byref(p), ctypes.byref(c), ctypes.byref(size))
    return size.value


def _attend(name, q, k_cache, v_cache, prefix_pages, prefix_len, block_table, q_start, kv_len,
            scale, window, n_sink, max_q, out, return_lse, workspace, stream):
    cache, shape, dt = _cache(k_cache, v_cache)
    n_pages, kv_heads, page, dim = shape
    qs = _rows("q", q, 3, dt)
    n_tok, q_heads, q_dim = q.shape
    if q_dim != dim:
        raise ValueError("q and the cache differ in head_dim")
    n = kv_len.shape[0]
    table = block_table.shape
    if len(table) != 2 or table[0] != n:
        raise ValueError(f"block_table must be a contiguous int32 GPU tensor of shape ({n}, any)")
    ints = (_ints("block_table", block_table, table), _ints("q_start", q_start, (n + 1,)),
            _ints("kv_len", kv_len, (n,)))
    if prefix_pages is not None:
        count = prefix_pages.shape[0]
        ints = (_ints("prefix_pages", prefix_pages, (count,)),) + ints
        if count * page < prefix_len:
            raise ValueError("prefix_pages must list every page of the prefix")
    device = q.device
    if out is None:
        out = q.new_empty(q.shape)
    os = _rows("out", out, 3, dt)
    if out.shape != q.shape:
        raise ValueError("out and q differ in shape")
    lse = torch.empty((n_tok, q_heads), dtype=_FLOAT32, device=device) if return_lse else None
    if max_q is None:
        max_q = max(1, n_tok)
    if workspace is None:  # torch's allocator orders its reuse by stream as the call needs it
        need = _workspace_bytes(device.index, n_tok, n, q_heads, kv_heads, dim, page, table[1],
                                max_q, prefix_len, window, n_sink)
        if stream is None and need:
            workspace = torch.empty(need, dtype=torch.uint8, device=device)
    elif not (workspace.is_cuda and workspace.is_contiguous()):
        raise ValueError("workspace must be a contiguous GPU tensor")
    _call(name,
          _pack_attn(n, n_tok, q_heads, max_q, table[1], window, n_sink, prefix_len,
                     dim ** -0.5 if scale is None else scale, _fs.F_DEVICE_PTRS, qs[0], qs[1],
                     os[0], os[1]),
          cache, q.data_ptr(), *ints, out.data_ptr(), None if lse is None else lse.data_ptr(),
          None if workspace is None else workspace.data_ptr(),
          0 if workspace is None else workspace.nbytes, _stream(stream, device))
    return (out, lse) if return_lse else out


def attend(q, k_cache, v_cache, block_table, q_start, kv_len, *, scale=None, window: int = 0,
           n_sink: int = 0, max_q=None, out=None, return_lse: bool = False, workspace=None,
           stream=None):
    """fsched_attend: attention of ``q`` [n_tok, q_heads, head_dim], the requests'
    new tokens one after the other (``q_start`` [n_req + 1]), over the tokens that
    each request holds (``kv_len``, ``block_table`` [n_req, width]).

    ``window`` 0: every earlier token is seen; else the last ``window`` and the first
    ``n_sink``.  ``max_q``: no request has more new tokens (1 for a decode step; None:
    not known).  ``scale`` None: head_dim ** -0.5.  ``workspace``: a GPU tensor of
    ``attend_workspace`` bytes, for calls that may not allocate.  None: taken from
    torch's allocator (with ``stream`` given: from the library's pool).
    Returns out, or (out, lse [n_tok, q_heads] float32) with ``return_lse``."""
    return _attend("fsched_attend", q, k_cache, v_cache, None, 0, block_table, q_start, kv_len,
                   scale, window, n_sink, max_q, out, return_lse, workspace, stream)


def attend_shared(q, k_cache, v_cache, prefix_pages, prefix_len: int, block_table, q_start,
                  kv_len, *, scale=None, window: int = 0, n_sink: int = 0, max_q=None, out=None,
                  return_lse: bool = False, workspace=None, stream=None):
    """fsched_attend_shared: ``attend`` for requests that all begin with the
    ``prefix_len`` tokens held in ``prefix_pages``; ``block_table`` and ``kv_len``
    describe each request's own tokens behind them."""
    return _attend("fsched_attend_shared", q, k_cache, v_cache, prefix_pages, prefix_len,
                   block_table, q_start, kv_len, scale, window, n_sink, max_q, out, return_lse,
                   workspace, stream)


def attend_workspace(n_tok: int, n_req: int, q_heads: int, kv_heads: int, head_dim: int, *,
                     page_size: int, table_width: int, max_q=None, prefix_len: int = 0,
                     window: int = 0, n_sink: int = 0):
    """A workspace (uint8 GPU tensor) for ``attend`` / ``attend_shared`` calls of this
    shape, 256-byte aligned; calls that may overlap in time need one each."""
    device = torch.device("cuda", torch.cuda.current_device())
    size = _workspace_bytes(device.index, n_tok, n_req, q_heads, kv_heads, head_dim, page_size,
                            table_width, max(1, n_tok) if max_q is None else max_q, prefix_len,
                            window, n_sink)
    return torch.empty(max(256, size), dtype=torch.uint8, device=device)
