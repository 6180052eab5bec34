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

import paper_2608_02244_amd as _fs

_I32, _I64, _F32, _U32, _P = (ctypes.c_int32, ctypes.c_int64, ctypes.c_float, ctypes.c_uint32,
                              ctypes.c_void_p)
_DTYPES = {"torch.bfloat16": 0, "torch.float16": 1}  # torch itself is loaded by the calls


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


def _stream(stream):
    import torch
    return (stream if stream is not None else torch.cuda.current_stream()).cuda_stream


def _call(name, *args):
    rc = getattr(_fs.lib(), name)(*args)
    if rc:
        raise _fs.FschedError(rc, name)


def _ints(name, x, shape):
    """Address of a contiguous int32 tensor of the given shape (None: any extent)."""
    import torch
    if x.dtype != torch.int32 or not x.is_cuda or not x.is_contiguous() \
            or x.dim() != len(shape) or any(s is not None and s != n
                                            for s, n in zip(shape, x.shape)):
        raise ValueError(f"{name} must be a contiguous int32 GPU tensor of shape "
                         f"{tuple('any' if s is None else s for s in shape)}")
    return x.data_ptr()


def _last_contiguous(name, x, dim, dtype):
    """A ``dim``-dimensional GPU tensor of the cache's type, last dimension contiguous."""
    if x.dim() != dim or x.dtype != dtype or not x.is_cuda or \
            (x.shape[-1] > 1 and x.stride(-1) != 1):
        raise ValueError(f"{name} must be a {dim}-dimensional {dtype} GPU tensor whose last "
                         "dimension is contiguous")


def _cache(k_cache, v_cache):
    dt = _DTYPES.get(str(k_cache.dtype))
    if dt is None:
        raise ValueError("the cache must be bfloat16 or float16")
    _last_contiguous("k_cache", k_cache, 4, k_cache.dtype)
    _last_contiguous("v_cache", v_cache, 4, k_cache.dtype)
    if k_cache.shape != v_cache.shape:
        raise ValueError("k_cache and v_cache differ in shape")
    n_pages, heads, page, dim = k_cache.shape
    return KvCache(k=k_cache.data_ptr(), v=v_cache.data_ptr(),
                   k_stride=(_I64 * 3)(*k_cache.stride()[:3]),
                   v_stride=(_I64 * 3)(*v_cache.stride()[:3]), n_pages=n_pages, page_size=page,
                   kv_heads=heads, head_dim=dim, dtype=dt)


def kv_layout(old_len, new_len, block_table, free_pages, *, page_size: int, n_tok: int,
              first_pos: int = 0, stream=None):
    """fsched_kv_layout: places for the step's new tokens.

    ``block_table`` [n_req, width] is updated in place.  Returns (slots [n_tok],
    positions [n_tok], q_start [n_req + 1], kv_len [n_req], used [2]), int32."""
    import torch
    n = old_len.shape[0]
    args = [_ints("old_len", old_len, (n,)), _ints("new_len", new_len, (n,)),
            _ints("free_pages", free_pages, (None,)),
            _ints("block_table", block_table, (n, None))]
    p = LayoutParams(n_req=n, n_tok=n_tok, page_size=page_size, table_width=block_table.shape[1],
                     n_free=free_pages.shape[0], first_pos=first_pos, flags=_fs.F_DEVICE_PTRS)
    # one allocation: slots, positions, q_start, kv_len, used, each on 16 bytes
    sizes = (max(0, n_tok), max(0, n_tok), n + 1, n, 2)
    room = [(x + 3) & ~3 for x in sizes]
    parts = torch.empty(sum(room), dtype=torch.int32, device=old_len.device).split(room)
    outs = tuple(x[:k] for x, k in zip(parts, sizes))
    _call("fsched_kv_layout", ctypes.byref(p), *args, *[x.data_ptr() for x in outs],
          _stream(stream))
    return outs


def qk_norm_rope(qkv, positions, slots, cos_sin, k_cache, v_cache, q_weight=None, k_weight=None,
                 *, eps: float = 1e-6, interleaved: bool = False, out=None, stream=None):
    """fsched_qk_norm_rope: ``qkv`` [n_tok, q_heads + 2 kv_heads, head_dim] to the
    rotated queries [n_tok, q_heads, head_dim] (``out``, made if None), keys and
    values put into the caches at ``slots`` (None: nowhere).  ``cos_sin`` [n_pos,
    rot_dim] f32 (None: no rotation, ``positions`` may be None)."""
    import torch
    c = _cache(k_cache, v_cache)
    dt, dim = k_cache.dtype, c.head_dim
    _last_contiguous("qkv", qkv, 3, dt)
    n, heads = qkv.shape[:2]
    q_heads = heads - 2 * c.kv_heads
    if q_heads < 1 or qkv.shape[2] != dim or (heads > 1 and qkv.stride(1) != dim):
        raise ValueError("qkv must be [n_tok, q_heads + 2 kv_heads, head_dim] with heads "
                         "head_dim apart")
    if cos_sin is not None and (cos_sin.dtype != torch.float32 or not cos_sin.is_cuda or
                                cos_sin.dim() != 2 or not cos_sin.is_contiguous()):
        raise ValueError("cos_sin must be a contiguous float32 GPU tensor [n_pos, rot_dim]")
    for name, w in (("q_weight", q_weight), ("k_weight", k_weight)):
        if w is not None:
            _last_contiguous(name, w, 1, dt)
            if w.shape[0] != dim:
                raise ValueError(f"{name} must have head_dim elements")
    if out is None:
        out = torch.empty((n, q_heads, dim), dtype=dt, device=qkv.device)
    else:
        _last_contiguous("out", out, 3, dt)
        if tuple(out.shape) != (n, q_heads, dim):
            raise ValueError(f"out must have shape {(n, q_heads, dim)}")
    if cos_sin is not None and positions is None:
        raise ValueError("a rotation needs positions")
    p = RopeParams(n_tok=n, q_heads=q_heads, rot_dim=0 if cos_sin is None else cos_sin.shape[1],
                   n_pos=0 if cos_sin is None else cos_sin.shape[0], interleaved=int(interleaved),
                   eps=eps, flags=_fs.F_DEVICE_PTRS, qkv_stride=qkv.stride(0),
                   q_token_stride=out.stride(0), q_head_stride=out.stride(1))

    def ptr(x):
        return None if x is None else x.data_ptr()
    _call("fsched_qk_norm_rope", ctypes.byref(p), ctypes.byref(c), qkv.data_ptr(),
          None if positions is None else _ints("positions", positions, (n,)),
          None if slots is None else _ints("slots", slots, (n,)), ptr(cos_sin), ptr(q_weight),
          ptr(k_weight), out.data_ptr(), _stream(stream))
    return out


def _attend(name, q, k_cache, v_cache, prefix_pages, prefix_len, block_table, q_start, kv_len,
            scale, window, n_sink, max_q, out, return_lse, workspace, stream):
    import torch
    c = _cache(k_cache, v_cache)
    _last_contiguous("q", q, 3, k_cache.dtype)
    n_tok, q_heads, dim = q.shape
    if dim != c.head_dim:
        raise ValueError("q and the cache differ in head_dim")
    n = kv_len.shape[0]
    ints = [_ints("block_table", block_table, (n, None)), _ints("q_start", q_start, (n + 1,)),
            _ints("kv_len", kv_len, (n,))]
    if prefix_pages is not None:
        need = -(-prefix_len // c.page_size) if prefix_len > 0 else 0
        pages = _ints("prefix_pages", prefix_pages, (None,))
        if prefix_pages.shape[0] < need:
            raise ValueError(f"prefix_pages must list the {need} pages of the prefix")
        ints.insert(0, pages)
    if out is None:
        out = torch.empty((n_tok, q_heads, dim), dtype=q.dtype, device=q.device)
    else:
        _last_contiguous("out", out, 3, q.dtype)
        if out.shape != q.shape:
            raise ValueError("out and q differ in shape")
    lse = torch.empty((n_tok, q_heads), dtype=torch.float32, device=q.device) \
        if return_lse else None
    if workspace is not None and not (workspace.is_cuda and workspace.is_contiguous()):
        raise ValueError("workspace must be a contiguous GPU tensor")
    qs, os = q.stride(), out.stride()
    p = AttnParams(n_req=n, n_tok=n_tok, q_heads=q_heads,
                   max_q=max(1, n_tok) if max_q is None else max_q,
                   table_width=block_table.shape[1], window=window, n_sink=n_sink,
                   prefix_len=prefix_len, scale=dim ** -0.5 if scale is None else scale,
                   flags=_fs.F_DEVICE_PTRS, q_token_stride=qs[0], q_head_stride=qs[1],
                   out_token_stride=os[0], out_head_stride=os[1])
    _call(name, ctypes.byref(p), ctypes.byref(c), q.data_ptr(), *ints, out.data_ptr(),
          None if lse is None else lse.data_ptr(),
          None if workspace is None else workspace.data_ptr(),
          0 if workspace is None else workspace.numel() * workspace.element_size(),
          _stream(stream))
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
    ``attend_workspace`` bytes, for calls that may not allocate (graph capture).
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
                     window: int = 0, n_sink: int = 0, device="cuda"):
    """A workspace (uint8 GPU tensor) for ``attend`` / ``attend_shared`` calls of this
    shape, 256-byte aligned; calls that may overlap in time need one each."""
    import torch
    c = KvCache(n_pages=0, page_size=page_size, kv_heads=kv_heads, head_dim=head_dim)
    p = AttnParams(n_req=n_req, n_tok=n_tok, q_heads=q_heads,
                   max_q=max(1, n_tok) if max_q is None else max_q, table_width=table_width,
                   window=window, n_sink=n_sink, prefix_len=prefix_len, scale=1.0,
                   flags=_fs.F_DEVICE_PTRS)
    size = _I64(0)
    _call("fsched_attend_workspace", ctypes.byref(p), ctypes.byref(c), ctypes.byref(size))
    return torch.empty(max(256, size.value), dtype=torch.uint8, device=device)
