"""The operators of a serving step: KV placement, norm and rotation of queries and
keys with the store into the cache, and attention over the paged cache; the same over a
cache of 4 bits, the attention weight of held tokens, and pages given up by it.

Binding of ``fsched_kv_layout``, ``fsched_qk_norm_rope``, ``fsched_attend``,
``fsched_attend_shared``, ``fsched_qk_norm_rope4``, ``fsched_kv4_read``,
``fsched_attend4``, ``fsched_attend_weight``, ``fsched_attend4_weight`` and
``fsched_kv_evict`` (``include/fsched.h`` says what each computes).  Every
array is a torch tensor, all of a call's on one GPU; the calls are enqueued on the
current torch stream and nothing is synchronised.  They are for serving: no gradient
flows through them.

With ``stream`` (a torch.cuda.Stream) a call runs as under ``torch.cuda.stream``: its
outputs and workspace are allocated for that stream, and the caller orders the
streams (inputs written on another one; results read on another one).  It is a stream of
the tensors' device (ValueError).

A cache is a pair of tensors [n_pages, kv_heads, page_size, head_dim]; a permuted
view (another order of page, head and slot in memory) does as well, as long as the
head dimension is contiguous.  A cache of 4 bits is one uint8 tensor [n_pages, kv_heads,
page_size / 16, 17 head_dim] (``kv4_cache`` makes one) that holds keys and values.
"""
from __future__ import annotations

import ctypes
import os

import torch

import paper_2608_02244_amd as _fs

try:
    from . import _step  # links libfsched.so, which lies beside it
except ImportError as e:
    raise RuntimeError(f"{os.path.dirname(os.path.abspath(__file__))}/_step.so is not built or "
                       f"does not load ({e}); run __graft_entry__.build() first (there is no "
                       "CPU fallback)") from e

_I32, _I64, _F32, _U32, _P = (ctypes.c_int32, ctypes.c_int64, ctypes.c_float, ctypes.c_uint32,
                              ctypes.c_void_p)


class KvCache(ctypes.Structure):
    _fields_ = [("k", _P), ("v", _P), ("k_stride", _I64 * 3), ("v_stride", _I64 * 3),
                ("n_pages", _I32), ("page_size", _I32), ("kv_heads", _I32), ("head_dim", _I32),
                ("dtype", _I32), ("reserved", _I32)]


class Kv4Cache(ctypes.Structure):
    _fields_ = [("data", _P), ("stride", _I64 * 3)] + \
        [(n, _I32) for n in ("n_pages", "page_size", "kv_heads", "head_dim", "dtype", "reserved")]


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


class ReadParams(ctypes.Structure):
    _fields_ = [("n_tok", _I32), ("flags", _U32), ("token_stride", _I64), ("head_stride", _I64)]


class EvictParams(ctypes.Structure):
    _fields_ = [(n, _I32) for n in ("n_req", "table_width", "page_size", "n_sink", "n_recent",
                                    "n_freed")] + \
        [("flags", _U32), ("reserved", _I32), ("weight_stride", _I64)]


def _current(x):
    """Address of torch's current stream on the device of ``x`` (what is no GPU tensor the
    call itself refuses)."""
    if not isinstance(x, torch.Tensor) or not x.is_cuda:
        return 0
    return torch._C._cuda_getCurrentRawStream(x.get_device())


def _on(stream, x):
    """``stream`` as torch's current one; it must be of the device of ``x``, whose current
    stream a call takes."""
    if isinstance(x, torch.Tensor) and x.device != stream.device:
        raise ValueError(f"the stream is on {stream.device}, the tensors are on {x.device}")
    return torch.cuda.stream(stream)


def kv_layout(old_len, new_len, block_table, free_pages, *, page_size: int, n_tok: int,
              first_pos: int = 0, stream=None):
    """fsched_kv_layout: places for the step's new tokens.

    ``block_table`` [n_req, width] is updated in place.  Returns (slots [n_tok],
    positions [n_tok], q_start [n_req + 1], kv_len [n_req], used [2]), int32."""
    if stream is not None:
        with _on(stream, old_len):
            return kv_layout(old_len, new_len, block_table, free_pages, page_size=page_size,
                             n_tok=n_tok, first_pos=first_pos)
    return _step.kv_layout(old_len, new_len, block_table, free_pages, page_size, n_tok, first_pos,
                           _current(old_len))


def qk_norm_rope(qkv, positions, slots, cos_sin, k_cache, v_cache, q_weight=None, k_weight=None,
                 *, eps: float = 1e-6, interleaved: bool = False, out=None, stream=None):
    """fsched_qk_norm_rope: ``qkv`` [n_tok, q_heads + 2 kv_heads, head_dim] to the
    rotated queries [n_tok, q_heads, head_dim] (``out``, made if None), keys and
    values put into the caches at ``slots`` (None: nowhere).  ``cos_sin`` [n_pos,
    rot_dim] f32 (None: no rotation, ``positions`` may be None)."""
    if stream is not None:
        with _on(stream, qkv):
            return qk_norm_rope(qkv, positions, slots, cos_sin, k_cache, v_cache, q_weight,
                                k_weight, eps=eps, interleaved=interleaved, out=out)
    return _step.qk_norm_rope(qkv, positions, slots, cos_sin, k_cache, v_cache, q_weight,
                              k_weight, eps, interleaved, out, _current(qkv))


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
    torch's allocator.
    Returns out, or (out, lse [n_tok, q_heads] float32) with ``return_lse``."""
    if stream is not None:
        with _on(stream, q):
            return attend(q, k_cache, v_cache, block_table, q_start, kv_len,
                          scale=scale, window=window, n_sink=n_sink, max_q=max_q, out=out,
                          return_lse=return_lse, workspace=workspace)
    return _step.attend(q, k_cache, v_cache, None, 0, block_table, q_start, kv_len, scale, window,
                        n_sink, max_q, out, return_lse, workspace, _current(q))


def attend_shared(q, k_cache, v_cache, prefix_pages, prefix_len: int, block_table, q_start,
                  kv_len, *, scale=None, window: int = 0, n_sink: int = 0, max_q=None, out=None,
                  return_lse: bool = False, workspace=None, stream=None):
    """fsched_attend_shared: ``attend`` for requests that all begin with the
    ``prefix_len`` tokens held in ``prefix_pages``; ``block_table`` and ``kv_len``
    describe each request's own tokens behind them."""
    if stream is not None:
        with _on(stream, q):
            return attend_shared(q, k_cache, v_cache, prefix_pages, prefix_len, block_table,
                                 q_start, kv_len, scale=scale, window=window, n_sink=n_sink,
                                 max_q=max_q, out=out, return_lse=return_lse,
                                 workspace=workspace)
    return _step.attend(q, k_cache, v_cache, prefix_pages, prefix_len, block_table, q_start,
                        kv_len, scale, window, n_sink, max_q, out, return_lse, workspace,
                        _current(q))


def attend_workspace(n_tok: int, n_req: int, q_heads: int, kv_heads: int, head_dim: int, *,
                     page_size: int, table_width: int, max_q=None, prefix_len: int = 0,
                     window: int = 0, n_sink: int = 0):
    """A workspace (uint8 GPU tensor) for ``attend`` / ``attend_shared`` calls of this
    shape, 256-byte aligned; calls that may overlap in time need one each."""
    return _workspace("fsched_attend_workspace",
                      KvCache(n_pages=0, page_size=page_size, kv_heads=kv_heads,
                              head_dim=head_dim),
                      n_tok, n_req, q_heads, table_width, max_q, prefix_len, window, n_sink)


def _workspace(name, c, n_tok, n_req, q_heads, table_width, max_q, prefix_len, window, n_sink):
    p = AttnParams(n_req=n_req, n_tok=n_tok, q_heads=q_heads,
                   max_q=max(1, n_tok) if max_q is None else max_q, table_width=table_width,
                   window=window, n_sink=n_sink, prefix_len=prefix_len, scale=1.0,
                   flags=_fs.F_DEVICE_PTRS)
    size = _I64(0)
    rc = getattr(_fs.lib(), name)(ctypes.byref(p), ctypes.byref(c), ctypes.byref(size))
    if rc:
        raise _fs.FschedError(rc, name)
    return torch.empty(max(256, size.value), dtype=torch.uint8, device="cuda")


def kv4_cache(n_pages: int, kv_heads: int, page_size: int, head_dim: int, *, device="cuda"):
    """An empty cache of 4 bits an element (its contents are undefined): uint8 [n_pages,
    kv_heads, page_size / 16, 17 head_dim], keys and values."""
    if not 16 <= page_size <= 65536 or page_size & (page_size - 1):
        raise ValueError("a cache of 4 bits has pages of 16 to 65,536 tokens, a power of two")
    return torch.empty(n_pages, kv_heads, page_size // 16, 17 * head_dim, dtype=torch.uint8,
                       device=device)


def qk_norm_rope4(qkv, positions, slots, cos_sin, cache, q_weight=None, k_weight=None, *,
                  eps: float = 1e-6, interleaved: bool = False, out=None, stream=None):
    """fsched_qk_norm_rope4: ``qk_norm_rope`` with keys and values put into a cache of 4
    bits."""
    if stream is not None:
        with _on(stream, qkv):
            return qk_norm_rope4(qkv, positions, slots, cos_sin, cache, q_weight, k_weight,
                                 eps=eps, interleaved=interleaved, out=out)
    return _step.qk_norm_rope4(qkv, positions, slots, cos_sin, cache, q_weight, k_weight, eps,
                               interleaved, out, _current(qkv))


def kv4_read(cache, slots, *, dtype=torch.bfloat16, stream=None):
    """fsched_kv4_read: what a cache of 4 bits holds at ``slots`` [n] (-1: zeros), as
    (keys, values) [n, kv_heads, head_dim] of ``dtype``, the type of the rows that were
    stored."""
    if dtype not in (torch.bfloat16, torch.float16):
        raise ValueError("dtype must be torch.bfloat16 or torch.float16")
    if stream is not None:
        with _on(stream, cache):
            return kv4_read(cache, slots, dtype=dtype)
    return _step.kv4_read(cache, slots, dtype == torch.float16, _current(cache))


def attend4(q, cache, block_table, q_start, kv_len, *, prefix_pages=None, prefix_len: int = 0,
            scale=None, window: int = 0, n_sink: int = 0, max_q=None, out=None,
            return_lse: bool = False, workspace=None, stream=None):
    """fsched_attend4: ``attend`` (with ``prefix_pages`` and ``prefix_len``:
    ``attend_shared``) over a cache of 4 bits.  The elements of ``q`` say how the cache's
    are read.  ``workspace``: of ``attend4_workspace``."""
    if stream is not None:
        with _on(stream, q):
            return attend4(q, cache, block_table, q_start, kv_len, prefix_pages=prefix_pages,
                           prefix_len=prefix_len, scale=scale, window=window, n_sink=n_sink,
                           max_q=max_q, out=out, return_lse=return_lse, workspace=workspace)
    return _step.attend4(q, cache, prefix_pages, prefix_len, block_table, q_start, kv_len, scale,
                         window, n_sink, max_q, out, return_lse, workspace, _current(q))


def attend4_workspace(n_tok: int, n_req: int, q_heads: int, kv_heads: int, head_dim: int, *,
                      page_size: int, table_width: int, max_q=None, prefix_len: int = 0,
                      window: int = 0, n_sink: int = 0):
    """``attend_workspace`` for ``attend4`` calls."""
    return _workspace("fsched_attend4_workspace",
                      Kv4Cache(n_pages=0, page_size=page_size, kv_heads=kv_heads,
                               head_dim=head_dim),
                      n_tok, n_req, q_heads, table_width, max_q, prefix_len, window, n_sink)


def attend_weight(q, lse, k_cache, block_table, q_start, kv_len, weight, *, scale=None,
                  window: int = 0, n_sink: int = 0, prefix_len: int = 0, max_q=None, stream=None):
    """fsched_attend_weight: adds to ``weight`` [n_req, width * page_size] (float32, rows
    may be apart) what each held token gets of the new tokens' attention, summed over
    tokens and heads.  ``lse`` [n_tok, q_heads] is what ``attend`` of the same arguments
    returned (``attend_shared`` with ``prefix_len``).  Returns ``weight``."""
    if stream is not None:
        with _on(stream, q):
            return attend_weight(q, lse, k_cache, block_table, q_start, kv_len, weight,
                                 scale=scale, window=window, n_sink=n_sink,
                                 prefix_len=prefix_len, max_q=max_q)
    return _step.attend_weight(q, lse, k_cache, block_table, q_start, kv_len, weight, scale,
                               window, n_sink, max_q, prefix_len, _current(q))


def attend4_weight(q, lse, cache, block_table, q_start, kv_len, weight, *, scale=None,
                   window: int = 0, n_sink: int = 0, prefix_len: int = 0, max_q=None,
                   stream=None):
    """fsched_attend4_weight: ``attend_weight`` over a cache of 4 bits."""
    if stream is not None:
        with _on(stream, q):
            return attend4_weight(q, lse, cache, block_table, q_start, kv_len, weight,
                                  scale=scale, window=window, n_sink=n_sink,
                                  prefix_len=prefix_len, max_q=max_q)
    return _step.attend4_weight(q, lse, cache, block_table, q_start, kv_len, weight, scale,
                                window, n_sink, max_q, prefix_len, _current(q))


def kv_evict(weight, kv_len, block_table, budget, *, page_size: int, n_sink: int = 0,
             n_recent: int = 0, n_freed=None, stream=None):
    """fsched_kv_evict: pages of least ``weight`` [n_req, width * page_size] given up until
    every request holds at most ``budget`` [n_req] tokens, but for its first ``n_sink`` and
    last ``n_recent``.  ``n_freed``: room for ids of freed pages (None: for the whole
    table's).

    Returns (block_table, weight, kv_len, freed [n_freed], count [1]), new tensors: tables
    and weights closed up (behind what stays -1 and 0), the ids of the freed pages with -1
    behind them, and how many there are.  A page that several requests list is given up by
    each of them for itself: its id is there once for each."""
    if stream is not None:
        with _on(stream, weight):
            return kv_evict(weight, kv_len, block_table, budget, page_size=page_size,
                            n_sink=n_sink, n_recent=n_recent, n_freed=n_freed)
    return _step.kv_evict(weight, kv_len, block_table, budget, page_size, n_sink, n_recent,
                          n_freed, _current(weight))
