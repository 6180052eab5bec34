"""The operators of a serving step: KV placement, norm and rotation of queries and
keys with the store into the cache, and attention over the paged cache.

Binding of ``fsched_kv_layout``, ``fsched_qk_norm_rope``, ``fsched_attend`` and
``fsched_attend_shared`` (``include/fsched.h`` says what each computes).  Every
array is a torch tensor, all of a call's on one GPU; the calls are enqueued on the
current torch stream and nothing is synchronised.  They are for serving: no gradient
flows through them.

With ``stream`` (a torch.cuda.Stream) a call runs as under ``torch.cuda.stream``: its
outputs and workspace are allocated for that stream, and the caller orders the
streams (inputs written on another one; results read on another one).  It is a stream of
the tensors' device (ValueError).

A cache is a pair of tensors [n_pages, kv_heads, page_size, head_dim]; a permuted
view (another order of page, head and slot in memory) does as well, as long as the
head dimension is contiguous.
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
    c = KvCache(n_pages=0, page_size=page_size, kv_heads=kv_heads, head_dim=head_dim)
    p = AttnParams(n_req=n_req, n_tok=n_tok, q_heads=q_heads,
                   max_q=max(1, n_tok) if max_q is None else max_q, table_width=table_width,
                   window=window, n_sink=n_sink, prefix_len=prefix_len, scale=1.0,
                   flags=_fs.F_DEVICE_PTRS)
    size = _I64(0)
    rc = _fs.lib().fsched_attend_workspace(ctypes.byref(p), ctypes.byref(c), ctypes.byref(size))
    if rc:
        raise _fs.FschedError(rc, "fsched_attend_workspace")
    return torch.empty(max(256, size.value), dtype=torch.uint8, device="cuda")
