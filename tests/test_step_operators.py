"""The step operators' C entry points and their binding, without a GPU: layouts of
their structs and what they refuse before any device work."""
import ctypes

import numpy as np
import pytest

import paper_2608_02244_amd as fs
from paper_2608_02244_amd import step

D = ctypes.c_void_p(0x10000)  # aligned and never dereferenced: every case ends before device work
DEV = fs.F_DEVICE_PTRS


def test_struct_sizes():
    assert [ctypes.sizeof(t) for t in (step.KvCache, step.LayoutParams, step.RopeParams,
                                       step.AttnParams)] == [88, 32, 56, 72]
    assert step.KvCache.n_pages.offset == 64 and step.RopeParams.qkv_stride.offset == 32
    assert step.AttnParams.scale.offset == 32 and step.AttnParams.q_token_stride.offset == 40


def cache(**kw):
    v = dict(k=0x20000, v=0x30000, k_stride=(ctypes.c_int64 * 3)(8192, 2048, 128),
             v_stride=(ctypes.c_int64 * 3)(8192, 2048, 128), n_pages=10, page_size=16, kv_heads=4,
             head_dim=128, dtype=0)
    v.update(kw)
    return step.KvCache(**v)


def strides(*x):
    return (ctypes.c_int64 * 3)(*x)


BAD_CACHE = [(dict(n_pages=-1), fs.EINVAL), (dict(page_size=0), fs.EINVAL),
             (dict(page_size=24), fs.EINVAL), (dict(page_size=131072), fs.ETOOLARGE),
             (dict(kv_heads=0), fs.EINVAL), (dict(kv_heads=1025), fs.ETOOLARGE),
             (dict(head_dim=0), fs.EINVAL), (dict(head_dim=80), fs.ENOTIMPL),
             (dict(dtype=2), fs.EINVAL), (dict(reserved=1), fs.EINVAL),
             (dict(k=0x20002), fs.EINVAL), (dict(v=0x30008), fs.EINVAL),
             (dict(k_stride=strides(8192, 2048, 132)), fs.EINVAL),
             (dict(v_stride=strides(-8192, 2048, 128)), fs.EINVAL),
             (dict(k=None), fs.EINVAL)]


def layout(p=None, ptr=D, **kw):
    v = dict(n_req=4, n_tok=8, page_size=16, table_width=8, n_free=16, first_pos=0, flags=DEV)
    v.update(kw)
    p = step.LayoutParams(**v)
    return fs.lib().fsched_kv_layout(ctypes.byref(p), *[ptr] * 9, None)


@pytest.mark.parametrize("kw,code", [
    (dict(flags=0), fs.EINVAL), (dict(flags=DEV | 8), fs.EINVAL), (dict(n_req=-1), fs.EINVAL),
    (dict(n_tok=-1), fs.EINVAL), (dict(page_size=0), fs.EINVAL), (dict(page_size=12), fs.EINVAL),
    (dict(table_width=-1), fs.EINVAL), (dict(n_free=-1), fs.EINVAL),
    (dict(first_pos=-1), fs.EINVAL), (dict(reserved=1), fs.EINVAL),
    (dict(n_req=4097), fs.ETOOLARGE), (dict(n_tok=(1 << 24) + 1), fs.ETOOLARGE),
    (dict(page_size=1 << 17), fs.ETOOLARGE),
    (dict(table_width=1 << 28, page_size=16), fs.ETOOLARGE), (dict(ptr=None), fs.EINVAL)])
def test_layout_refuses(kw, code):
    assert layout(**kw) == code


def test_null_params_are_refused():
    L = fs.lib()
    c, x = cache(), ctypes.c_int64()
    assert L.fsched_kv_layout(None, *[D] * 9, None) == fs.EINVAL
    assert L.fsched_qk_norm_rope(None, ctypes.byref(c), *[D] * 7, None) == fs.EINVAL
    assert L.fsched_attend(None, ctypes.byref(c), *[D] * 6, None, 0, None) == fs.EINVAL
    assert L.fsched_attend_shared(None, ctypes.byref(c), *[D] * 7, None, 0, None) == fs.EINVAL
    assert L.fsched_attend_workspace(None, ctypes.byref(c), ctypes.byref(x)) == fs.EINVAL
    p = attn_params()
    assert L.fsched_attend(ctypes.byref(p), None, *[D] * 6, None, 0, None) == fs.EINVAL
    assert L.fsched_attend_workspace(ctypes.byref(p), ctypes.byref(c), None) == fs.EINVAL


def rope(c=None, ptrs=None, **kw):
    v = dict(n_tok=4, q_heads=8, rot_dim=128, n_pos=64, interleaved=0, eps=1e-6, flags=DEV,
             qkv_stride=16 * 128, q_token_stride=8 * 128, q_head_stride=128)
    v.update(kw)
    p, c = step.RopeParams(**v), c or cache()
    ptrs = ptrs or [D] * 7
    return fs.lib().fsched_qk_norm_rope(ctypes.byref(p), ctypes.byref(c), *ptrs, None)


@pytest.mark.parametrize("kw,code", [
    (dict(flags=0), fs.EINVAL), (dict(flags=DEV | 32), fs.EINVAL), (dict(n_tok=-1), fs.EINVAL),
    (dict(q_heads=0), fs.EINVAL), (dict(q_heads=1025), fs.ETOOLARGE),
    (dict(rot_dim=-16), fs.EINVAL), (dict(rot_dim=24), fs.EINVAL), (dict(rot_dim=144), fs.EINVAL),
    (dict(n_pos=-1), fs.EINVAL), (dict(interleaved=2), fs.EINVAL), (dict(eps=-1.0), fs.EINVAL),
    (dict(eps=float("nan")), fs.EINVAL), (dict(eps=float("inf")), fs.EINVAL),
    (dict(qkv_stride=2044), fs.EINVAL), (dict(q_token_stride=-8), fs.EINVAL),
    (dict(q_head_stride=4), fs.EINVAL), (dict(reserved=3), fs.EINVAL),
    (dict(n_tok=(1 << 24) + 1), fs.ETOOLARGE), (dict(n_tok=0), fs.OK)])
def test_rope_refuses(kw, code):
    assert rope(**kw) == code


@pytest.mark.parametrize("i", range(7))
def test_rope_refuses_pointers(i):
    # order: qkv, positions, slots, cos_sin, q_weight, k_weight, q_out
    odd = [D] * 7
    odd[i] = ctypes.c_void_p(0x10004)
    if i not in (1, 2):  # index arrays need no more than their own alignment
        assert rope(ptrs=odd) == fs.EINVAL
    null = [D] * 7
    null[i] = None
    if i in (0, 1, 3, 6):
        assert rope(ptrs=null) == fs.EINVAL


@pytest.mark.parametrize("kw,code", BAD_CACHE)
def test_rope_refuses_caches(kw, code):
    assert rope(c=cache(**kw)) == code


def attn_params(**kw):
    v = dict(n_req=4, n_tok=8, q_heads=8, max_q=8, table_width=8, window=0, n_sink=0,
             prefix_len=0, scale=0.1, flags=DEV, q_token_stride=1024, q_head_stride=128,
             out_token_stride=1024, out_head_stride=128)
    v.update(kw)
    return step.AttnParams(**v)


def attend(c=None, ptrs=None, ws=None, ws_bytes=0, **kw):
    p, c = attn_params(**kw), c or cache()
    return fs.lib().fsched_attend(ctypes.byref(p), ctypes.byref(c), *(ptrs or [D] * 6), ws,
                                  ws_bytes, None)


def attend_shared(c=None, ptrs=None, **kw):
    p, c = attn_params(**kw), c or cache()
    return fs.lib().fsched_attend_shared(ctypes.byref(p), ctypes.byref(c), *(ptrs or [D] * 7),
                                         None, 0, None)


BAD_ATTN = [
    (dict(flags=0), fs.EINVAL), (dict(flags=DEV | 16), fs.EINVAL), (dict(n_req=-1), fs.EINVAL),
    (dict(n_tok=-1), fs.EINVAL), (dict(q_heads=0), fs.EINVAL), (dict(q_heads=6), fs.EINVAL),
    (dict(q_heads=1028), fs.ETOOLARGE), (dict(max_q=0), fs.EINVAL), (dict(max_q=9), fs.EINVAL),
    (dict(table_width=-1), fs.EINVAL), (dict(window=-1), fs.EINVAL), (dict(n_sink=-1), fs.EINVAL),
    (dict(prefix_len=-1), fs.EINVAL), (dict(scale=0.0), fs.EINVAL), (dict(scale=-1.0), fs.EINVAL),
    (dict(scale=float("nan")), fs.EINVAL), (dict(scale=float("inf")), fs.EINVAL),
    (dict(q_token_stride=1020), fs.EINVAL), (dict(q_head_stride=-128), fs.EINVAL),
    (dict(out_token_stride=4), fs.EINVAL), (dict(out_head_stride=132), fs.EINVAL),
    (dict(n_req=4097), fs.ETOOLARGE), (dict(n_tok=(1 << 24) + 1), fs.ETOOLARGE),
    (dict(table_width=1 << 27), fs.ETOOLARGE)]


@pytest.mark.parametrize("kw,code", BAD_ATTN + [(dict(n_tok=0), fs.OK), (dict(n_req=0), fs.OK)])
def test_attend_refuses(kw, code):
    assert attend(**kw) == code
    assert attend_shared(**kw) == code


def test_attend_refuses_a_prefix_and_shared_its_length():
    assert attend(prefix_len=16) == fs.EINVAL
    assert attend_shared(prefix_len=1 << 30) == fs.ETOOLARGE
    null = [D] * 7
    null[1] = None  # the prefix's pages
    assert attend_shared(ptrs=null, prefix_len=16) == fs.EINVAL


@pytest.mark.parametrize("i", range(5))
def test_attend_refuses_pointers(i):
    # order: q, table, q_start, kv_len, out, lse
    null = [D] * 6
    null[i] = None
    assert attend(ptrs=null) == fs.EINVAL
    if i in (0, 4):
        odd = [D] * 6
        odd[i] = ctypes.c_void_p(0x10008)
        assert attend(ptrs=odd) == fs.EINVAL


@pytest.mark.parametrize("kw,code", BAD_CACHE)
def test_attend_refuses_caches(kw, code):
    assert attend(c=cache(**kw)) == code


def test_attend_refuses_an_unaligned_workspace():
    assert attend(ws=ctypes.c_void_p(0x10010), ws_bytes=1 << 40) == fs.EINVAL


def test_workspace_size_is_refused_like_the_call_and_zero_without_work():
    L, x, c = fs.lib(), ctypes.c_int64(-1), cache()
    for kw, code in BAD_ATTN:
        p = attn_params(**kw)
        assert L.fsched_attend_workspace(ctypes.byref(p), ctypes.byref(c), ctypes.byref(x)) == code
    p = attn_params(n_tok=0)
    assert L.fsched_attend_workspace(ctypes.byref(p), ctypes.byref(c), ctypes.byref(x)) == fs.OK
    assert x.value == 0


def test_binding_refuses_what_is_not_on_the_gpu():
    import torch
    i = torch.zeros(4, dtype=torch.int32)
    x = torch.zeros(4, 8, 64, dtype=torch.bfloat16)
    kv = torch.zeros(2, 2, 16, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="old_len"):
        fs.kv_layout(i, i, i.view(4, 1), i, page_size=16, n_tok=4)
    with pytest.raises(ValueError, match="k_cache"):
        fs.qk_norm_rope(x, i, i, None, kv, kv)
    with pytest.raises(ValueError, match="k_cache"):
        fs.attend(x, kv, kv, i.view(4, 1), i, i)
    with pytest.raises(ValueError, match="bfloat16 or float16"):
        fs.attend(x, kv.float(), kv.float(), i.view(4, 1), i, i)


def test_binding_refuses_tensors_of_several_devices():
    import torch
    i = torch.zeros(4, dtype=torch.int32)
    m = torch.zeros(4, 1, dtype=torch.int32, device="meta")
    with pytest.raises(ValueError, match="one GPU"):
        fs.kv_layout(i, i, m, i, page_size=16, n_tok=4)
    with pytest.raises(ValueError, match="one GPU"):
        fs.attend(m, m, m, i.view(4, 1), i, i)


def test_package_still_loads_without_torch_in_hand():
    """The evaluation calls work on numpy arrays alone: importing the package and its
    step binding loads no torch."""
    import subprocess
    import sys
    code = "import sys; import paper_2608_02244_amd; sys.exit('torch' in sys.modules)"
    assert subprocess.run([sys.executable, "-c", code]).returncode == 0
    assert np.dtype(np.int32).itemsize == 4
