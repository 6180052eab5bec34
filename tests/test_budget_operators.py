"""The C entry points of the cache of 4 bits, attention weights and evictions and their
binding, without a GPU: layouts of their structs and what they refuse before any device
work."""
import ctypes

import pytest

import paper_2608_02244_amd as fs
from paper_2608_02244_amd import step

D = ctypes.c_void_p(0x10000)  # aligned and never dereferenced: every case ends before device work
DEV = fs.F_DEVICE_PTRS


def ref(x):
    return ctypes.byref(x)


def strides(*x):
    return (ctypes.c_int64 * 3)(*x)


def test_struct_sizes():
    assert [ctypes.sizeof(t) for t in (step.Kv4Cache, step.ReadParams, step.EvictParams)] == \
        [56, 24, 40]
    assert step.Kv4Cache.n_pages.offset == 32 and step.EvictParams.weight_stride.offset == 32


def cache4(**kw):
    v = dict(data=0x20000, stride=strides(4 * 2176, 2176, 2176), n_pages=10, page_size=16,
             kv_heads=4, head_dim=128, dtype=0)
    v.update(kw)
    return step.Kv4Cache(**v)


def cache(**kw):
    v = dict(k=0x20000, v=0x30000, k_stride=strides(8192, 2048, 128),
             v_stride=strides(8192, 2048, 128), n_pages=10, page_size=16, kv_heads=4,
             head_dim=128, dtype=0)
    v.update(kw)
    return step.KvCache(**v)


BAD_CACHE = [(dict(n_pages=-1), fs.EINVAL), (dict(page_size=0), fs.EINVAL),
             (dict(page_size=8), fs.EINVAL), (dict(page_size=48), fs.EINVAL),
             (dict(page_size=131072), fs.ETOOLARGE), (dict(kv_heads=0), fs.EINVAL),
             (dict(kv_heads=1025), fs.ETOOLARGE), (dict(head_dim=0), fs.EINVAL),
             (dict(head_dim=96), fs.ENOTIMPL), (dict(dtype=2), fs.EINVAL),
             (dict(reserved=1), fs.EINVAL), (dict(data=0x20008), fs.EINVAL),
             (dict(data=None), fs.EINVAL), (dict(stride=strides(8704, 2176, 2184)), fs.EINVAL),
             (dict(stride=strides(-16, 2176, 2176)), fs.EINVAL),
             (dict(stride=strides(1 << 41, 2176, 2176)), fs.ETOOLARGE)]


def rope4(c=None, ptrs=None, **kw):
    v = dict(n_tok=4, q_heads=8, rot_dim=128, n_pos=64, interleaved=0, eps=1e-6, flags=DEV,
             qkv_stride=16 * 128, q_token_stride=8 * 128, q_head_stride=128)
    v.update(kw)
    return fs.lib().fsched_qk_norm_rope4(ref(step.RopeParams(**v)), ref(c or cache4()),
                                         *(ptrs or [D] * 7), None)


def attn_params(**kw):
    v = dict(n_req=4, n_tok=8, q_heads=8, max_q=8, table_width=8, window=0, n_sink=0,
             prefix_len=0, scale=0.1, flags=DEV, q_token_stride=1024, q_head_stride=128,
             out_token_stride=1024, out_head_stride=128)
    v.update(kw)
    return step.AttnParams(**v)


def attend4(c=None, ptrs=None, ws=None, ws_bytes=0, **kw):
    return fs.lib().fsched_attend4(ref(attn_params(**kw)), ref(c or cache4()),
                                   *(ptrs or [D] * 7), ws, ws_bytes, None)


def weight(c=None, ptrs=None, stride=128, ws=None, ws_bytes=0, **kw):
    """Over either kind of cache; order: q, lse, table, q_start, kv_len, weight."""
    c = c or cache4()
    f = fs.lib().fsched_attend4_weight if isinstance(c, step.Kv4Cache) else \
        fs.lib().fsched_attend_weight
    return f(ref(attn_params(**kw)), ref(c), *(ptrs or [D] * 6), stride, ws, ws_bytes, None)


def read4(c=None, ptrs=None, **kw):
    v = dict(n_tok=4, flags=DEV, token_stride=512, head_stride=128)
    v.update(kw)
    return fs.lib().fsched_kv4_read(ref(step.ReadParams(**v)), ref(c or cache4()),
                                    *(ptrs or [D] * 3), None)


def evict(ptrs=None, ws=None, ws_bytes=0, **kw):
    v = dict(n_req=4, table_width=8, page_size=16, n_sink=0, n_recent=0, n_freed=32, flags=DEV,
             weight_stride=128)
    v.update(kw)
    return fs.lib().fsched_kv_evict(ref(step.EvictParams(**v)), *(ptrs or [D] * 9), ws, ws_bytes,
                                    None)


def without(n, i, value=None):
    p = [D] * n
    p[i] = value
    return p


@pytest.mark.parametrize("kw,code", BAD_CACHE)
def test_caches_are_refused(kw, code):
    c = cache4(**kw)
    assert rope4(c) == attend4(c) == weight(c) == read4(c) == code
    x = ctypes.c_int64()
    if kw != dict(data=None):
        for f in (fs.lib().fsched_attend4_workspace, fs.lib().fsched_attend4_weight_workspace):
            assert f(ref(attn_params()), ref(c), ref(x)) == code


BAD_ATTN = [
    (dict(flags=0), fs.EINVAL), (dict(flags=DEV | 16), fs.EINVAL), (dict(n_req=-1), fs.EINVAL),
    (dict(n_tok=-1), fs.EINVAL), (dict(q_heads=0), fs.EINVAL), (dict(q_heads=6), fs.EINVAL),
    (dict(q_heads=1028), fs.ETOOLARGE), (dict(max_q=0), fs.EINVAL), (dict(max_q=9), fs.EINVAL),
    (dict(table_width=-1), fs.EINVAL), (dict(window=-1), fs.EINVAL), (dict(n_sink=-1), fs.EINVAL),
    (dict(prefix_len=-1), fs.EINVAL), (dict(scale=0.0), fs.EINVAL),
    (dict(scale=float("nan")), fs.EINVAL), (dict(q_token_stride=1020), fs.EINVAL),
    (dict(q_head_stride=-128), fs.EINVAL), (dict(n_req=4097), fs.ETOOLARGE),
    (dict(n_tok=(1 << 24) + 1), fs.ETOOLARGE), (dict(table_width=1 << 27), fs.ETOOLARGE)]


@pytest.mark.parametrize("kw,code", BAD_ATTN + [(dict(n_tok=0), fs.OK), (dict(n_req=0), fs.OK)])
def test_attention_parameters_are_refused(kw, code):
    assert attend4(**kw) == code
    stride = max(128, 16 * kw.get("table_width", 0))
    assert weight(stride=stride, **kw) == weight(cache(), stride=stride, **kw) == code
    x = ctypes.c_int64(-1)
    for f, c in ((fs.lib().fsched_attend4_workspace, cache4()),
                 (fs.lib().fsched_attend4_weight_workspace, cache4()),
                 (fs.lib().fsched_attend_weight_workspace, cache())):
        assert f(ref(attn_params(**kw)), ref(c), ref(x)) == code
        assert code or x.value == 0


@pytest.mark.parametrize("i", range(6))
def test_pointers_are_refused(i):
    # q, prefix pages (only with a prefix), table, q_start, kv_len, out
    assert attend4(ptrs=without(7, i), prefix_len=16) == fs.EINVAL
    # q, lse, table, q_start, kv_len, weight
    assert weight(ptrs=without(6, i)) == weight(cache(), ptrs=without(6, i)) == fs.EINVAL
    if i in (0, 5):
        assert attend4(ptrs=without(7, i, ctypes.c_void_p(0x10008))) == fs.EINVAL
    if i < 3:  # slots, k_out, v_out
        assert read4(ptrs=without(3, i)) == fs.EINVAL
        if i:
            assert read4(ptrs=without(3, i, ctypes.c_void_p(0x10008))) == fs.EINVAL
    if i in (0, 1, 3):
        assert rope4(ptrs=without(7, i)) == fs.EINVAL


def test_weights_rows_and_sizes_are_refused():
    assert weight(stride=127) == weight(cache(), stride=127) == fs.EINVAL
    assert weight(stride=1 << 41) == fs.ETOOLARGE
    assert weight(q_token_stride=1 << 26) == fs.ETOOLARGE
    assert weight(n_tok=1 << 24, max_q=1 << 24, q_heads=1024, q_token_stride=0) == fs.ETOOLARGE
    assert weight(cache(v=None, k=None)) == fs.EINVAL
    assert weight(table_width=0, stride=0) == fs.OK
    assert weight(ws=ctypes.c_void_p(0x10010), ws_bytes=1 << 40) == fs.EINVAL
    assert attend4(ws=ctypes.c_void_p(0x10010), ws_bytes=1 << 40) == fs.EINVAL


@pytest.mark.parametrize("kw,code", [
    (dict(flags=0), fs.EINVAL), (dict(flags=DEV | 8), fs.EINVAL), (dict(n_tok=-1), fs.EINVAL),
    (dict(token_stride=500), fs.EINVAL), (dict(head_stride=-128), fs.EINVAL),
    (dict(n_tok=(1 << 24) + 1), fs.ETOOLARGE), (dict(n_tok=0), fs.OK)])
def test_read_refuses(kw, code):
    assert read4(**kw) == code


@pytest.mark.parametrize("kw,code", [
    (dict(flags=0), fs.EINVAL), (dict(n_tok=-1), fs.EINVAL), (dict(q_heads=0), fs.EINVAL),
    (dict(rot_dim=24), fs.EINVAL), (dict(rot_dim=144), fs.EINVAL), (dict(eps=-1.0), fs.EINVAL),
    (dict(interleaved=2), fs.EINVAL), (dict(qkv_stride=2044), fs.EINVAL), (dict(n_tok=0), fs.OK)])
def test_store_refuses(kw, code):
    assert rope4(**kw) == code


@pytest.mark.parametrize("kw,code", [
    (dict(flags=0), fs.EINVAL), (dict(flags=DEV | 32), fs.EINVAL), (dict(n_req=-1), fs.EINVAL),
    (dict(table_width=-1), fs.EINVAL), (dict(page_size=0), fs.EINVAL),
    (dict(page_size=12), fs.EINVAL), (dict(n_sink=-1), fs.EINVAL), (dict(n_recent=-1), fs.EINVAL),
    (dict(n_freed=-1), fs.EINVAL), (dict(reserved=1), fs.EINVAL),
    (dict(weight_stride=127), fs.EINVAL), (dict(n_req=4097), fs.ETOOLARGE),
    (dict(page_size=1 << 17, weight_stride=1 << 21), fs.ETOOLARGE),
    (dict(table_width=1 << 27, weight_stride=1 << 31), fs.ETOOLARGE),
    (dict(n_req=4096, table_width=1 << 19, weight_stride=1 << 23), fs.ETOOLARGE)])
def test_evict_refuses(kw, code):
    assert evict(**kw) == code
    v = dict(n_req=4, table_width=8, page_size=16, n_freed=32, flags=DEV, weight_stride=128)
    v.update(kw)
    assert fs.lib().fsched_kv_evict_workspace(ref(step.EvictParams(**v)),
                                              ref(ctypes.c_int64())) == code


@pytest.mark.parametrize("i", range(9))
def test_evict_refuses_pointers(i):
    assert evict(ptrs=without(9, i)) == fs.EINVAL
    assert evict(ws=ctypes.c_void_p(0x10010), ws_bytes=1 << 40) == fs.EINVAL


def test_null_structs_are_refused():
    L, x = fs.lib(), ctypes.c_int64()
    p, c, k = attn_params(), cache4(), cache()
    assert L.fsched_qk_norm_rope4(None, ref(c), *[D] * 7, None) == fs.EINVAL
    assert L.fsched_kv4_read(None, ref(c), *[D] * 3, None) == fs.EINVAL
    assert L.fsched_kv4_read(ref(step.ReadParams(n_tok=1, flags=DEV)), None, *[D] * 3,
                             None) == fs.EINVAL
    assert L.fsched_attend4(None, ref(c), *[D] * 7, None, 0, None) == fs.EINVAL
    assert L.fsched_attend4(ref(p), None, *[D] * 7, None, 0, None) == fs.EINVAL
    assert L.fsched_attend4_workspace(ref(p), ref(c), None) == fs.EINVAL
    assert L.fsched_attend_weight(None, ref(k), *[D] * 6, 128, None, 0, None) == fs.EINVAL
    assert L.fsched_attend4_weight(ref(p), None, *[D] * 6, 128, None, 0, None) == fs.EINVAL
    assert L.fsched_attend_weight_workspace(ref(p), ref(k), None) == fs.EINVAL
    assert L.fsched_kv_evict(None, *[D] * 9, None, 0, None) == fs.EINVAL
    assert L.fsched_kv_evict_workspace(None, ref(x)) == fs.EINVAL


def test_binding_refuses():
    import torch
    i = torch.zeros(4, dtype=torch.int32)
    x = torch.zeros(4, 8, 64, dtype=torch.bfloat16)
    f = torch.zeros(4, 16)
    c = torch.zeros(2, 2, 1, 17 * 64, dtype=torch.uint8)
    kv = torch.zeros(2, 2, 16, 64, dtype=torch.bfloat16)
    lse = torch.zeros(4, 8)
    calls = [lambda: fs.qk_norm_rope4(x, i, i, None, c), lambda: fs.kv4_read(c, i),
             lambda: fs.attend4(x, c, i.view(4, 1), i, i),
             lambda: fs.attend4_weight(x, lse, c, i.view(4, 1), i, i, f),
             lambda: fs.attend_weight(x, lse, kv, i.view(4, 1), i, i, f),
             lambda: fs.kv_evict(f, i, i.view(4, 1), i, page_size=16)]
    for call in calls:  # nothing is on the GPU
        with pytest.raises(ValueError, match="GPU tensor"):
            call()
    with pytest.raises(ValueError, match="dtype"):
        fs.kv4_read(c, i, dtype=torch.float32)
    for page in (8, 24 + 1):
        with pytest.raises(ValueError, match="16"):
            fs.kv4_cache(3, 2, page, 64, device="cpu")
    assert fs.kv4_cache(3, 2, 32, 128, device="cpu").shape == (3, 2, 2, 17 * 128)
    m = torch.zeros(2, 2, 1, 17 * 64, dtype=torch.uint8, device="meta")
    with pytest.raises(ValueError, match="one GPU"):
        fs.attend4(x, m, i.view(4, 1), i, i)


def test_binding_refuses_streams_and_what_is_no_tensor():
    import types

    import torch
    other = types.SimpleNamespace(device=torch.device("cuda", 1))
    i = torch.zeros(4, dtype=torch.int32)
    kv = torch.zeros(2, 2, 16, 64, dtype=torch.bfloat16)

    def calls(first, **kw):
        return [lambda: fs.qk_norm_rope4(first, i, i, None, i, **kw),
                lambda: fs.kv4_read(first, i, **kw), lambda: fs.attend4(first, i, i, i, i, **kw),
                lambda: fs.attend_weight(first, i, kv, i, i, i, i, **kw),
                lambda: fs.attend4_weight(first, i, i, i, i, i, i, **kw),
                lambda: fs.kv_evict(first, i, i, i, page_size=16, **kw)]
    for call in calls(i, stream=other):
        with pytest.raises(ValueError, match="stream is on cuda:1"):
            call()
    for first in ([0, 0], None, 7):
        for call in calls(first):
            with pytest.raises(ValueError, match="must be a"):
                call()


@pytest.mark.parametrize("page", [0, -16, 8, 48, 80, 96, 131072])
def test_cache_of_pages_that_every_call_refuses_is_not_made(page):
    with pytest.raises(ValueError, match="power of two"):
        fs.kv4_cache(3, 2, page, 64, device="cpu")
    for page in (16, 64, 65536):
        assert fs.kv4_cache(1, 1, page, 64, device="cpu").shape == (1, 1, page // 16, 17 * 64)


@pytest.mark.parametrize("page,width,alone", [(16, 200, True), (1, 4096, True), (1, 4097, False),
                                              (16, 2048, True), (16, 2049, False), (8, 0, True)])
def test_evict_workspace_is_what_the_call_uses(page, width, alone):
    """The freed ids (4 bytes a page) and their number; rows that no single block holds have
    scores and places beside them (12 bytes a page)."""
    p = step.EvictParams(n_req=500, table_width=width, page_size=page, flags=DEV,
                         weight_stride=width * page)
    x = ctypes.c_int64()
    assert fs.lib().fsched_kv_evict_workspace(ref(p), ref(x)) == fs.OK
    need = 500 * (width * (4 if alone else 16) + 4)
    assert need <= x.value < need + 4 * 256
