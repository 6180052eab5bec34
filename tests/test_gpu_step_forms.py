"""Forms of the step operators beyond those of test_gpu_step_operators.py, against the same
64-bit references and tolerances, and what the binding refuses with GPU tensors in hand."""
import pytest

import paper_2608_02244_amd as fs
from test_gpu_step_operators import Batch, dev, log  # noqa: F401 (dev: fixture)

pytestmark = pytest.mark.gpu


def test_out_of_memory_is_torch_s_error(dev):
    """An output of 8 TiB, of queries that take 512 bytes: nothing is launched."""
    import torch
    q = torch.zeros(1, 1, 256, dtype=torch.bfloat16, device=dev).expand(1 << 24, 1024, 256)
    kv = torch.zeros(1, 1, 16, 256, dtype=torch.bfloat16, device=dev)
    i = torch.zeros(2, dtype=torch.int32, device=dev)
    log("attend, an output of 8 TiB")
    with pytest.raises(torch.OutOfMemoryError):
        fs.attend(q, kv, kv, i[:1].view(1, 1), i, i[:1])


def test_expanded_tensors_are_read_but_not_written(dev):
    """Rows that share memory would be written by several waves at once."""
    import torch
    b = Batch(dev, [1, 1, 2], [5, 40, 17], 8, 2, 64)
    one = torch.zeros(1, 8, 64, dtype=torch.bfloat16, device=dev)
    with pytest.raises(ValueError, match="out is written"):
        b.call(out=one.expand(4, 8, 64))
    with pytest.raises(ValueError, match="out is written"):
        b.call(out=one[:, :1].expand(4, 8, 64))
    qkv = torch.randn(4, 12, 64, device=dev).bfloat16()
    slots = torch.arange(4, dtype=torch.int32, device=dev)
    kv = [torch.zeros(2, 2, 16, 64, device=dev).bfloat16() for _ in range(2)]
    with pytest.raises(ValueError, match="out is written"):
        fs.qk_norm_rope(qkv, None, None, None, *kv, out=one.expand(4, 8, 64))
    for i, name in enumerate(("k_cache", "v_cache")):
        bad = list(kv)
        bad[i] = kv[i][:, :1].expand(2, 2, 16, 64)
        with pytest.raises(ValueError, match=name + " is written"):
            fs.qk_norm_rope(qkv, None, slots, None, *bad)
        fs.qk_norm_rope(qkv, None, None, None, *bad)  # nothing is stored
    # read they may be: one token's queries for all, one key head's keys for both
    same = b.args[0][:1].expand(4, 8, 64)
    k = b.args[1][:, :1].expand(b.args[1].shape)
    got = fs.attend(same, k, *b.args[2:], scale=b.scale, max_q=2)
    want = fs.attend(same.contiguous(), k.contiguous(), *b.args[2:], scale=b.scale, max_q=2)
    assert torch.equal(got, want)


DRAFTS = ([1, 2, 3, 4, 1, 4, 0, 3], [1, 16, 17, 40, 90, 6, 0, 129])  # new and held tokens


@pytest.mark.parametrize("heads", [(8, 1), (64, 8), (7, 1)], ids=lambda h: f"{h[0]}x{h[1]}")
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("page,dt", [(1, "bf16"), (8, "f16"), (8, "bf16"), (16, "f16"),
                                     (16, "bf16")])
def test_drafts_of_17_to_32_rows(dev, heads, D, page, dt):
    """Two row tiles per request and key head, alone and beside the blocks over a prefix."""
    new, own = DRAFTS
    Batch(dev, new, own, *heads, D, dt, page=page, seed=page).check()
    Batch(dev, new, own, *heads, D, dt, page=page, prefix=70, seed=page).check()
    Batch(dev, new, own, *heads, D, dt, page=page, prefix=70, window=50, sinks=3,
          seed=page).check()


@pytest.mark.parametrize("heads", [(17, 1), (24, 1), (64, 2)], ids=lambda h: f"{h[0]}x{h[1]}")
@pytest.mark.parametrize("D,dt", [(64, "bf16"), (128, "f16"), (256, "bf16"), (256, "f16")])
@pytest.mark.parametrize("page", [4, 16])
def test_17_to_32_query_heads_per_key_head(dev, heads, D, dt, page):
    """One token fills two row tiles (or, with heads of 256, a block of the tiles kind);
    prompts beside decoding requests, with and without a prefix."""
    for new, own in (([1] * 5 + [0, 1], [1, 31, 32, 200, 3, 0, 0]), ([1, 20, 1, 2], [64, 33, 5, 9])):
        Batch(dev, new, own, *heads, D, dt, page=page, seed=D).check()
        Batch(dev, new, own, *heads, D, dt, page=page, prefix=33, seed=D).check()


@pytest.mark.parametrize("page", [1, 8, 64])
@pytest.mark.parametrize("heads", [(8, 1), (4, 4), (10, 2)], ids=lambda h: f"{h[0]}x{h[1]}")
def test_heads_of_256_in_f16(dev, page, heads):
    for new, own, prefix in (([1] * 6, [1, 2, 31, 33, 129, 450], 0),
                             ([2, 3, 4, 1], [2, 50, 4, 9], 0), ([70, 1, 33], [70, 300, 65], 0),
                             ([1, 2, 40, 1], [5, 40, 60, 0], 100)):
        Batch(dev, new, own, *heads, 256, "f16", page=page, prefix=prefix, seed=page).check()
    Batch(dev, [1, 4, 60], [300, 90, 200], *heads, 256, "f16", page=page, window=64, sinks=5,
          seed=page).check()


@pytest.mark.parametrize("n,prefix", [(300, 0), (300, 21), (700, 0)])
def test_tiles_of_more_requests_than_threads(dev, n, prefix):
    """The search for a block's tile goes over several requests per thread: lengths from
    none to 70 new tokens, held ones over all of the eight classes of work."""
    new = [(0, 1, 9, 1, 2, 1, 17, 1, 1, 70 if i % 3 == 0 else 1)[i % 10] for i in range(n)]
    own = [m + (37 * i) % (40 if i % 7 else 900) for i, m in enumerate(new)]
    Batch(dev, new, own, 4, 1, 64, prefix=prefix, seed=n).check()


def test_tokens_past_max_q_are_not_computed(dev):
    """The others are, at their own positions, and hold the tolerances; out and lse of the
    tokens past max_q stay as they were."""
    import ctypes

    import torch
    from paper_2608_02244_amd import step
    for max_q, new, own in ((1, [1, 3, 1, 40], [20, 30, 5, 60]), (20, [1, 60, 4, 21], [9, 99, 7, 21])):
        b = Batch(dev, new, own, 8, 2, 64)
        ro, rl, to, tl = b.reference()
        computed = torch.cat([torch.arange(m) < max_q for m in new])
        q, k, v, table, q_start, kv_len = b.args
        n = len(b.q)
        out = torch.full_like(q, 5.0)
        lse = torch.full((n, 8), 7.0, device=dev)
        c = step.KvCache(k=k.data_ptr(), v=v.data_ptr(), n_pages=k.shape[0], page_size=16,
                         kv_heads=2, head_dim=64, dtype=0, k_stride=k.stride()[:3],
                         v_stride=v.stride()[:3])
        p = step.AttnParams(n_req=len(new), n_tok=n, q_heads=8, max_q=max_q,
                            table_width=table.shape[1], scale=b.scale,
                            flags=fs.F_DEVICE_PTRS | fs.F_SYNC, q_token_stride=q.stride(0),
                            q_head_stride=q.stride(1), out_token_stride=out.stride(0),
                            out_head_stride=out.stride(1))
        log(f"attend new={new} own={own} max_q={max_q}")
        torch.cuda.synchronize()
        assert fs.lib().fsched_attend(ctypes.byref(p), ctypes.byref(c), *[x.data_ptr() for x in (
            q, table, q_start, kv_len, out, lse)], None, 0, None) == fs.OK
        out, lse = out.double().cpu(), lse.double().cpu()
        assert ((out - ro).abs() <= to)[computed].all()
        assert ((lse - rl).abs() <= tl)[computed].all()
        assert (out[~computed] == 5.0).all() and (lse[~computed] == 7.0).all()


def test_workspace_that_is_too_small_is_refused(dev):
    import torch
    b = Batch(dev, [1] * 20 + [50, 1], [37 * i % 900 + 1 for i in range(20)] + [800, 3], 16, 2, 128)
    ws = fs.attend_workspace(len(b.q), len(b.own), 16, 2, 128, page_size=16,
                             table_width=b.table.shape[1], max_q=50)
    assert ws.numel() > 256
    for room in (ws[:256], ws[:-1].clone(), torch.empty(0, dtype=torch.uint8, device=dev)):
        with pytest.raises(fs.FschedError) as e:
            b.call(workspace=room)
        assert e.value.code == fs.ESCRATCH
    out, _ = b.call()
    got, _ = b.call(workspace=ws)
    assert torch.equal(out, got)
