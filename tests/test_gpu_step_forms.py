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
