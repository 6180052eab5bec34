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
