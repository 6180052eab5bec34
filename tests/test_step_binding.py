"""What the binding of the step operators refuses before it calls the library, without a
GPU."""
import types

import pytest
import torch

import paper_2608_02244_amd as fs


def calls(first, **kw):
    """Every operator with ``first`` as its first argument, the others on the CPU."""
    i = torch.zeros(4, dtype=torch.int32)
    kv = torch.zeros(2, 2, 16, 64, dtype=torch.bfloat16)
    return [lambda: fs.kv_layout(first, i, i.view(4, 1), i, page_size=16, n_tok=4, **kw),
            lambda: fs.qk_norm_rope(first, i, i, None, kv, kv, **kw),
            lambda: fs.attend(first, kv, kv, i.view(4, 1), i, i, **kw),
            lambda: fs.attend_shared(first, kv, kv, i, 1, i.view(4, 1), i, i, **kw)]


def test_a_stream_of_another_device_is_refused():
    """It was made current on its own device, and the call ran on whatever stream was
    current on the tensors'."""
    other = types.SimpleNamespace(device=torch.device("cuda", 1))
    for call in calls(torch.zeros(4, dtype=torch.int32), stream=other):
        with pytest.raises(ValueError, match="stream is on cuda:1"):
            call()


def test_a_first_argument_that_is_no_tensor_is_refused_like_the_others():
    for first in ([0, 0, 0, 0], None, 7):
        for call in calls(first):
            with pytest.raises(ValueError, match="must be a"):
                call()
