"""What the binding of the step operators refuses before it calls the library, without a
GPU."""
import os
import shutil
import subprocess
import sys
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


def test_without_the_binding_the_package_says_so_and_hasattr_answers(tmp_path):
    """A copy of the package without _step.so: the evaluation calls are there, the step
    operators are missing attributes whose message names the cause."""
    copy = tmp_path / "paper_2608_02244_amd"
    copy.mkdir()
    for name in ("__init__.py", "step.py"):
        shutil.copy(os.path.join(os.path.dirname(fs.__file__), name), copy)
    code = ("import paper_2608_02244_amd as fs\n"
            "assert fs.__file__.startswith(%r), fs.__file__\n"
            "assert hasattr(fs, 'simulate') and not hasattr(fs, 'attend')\n"
            "try: fs.kv_layout\n"
            "except AttributeError as e: assert '_step.so is not built' in str(e), e\n"
            "else: raise AssertionError\n"
            "try: from paper_2608_02244_amd import step\n"
            "except RuntimeError as e: assert '_step.so is not built' in str(e), e\n"
            "else: raise AssertionError\n" % str(tmp_path))
    r = subprocess.run([sys.executable, "-c", code], cwd=tmp_path, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
