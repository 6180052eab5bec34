"""The build of the native libraries: what it needs, and what the compiler may not warn
about (the compilers themselves run in ``__graft_entry__.build()``)."""
import os
import sys

import pytest

from paper_2608_02244_amd import buildlib


@pytest.fixture
def dry(monkeypatch, tmp_path):
    """build() with commands that only leave their output files, in a folder of its own."""
    ran = []

    def run(cmd, what):
        ran.append(cmd)
        open(cmd[cmd.index("-o") + 1], "w").close()
    monkeypatch.setattr(buildlib, "_run", run)
    monkeypatch.setattr(buildlib, "BUILD_DIR", str(tmp_path / "_build"))
    for name in ("LIB", "BIND_LIB"):
        monkeypatch.setattr(buildlib, name, str(tmp_path / os.path.basename(getattr(buildlib, name))))
    return ran


def test_build_makes_the_library_and_the_binding(dry):
    assert buildlib.build() == buildlib.LIB
    assert os.path.exists(buildlib.LIB) and os.path.exists(buildlib.BIND_LIB)


def test_build_without_torch_makes_the_library_alone(dry, monkeypatch, capsys):
    """The evaluation calls need no torch, and neither does building them; a binding that
    an earlier build left does not outlive its library."""
    open(buildlib.BIND_LIB, "w").close()
    monkeypatch.setitem(sys.modules, "torch", None)  # as if not installed
    assert buildlib.build() == buildlib.LIB
    assert os.path.exists(buildlib.LIB) and not os.path.exists(buildlib.BIND_LIB)
    assert "without the step operators" in capsys.readouterr().out


def test_binding_is_built_without_a_host_compiler(dry, monkeypatch):
    """hipcc compiles C++ as well."""
    which = buildlib.shutil.which
    monkeypatch.setattr(buildlib.shutil, "which",
                        lambda name, **kw: None if name in ("g++", "c++") else which(name, **kw))
    buildlib.build()
    bind = [c for c in dry if buildlib.BIND_SRC in c or buildlib.BIND_LIB + ".tmp" in c]
    assert len(bind) == 2 and all(c[0] == buildlib._hipcc() for c in bind)
