"""The build of the native libraries: what it needs, and what the compiler may not warn
about (the compilers themselves run in ``__graft_entry__.build()``)."""
import os
import re
import subprocess
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


def test_direct_loads_to_lds_keep_the_compiler_s_registers(tmp_path):
    """The loads take their LDS address from m0, a reserved register: naming it as
    clobbered is not honoured (the compiler warns), so they have to put it back."""
    src = tmp_path / "loads.hip"
    src.write_text('''#include "attend_tiles.hpp"
__global__ void two_loads(const char* p, unsigned off, unsigned base) {
  fs::load_to_lds(p + threadIdx.x * 16, base);
  fs::load_to_lds(p, off + threadIdx.x * 16, base + 1024);
  fs::wait_loads();
}
''')
    out = tmp_path / "loads.s"
    r = subprocess.run([buildlib._hipcc(), *buildlib.COMMON, "-Werror=inline-asm", "-x", "hip",
                        "--cuda-device-only", "-S", str(src), "-o", str(out)],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    writes = [x.split() for x in out.read_text().splitlines() if "s_mov_b32" in x and "m0" in x]
    saved = [x[1].strip(",") for x in writes if x[2] == "m0"]
    put_back = [x[2] for x in writes if x[1] == "m0,"]
    assert len(saved) == 2 and put_back[1::2] == saved


@pytest.mark.parametrize("wide", ["true", "false"])
def test_decode_kernels_of_heads_of_256_keep_their_registers(tmp_path, wide):
    """Bound by the cache's bytes, they have none to spare for scratch."""
    src = tmp_path / "rows.hip"
    src.write_text(f'''#include "attend_main.hpp"
template __global__ void fs::attend_rows_kernel<fs::Bf16, 256, 1, {wide}>(fs::AttnArgs, fs::MainPlan);
template __global__ void fs::attend_rows_kernel<fs::F16, 256, 1, {wide}>(fs::AttnArgs, fs::MainPlan);
''')
    r = subprocess.run([buildlib._hipcc(), *buildlib.COMMON, "-Rpass-analysis=kernel-resource-usage",
                        "-x", "hip", "--cuda-device-only", "-c", str(src), "-o",
                        str(tmp_path / "rows.o")], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    scratch = re.findall(r"ScratchSize \[bytes/lane\]: (\d+)", r.stderr)
    assert scratch == ["0", "0"]
