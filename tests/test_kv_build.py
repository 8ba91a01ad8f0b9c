"""The libraries need hipcc alone; the Python side of include/kv.h, which needs more, does not stand in their way, and is only loaded by
the Python and torch that it was built for."""
import importlib
import os
import stat
import subprocess
import sys
import sysconfig

import pytest

from tests.test_kv_abi import ROOT, A  # noqa: F401  (A: the fixture)

_TOOL = """#!/bin/sh
# writes the name of its output into it
while [ $# -gt 0 ]; do [ "$1" = -o ] && echo made > "$2"; shift; done
"""


def _tool(path, text=_TOOL):
    path.write_text(text)
    path.chmod(path.stat().st_mode | stat.S_IXUSR)
    return str(path)


@pytest.fixture
def build(tmp_path, monkeypatch):
    """build.py with every output and tool under tmp_path."""
    import paper_2605_10905_amd.build as b

    b = importlib.reload(b)
    for name in ("LIB", "LIB_KV", "CALL_KV"):
        monkeypatch.setattr(b, name, str(tmp_path / os.path.basename(getattr(b, name))))
    monkeypatch.setattr(b, "CSRC", str(tmp_path))
    monkeypatch.setattr(b, "HERE", str(tmp_path))
    monkeypatch.setattr(b, "HIPCC", _tool(tmp_path / "hipcc"))
    bin_ = tmp_path / "bin"
    bin_.mkdir()
    for name in ("sh", "echo"):
        os.symlink(f"/bin/{name}", bin_ / name)
    _tool(bin_ / "g++")
    monkeypatch.setenv("PATH", str(bin_))
    return b


def _built(b):
    return [os.path.exists(getattr(b, name)) for name in ("LIB", "LIB_KV", "CALL_KV")]


def test_everything_is_built(build):
    assert build.build(verbose=False) == build.LIB and _built(build) == [True] * 3


def test_without_a_host_compiler_the_libraries_are_built(build, tmp_path, capsys):
    os.remove(tmp_path / "bin" / "g++")
    open(build.CALL_KV, "w").close()  # (what an earlier build left does not fit the new library)
    assert build.build(verbose=False) == build.LIB and _built(build) == [True, True, False]
    assert "g++" in capsys.readouterr().err


def test_without_torch_the_libraries_are_built(build, monkeypatch, capsys):
    monkeypatch.setitem(sys.modules, "torch", None)
    assert build.build(verbose=False) == build.LIB and _built(build) == [True, True, False]
    assert "torch" in capsys.readouterr().err


def test_without_python_headers_the_libraries_are_built(build, tmp_path, monkeypatch, capsys):
    monkeypatch.setattr(sysconfig, "get_path", lambda name: str(tmp_path / "nothing"))
    assert build.build(verbose=False) == build.LIB and _built(build) == [True, True, False]
    assert "Python.h" in capsys.readouterr().err


def test_a_source_that_does_not_compile_is_an_error_after_the_libraries(build, tmp_path):
    _tool(tmp_path / "bin" / "g++", "#!/bin/sh\necho wrong; exit 1\n")
    with pytest.raises(RuntimeError, match="wrong"):
        build.build(verbose=False)
    assert _built(build) == [True, True, False]


def test_a_kernel_that_does_not_compile_is_an_error(build, tmp_path):
    _tool(tmp_path / "hipcc", "#!/bin/sh\necho wrong; exit 1\n")
    with pytest.raises(RuntimeError, match="wrong"):
        build.build(verbose=False)


def test_the_python_side_names_its_python(A):  # noqa: F811
    call = importlib.import_module("paper_2605_10905_amd.kv")._call
    assert call.__file__.endswith(sysconfig.get_config_var("EXT_SUFFIX"))


def test_the_python_side_of_another_torch_is_refused(A):  # noqa: F811
    """Tensors are read by their layout in memory, which another torch may have changed."""
    code = "import torch; torch.__version__ = '0.0.1'; import paper_2605_10905_amd as A; A.attn_version(); A.kv_decode"
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, cwd=ROOT, timeout=120)
    assert r.returncode != 0 and "ImportError" in r.stderr and "0.0.1" in r.stderr, r.stderr[-500:]
