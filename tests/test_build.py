"""The build: the library wants nvcc alone, the binding is left out where its prerequisites are missing and is rebuilt (or refused)
when it was made against another torch."""
import os
import subprocess

import pytest

from paper_2609_19758_b200 import attention as A
from paper_2609_19758_b200 import build as B


@pytest.mark.parametrize("missing", ["g++", "torch's headers", "Python.h"])
def test_the_library_is_built_without_the_binding_s_prerequisites(monkeypatch, tmp_path, capsys, missing):
    commands = []

    def run(cmd, **kw):
        commands.append(cmd)
        return subprocess.CompletedProcess(cmd, 0, "", "")

    monkeypatch.setattr(B.subprocess, "run", run)
    monkeypatch.setattr(B, "LIB", str(tmp_path / "libfpsk.so"))
    monkeypatch.setattr(B, "BINDING", str(tmp_path / "_binding.so"))
    if missing == "g++":
        which = B.shutil.which
        monkeypatch.setattr(B.shutil, "which", lambda name: None if name == "g++" else which(name))
    elif missing == "Python.h":
        monkeypatch.setattr(B.sysconfig, "get_paths", lambda: {"include": str(tmp_path)})
    else:
        exists = os.path.exists
        monkeypatch.setattr(B.os.path, "exists", lambda p: False if str(p).endswith("python_variable.h") else exists(p))
    assert B.build() == B.LIB
    assert len(commands) == len(B.sources()) + 1 and all("nvcc" in c[0] for c in commands)
    assert missing in capsys.readouterr().err


def test_the_library_comes_before_the_binding(monkeypatch, tmp_path):
    order = []
    monkeypatch.setattr(B, "LIB", str(tmp_path / "libfpsk.so"))
    monkeypatch.setattr(B, "_build_library", lambda out, verbose, bounds: order.append("library"))
    monkeypatch.setattr(B, "build_binding", lambda force: order.append("binding"))
    B.build()
    assert order == ["library", "binding"]


def test_a_binding_of_another_torch_is_told(monkeypatch, tmp_path):
    B.build()
    assert B.binding_is_current() and not B.needs_build(B.BINDING)
    other = tmp_path / "_binding.so"
    with open(B.BINDING, "rb") as f:
        other.write_bytes(f.read().replace(b"fpsk binding for torch ", b"fpsk binding for torch 0"))
    os.utime(other, (2 ** 32, 2 ** 32))          # newer than every source
    monkeypatch.setattr(B, "BINDING", str(other))
    assert not B.binding_is_current() and B.needs_build(B.BINDING)
    monkeypatch.setattr(A, "_binding", None)
    with pytest.raises(RuntimeError, match="build it again"):
        A._bind()
