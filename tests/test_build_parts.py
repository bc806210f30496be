"""The C library and the Python binding's helper are built apart: what stops the one does not stop
the other.  The compilers are stand-ins."""
import os
import subprocess
import sys
import types

import pytest

from paper_2412_06464_amd import build


@pytest.fixture
def tree(tmp_path, monkeypatch):
    """A build whose steps only write what they would make; the commands it ran."""
    lib, binding, ran = str(tmp_path / "lib.so"), str(tmp_path / "binding.so"), []
    for name, value in (("HERE", str(tmp_path)), ("LIB", lib), ("BINDING", binding)):
        monkeypatch.setattr(build, name, value)
    monkeypatch.setattr(build.build, "__defaults__", (False, lib, ()))
    monkeypatch.setattr(build.build_binding, "__defaults__", (binding,))

    def run(cmd, **kw):
        ran.append(cmd)
        fails = "broken" in cmd[0]
        if not fails:
            open(cmd[cmd.index("-o") + 1], "w").close()
        return types.SimpleNamespace(returncode=int(fails), stdout="", stderr="no\n")

    monkeypatch.setattr(subprocess, "run", run)
    return lib, binding, ran


def test_both(tree):
    build.build()
    assert os.path.exists(tree[0]) and os.path.exists(tree[1])
    assert len(tree[2]) == len(build.SOURCES) + 2


def test_without_torch(tree, monkeypatch, capsys):
    monkeypatch.setitem(sys.modules, "torch", None)  # import torch: ImportError
    assert build.build() == tree[0]
    assert os.path.exists(tree[0]) and not os.path.exists(tree[1])
    assert "no torch" in capsys.readouterr().err


def test_without_a_host_compiler(tree, monkeypatch, capsys):
    monkeypatch.setenv("CXX", "no-such-compiler")
    assert build.build() == tree[0]
    assert os.path.exists(tree[0]) and not os.path.exists(tree[1])
    assert "no-such-compiler" in capsys.readouterr().err


def test_a_binding_that_does_not_compile(tree, monkeypatch, tmp_path):
    """Is an error, of a build whose library is there."""
    cxx = tmp_path / "broken"
    cxx.write_text("")
    cxx.chmod(0o755)
    monkeypatch.setenv("CXX", str(cxx))
    with pytest.raises(RuntimeError, match="paged_binding"):
        build.build()
    assert os.path.exists(tree[0])
