"""The library builds where its Python binding's compiled half cannot: no torch for ROCm, or no headers of Python's."""

import os
import sys

import pytest

from paper_2609_33601_amd import build as b


@pytest.fixture
def commands(tmp_path, monkeypatch):
    """build() with its compilers replaced by ones that only leave their output; the commands that it ran."""
    ran = []

    def run(cmd, verbose):
        ran.append(cmd)
        open(cmd[cmd.index("-o") + 1], "w").close()

    monkeypatch.setattr(b, "_run", run)
    monkeypatch.setattr(b.check_waits, "compile_and_check", lambda *a: 1)
    monkeypatch.setattr(b, "OBJ_DIR", str(tmp_path / "obj"))
    monkeypatch.setattr(b, "LIB", str(tmp_path / "libjq.so"))
    monkeypatch.setattr(b, "BINDING", str(tmp_path / "_jq_block.so"))
    return ran


def _bindings(ran):
    return [c for c in ran if any(b.BINDING_SOURCE in a for a in c)]


def test_build_with_torch(commands):
    torch = pytest.importorskip("torch")
    if torch.version.hip is None:
        pytest.skip("torch is not for ROCm")
    assert b.build() == b.LIB and os.path.exists(b.LIB)
    assert len(_bindings(commands)) == 1 and os.path.exists(b.BINDING)


@pytest.mark.parametrize("missing", ["torch", "ROCm", "Python.h"])
def test_build_without(commands, monkeypatch, capsys, missing):
    if missing == "torch":
        for name in [n for n in sys.modules if n == "torch" or n.startswith("torch.")]:
            monkeypatch.delitem(sys.modules, name)
        monkeypatch.setitem(sys.modules, "torch", None)
    elif missing == "ROCm":
        monkeypatch.setattr(pytest.importorskip("torch").version, "hip", None)
    else:
        import sysconfig

        paths = sysconfig.get_paths()
        monkeypatch.setattr(sysconfig, "get_paths", lambda *a, **k: {**paths, "include": "/nowhere"})
    open(b.BINDING, "w").close()  # of an earlier build, for an earlier library
    assert b.build() == b.LIB and os.path.exists(b.LIB)
    assert not _bindings(commands), "a binding that cannot be compiled was tried"
    assert not os.path.exists(b.BINDING), "an earlier binding stays beside a new library"
    assert missing in capsys.readouterr().out, "nothing says why"
