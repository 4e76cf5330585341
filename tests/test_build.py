"""The C library is built and installed whatever becomes of the tensor binding (no compiler runs here)."""
import os
import sys

import pytest

from paper_2608_16354_amd import build as B


@pytest.fixture
def tree(tmp_path, monkeypatch):
    """Places of their own for what is built, and a compiler that writes its output file."""
    for name, at in (("BUILD", "objects"), ("LIB", "lib.so"), ("BINDING", "binding.so")):
        monkeypatch.setattr(B, name, str(tmp_path / at))
    done, broken = [], []

    def run(cmd):
        out = cmd[cmd.index("-o") + 1]
        done.append(os.path.basename(out))
        if any(b in out for b in broken):
            raise RuntimeError("build step failed: " + out)
        with open(out, "w") as f:
            f.write("new")
        return ""

    monkeypatch.setattr(B, "_run", run)
    return done, broken


def held(path):
    with open(path) as f:
        return f.read()


def test_both_are_built(tree):
    assert B.build() == B.LIB
    assert held(B.LIB) == held(B.BINDING) == "new"
    assert sorted(tree[0]) == sorted([f + ".o" for f in B.sources()] + ["lib.so.tmp", "binding.so.tmp"])


def test_a_binding_that_fails_leaves_the_library(tree):
    with open(B.BINDING, "w") as f:
        f.write("of another library")
    tree[1].append("binding.so")
    with pytest.raises(RuntimeError, match="binding.so.tmp") as e:
        B.build()
    assert held(B.LIB) == "new" and not os.path.exists(B.BINDING)
    assert "the library is built" in str(e.value)


def test_without_torch_the_library_is_built(tree, monkeypatch, capsys):
    monkeypatch.setitem(sys.modules, "torch", None)         # what an import of a missing package meets
    assert B.build() == B.LIB
    assert held(B.LIB) == "new" and not os.path.exists(B.BINDING)
    assert "torch" in capsys.readouterr().err


def test_a_library_that_fails_is_not_installed(tree):
    tree[1].append("api.cpp.o")
    with pytest.raises(RuntimeError, match="api.cpp.o"):
        B.build()
    assert not os.path.exists(B.LIB)
