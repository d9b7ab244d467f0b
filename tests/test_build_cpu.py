"""What the build needs: the C library neither torch nor its headers."""
import sys

import pytest

from paper_2505_15112_amd import build as B


@pytest.fixture
def linked(monkeypatch, tmp_path):
    """Compiles and links nothing; the libraries that would be linked."""
    out = []
    monkeypatch.setattr(B, "BUILD", str(tmp_path / "objects"))
    monkeypatch.setattr(B, "_compile", lambda src, *rest: src + ".o")
    monkeypatch.setattr(B, "_link", lambda objs, lib, *rest: out.append(lib))
    return out


def test_without_torch_the_c_library_is_built(linked, monkeypatch, capsys):
    monkeypatch.setitem(sys.modules, "torch", None)  # its import fails
    assert B.build() == B.LIB
    assert linked == [B.LIB, B.LIB_ADV]
    assert "torch" in capsys.readouterr().err


def test_a_binding_that_does_not_compile_comes_after_the_c_library(linked, monkeypatch):
    def fail(verbose):
        raise RuntimeError("no Python.h")

    monkeypatch.setattr(B, "_torch_args", fail)
    with pytest.raises(RuntimeError, match="Python.h"):
        B.build()
    assert linked == [B.LIB, B.LIB_ADV]
