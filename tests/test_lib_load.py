"""A library that lacks an entry point of this package is refused when it is
loaded, not when the entry point is first called."""
import os
import subprocess

import pytest

from paper_2607_00760_amd import _lib


def library(path, names):
    src = path.with_suffix(".c")
    src.write_text("".join(f"int {n}(void) {{ return 0; }}\n" for n in names))
    subprocess.run(["gcc", "-shared", "-fPIC", "-w", "-o", str(path), str(src)], check=True)
    return str(path)


@pytest.mark.parametrize("lost", ["mosaic_quant_append", "mosaic_qk_norm_rope", "mosaic_decode_attention"])
def test_missing_entry_point(tmp_path, monkeypatch, lost):
    monkeypatch.setattr(_lib, "_lib", None)
    monkeypatch.setattr(_lib, "LIB_PATH", library(tmp_path / "stale.so", [n for n in _lib.EXPORTED if n != lost]))
    with pytest.raises(ImportError, match=lost):
        _lib.load()
    assert _lib._lib is None


def test_whole_library(tmp_path, monkeypatch):
    monkeypatch.setattr(_lib, "_lib", None)
    monkeypatch.setattr(_lib, "LIB_PATH", library(tmp_path / "whole.so", _lib.EXPORTED))
    assert _lib.load() is _lib.load()


def test_no_library(tmp_path, monkeypatch):
    monkeypatch.setattr(_lib, "_lib", None)
    monkeypatch.setattr(_lib, "LIB_PATH", os.path.join(tmp_path, "none.so"))
    with pytest.raises(ImportError, match="missing"):
        _lib.load()
