"""The build's own logic, with a stand-in for nvcc and for the extension's compiler: the library does not wait for torch's headers or g++."""
import os
import sys

import pytest

from paper_2008_11343_b200 import build as b


@pytest.fixture
def place(tmp_path, monkeypatch):
    """Outputs in a folder of their own; an nvcc that writes what -o names, and fails while `broken` exists."""
    nvcc = tmp_path / "nvcc"
    nvcc.write_text(f'#!/bin/sh\nif [ -e {tmp_path}/broken ]; then echo no; exit 1; fi\nwhile [ "$1" != -o ]; do shift; done\necho made > "$2"\n')
    nvcc.chmod(0o755)
    monkeypatch.setenv("NVCC", str(nvcc))
    for name, file in (("LIB", "libapms.so"), ("LIB_CHECKED", "libapms_checked.so"), ("EXT", "_operators.so"), ("BUILD", "_build"), ("EXT_FOR", "_build/for.txt")):
        monkeypatch.setattr(b, name, str(tmp_path / file))
    monkeypatch.setattr(b, "_extension_command", lambda out: ["sh", "-c", f"echo made > {out}"])
    return tmp_path


def left_over(place):
    return [f for _, _, files in os.walk(place) for f in files if ".tmp" in f]


def test_everything_is_built_once(place):
    assert b.is_stale() and b.build() == b.LIB
    assert os.path.exists(b.LIB) and os.path.exists(b.EXT) and not b.is_stale() and not left_over(place)
    (place / "broken").write_text("")
    assert b.build() == b.LIB                                                # nothing is compiled again
    with pytest.raises(RuntimeError, match="nvcc failed building apms"):
        b.build(force=True)
    assert not left_over(place)


def no_torch(out):
    raise ImportError("No module named 'torch'")


@pytest.mark.parametrize("command,words", [
    (no_torch, "No module named 'torch'"),
    (lambda out: ["/nowhere/g++"], "/nowhere/g++"),
    (lambda out: ["sh", "-c", "echo wrong; exit 1"], "g++ failed building _operators.so"),
])
def test_the_library_is_there_without_the_extension(place, monkeypatch, capsys, command, words):
    b.build()
    os.remove(b.LIB)
    monkeypatch.setattr(b, "_extension_command", command)
    capsys.readouterr()
    assert b.build(force=True) == b.LIB and os.path.exists(b.LIB)
    said = capsys.readouterr().err
    assert words in said and "_operators.so is not built" in said and "nvcc" not in said
    assert not os.path.exists(b.EXT) and b.is_stale() and not left_over(place)            # no older extension stays
    assert b.build(checked=True) == b.LIB_CHECKED and not b.is_stale(b.LIB_CHECKED)       # which needs none


def test_another_torch_means_another_extension(place, monkeypatch):
    b.build()
    monkeypatch.setattr(b, "_torch_version", lambda: "99.0")
    before = os.stat(b.LIB).st_mtime_ns
    assert b.is_stale()
    b.build()
    assert not b.is_stale() and os.stat(b.LIB).st_mtime_ns == before                       # the library is left alone


def test_the_extension_without_a_library_fails(place, monkeypatch):
    """nvcc's failure is nvcc's, and the extension's compiler does not outlive it."""
    (place / "broken").write_text("")
    monkeypatch.setattr(b, "_extension_command", lambda out: ["sh", "-c", f"sleep 60; echo made > {out}"])
    with pytest.raises(RuntimeError, match="nvcc failed"):
        b.build()
    assert not os.path.exists(b.EXT) and not left_over(place)


def test_the_real_extension_is_built_for_this_torch():
    import torch

    b.build()
    with open(b.EXT_FOR) as f:
        assert f.read() == f"torch {torch.__version__}, python {sys.version_info.major}.{sys.version_info.minor}\n"
