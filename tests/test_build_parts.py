"""The C library is built by hipcc alone: neither a host compiler that fails nor a missing torch
keeps it from being linked."""

import os
import stat
import sys

import pytest

from paper_2608_03893_amd import build

HIPCC = """#!%s
import sys
open(sys.argv[sys.argv.index("-o") + 1], "w").write(" ".join(sys.argv[1:]))
"""


@pytest.fixture
def place(tmp_path, monkeypatch):
    """The build's paths in a folder of the test's own, with a hipcc that writes its arguments."""
    hipcc = tmp_path / "hipcc"
    hipcc.write_text(HIPCC % sys.executable)
    hipcc.chmod(hipcc.stat().st_mode | stat.S_IXUSR)
    monkeypatch.setenv("HIPCC", str(hipcc))
    for name, to in (("CSRC", "csrc"), ("LIB", "libkvx.so"), ("BIND", "_kvx_bind.so")):
        monkeypatch.setattr(build, name, str(tmp_path / to))
    (tmp_path / "csrc").mkdir()
    return tmp_path


def _broken(out):
    return ["false"]


def _no_torch(out):
    raise ImportError("No module named 'torch'")


@pytest.mark.parametrize("command", [_broken, _no_torch])
def test_the_library_is_linked_without_the_binding(place, monkeypatch, command):
    monkeypatch.setattr(build, "bind_command", command)
    with pytest.raises(RuntimeError, match="kvx_bind.cpp"):
        build.build()
    assert (place / "libkvx.so").exists() and not (place / "_kvx_bind.so").exists()


def test_both_parts_are_built(place, monkeypatch):
    monkeypatch.setattr(build, "bind_command", lambda out: [os.environ["HIPCC"], "-o", out])
    assert build.build() == str(place / "libkvx.so")
    assert (place / "libkvx.so").exists() and (place / "_kvx_bind.so").exists()
    assert sorted(os.listdir(place / "csrc")) == []


def test_a_kernel_that_does_not_compile_leaves_both_as_they_were(place, monkeypatch):
    monkeypatch.setattr(build, "bind_command", lambda out: ["sh", "-c", f": > {out}"])
    monkeypatch.setenv("HIPCC", "false")
    (place / "libkvx.so").write_text("old")
    with pytest.raises(RuntimeError, match="kvx_pages.hip"):
        build.build()
    assert (place / "libkvx.so").read_text() == "old" and not (place / "_kvx_bind.so").exists()
