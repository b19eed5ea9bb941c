"""What a build leaves where a part of it cannot be done, with stand-ins for the compilers."""
import os

import pytest

from paper_2608_24738_amd import build

COMPILER = """#!/bin/sh
while [ $# -gt 0 ]; do
  if [ "$1" = -o ]; then echo made > "$2"; fi
  shift
done
exit %d
"""


@pytest.fixture
def place(tmp_path, monkeypatch):
    def compiler(name, status):
        path = tmp_path / name
        path.write_text(COMPILER % status)
        path.chmod(0o755)
        monkeypatch.setenv({"hipcc": "HIPCC", "cxx": "CXX"}[name], str(path))
    monkeypatch.setattr(build, "LIB", str(tmp_path / "lib.so"))
    monkeypatch.setattr(build, "TORCH_OPS", str(tmp_path / "ops.so"))
    monkeypatch.setattr(build, "_torch_flags", lambda: ([], []))
    compiler("hipcc", 0)
    compiler("cxx", 0)
    return tmp_path, compiler, lambda: sorted(p.name for p in tmp_path.iterdir() if p.name not in ("hipcc", "cxx"))


def test_both(place):
    _, _, made = place
    assert build.build() == build.LIB and made() == ["lib.so", "ops.so"]


def test_the_library_needs_no_torch(place, monkeypatch):
    def none():
        raise ImportError("no torch here")
    _, _, made = place
    monkeypatch.setattr(build, "_torch_flags", none)
    with pytest.raises(RuntimeError, match="_torch_ops"):
        build.build()
    assert made() == ["lib.so"]


def test_the_library_needs_no_host_compiler(place, monkeypatch):
    tmp_path, compiler, made = place
    compiler("cxx", 1)
    with pytest.raises(RuntimeError, match="compiling _torch_ops"):
        build.build()
    monkeypatch.setenv("CXX", str(tmp_path / "nothing"))
    with pytest.raises(RuntimeError, match="_torch_ops"):
        build.build()
    assert made() == ["lib.so"]


def test_without_hipcc_there_is_nothing(place):
    _, compiler, made = place
    compiler("hipcc", 1)
    with pytest.raises(RuntimeError, match="compiling libtm_edt"):
        build.build()
    assert made() == []


def test_another_torch_makes_its_functions_stale(place, monkeypatch):
    build.build()
    monkeypatch.setattr(build, "DEPS", [])
    made = os.path.getmtime(build.TORCH_OPS)
    monkeypatch.setattr(build, "_torch_changed", lambda: made - 1)
    assert not build.is_stale()
    monkeypatch.setattr(build, "_torch_changed", lambda: made + 1)
    assert build.is_stale()


def test_when_torch_changed():
    assert build._torch_changed() > 0
