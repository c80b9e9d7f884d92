"""CPU tests: where what _encoder.so needs is missing, build() still builds librcd.so, says so and leaves no module of another build;
where it is there and does not compile, build() raises."""
import os
import stat
import sys

import pytest

from paper_2211_00839_amd import build


@pytest.fixture
def place(tmp_path, monkeypatch):
    """build() into tmp_path with compilers that only write what they are asked for."""
    def compiler(name, status=0):
        path = tmp_path / name
        path.write_text('#!/bin/sh\nwhile [ $# -gt 0 ]; do if [ "$1" = -o ]; then echo %s > "$2"; fi; shift; done\nexit %d\n' % (name, status))
        path.chmod(path.stat().st_mode | stat.S_IXUSR)
        return str(path)

    monkeypatch.setenv("HIPCC", compiler("hipcc"))
    monkeypatch.setenv("CXX", compiler("cxx"))
    monkeypatch.setattr(build, "HERE", str(tmp_path))
    monkeypatch.setattr(build, "LIB", str(tmp_path / "librcd.so"))
    monkeypatch.setattr(build, "MARSHAL", str(tmp_path / "_encoder.so"))
    return tmp_path, compiler


def test_everything_there(place):
    here, _ = place
    build.build()
    assert (here / "librcd.so").read_text() == "hipcc\n" and (here / "_encoder.so").read_text() == "cxx\n"


@pytest.mark.parametrize("what", ["compiler", "torch", "headers"])
def test_the_library_alone(place, what, monkeypatch, capsys):
    here, _ = place
    (here / "_encoder.so").write_text("of another build\n")
    if what == "compiler":
        monkeypatch.setenv("CXX", str(here / "no-such-compiler"))
    elif what == "torch":
        monkeypatch.setitem(sys.modules, "torch", None)
    else:
        monkeypatch.setattr(build.sysconfig, "get_path", lambda name: str(here))
    assert build.build() == str(here / "librcd.so")
    assert (here / "librcd.so").read_text() == "hipcc\n" and not (here / "_encoder.so").exists()
    assert "_encoder.so is not built" in capsys.readouterr().err
    assert not [f for f in os.listdir(here) if ".tmp." in f]


def test_what_does_not_compile_raises(place, monkeypatch):
    here, compiler = place
    monkeypatch.setenv("CXX", compiler("broken", 1))
    with pytest.raises(RuntimeError):
        build.build()
    assert not (here / "_encoder.so").exists() and not [f for f in os.listdir(here) if ".tmp." in f]
