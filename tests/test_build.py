"""What building needs and when it is done again: stand-ins for the compilers, files of a folder of the test's own."""
import os
import stat
import sys

import pytest

from paper_2609_21264_b200 import binding, build


def script(path, text):
    path.write_text("#!/bin/sh\n" + text)
    path.chmod(path.stat().st_mode | stat.S_IXUSR)
    return str(path)


# a compiler that writes a line into a log and its output file
WRITES = 'echo "%s" >> "%s"\nwhile [ $# -gt 0 ]; do if [ "$1" = "-o" ]; then echo built > "$2"; fi; shift; done\n'


@pytest.fixture
def files(tmp_path, monkeypatch):
    """The library, the extension module and the log of what was compiled."""
    log = tmp_path / "log"
    log.write_text("")
    for name, file in (("LIB_PATH", "lib.so"), ("CALLS_PATH", "calls.so"), ("CALLS_BUILT_FOR", "calls.built")):
        monkeypatch.setattr(build, name, str(tmp_path / file))
    nvcc = script(tmp_path / "nvcc", WRITES % ("library", log))
    monkeypatch.setattr(build, "_nvcc", lambda: nvcc)
    monkeypatch.setenv("CXX", script(tmp_path / "cxx", WRITES % ("calls", log)))
    return tmp_path / "lib.so", tmp_path / "calls.so", lambda: log.read_text().split()


def test_both_are_built_once(files):
    lib, calls, log = files
    assert build.build() == str(lib) and lib.exists() and calls.exists() and log() == ["library", "calls"]
    build.build()
    assert log() == ["library", "calls"]
    build.build(force=True)
    assert log() == ["library", "calls"] * 2


def test_the_library_needs_no_torch(files, monkeypatch):
    lib, calls, log = files
    monkeypatch.setitem(sys.modules, "torch", None)            # (an import of it raises)
    with pytest.warns(UserWarning, match="torch"):
        assert build.build() == str(lib)
    assert lib.exists() and not calls.exists() and log() == ["library"]
    with pytest.warns(UserWarning, match="torch"):             # and where nothing is left to compile
        assert build.build() == str(lib)
    assert log() == ["library"]


def test_the_library_is_there_where_the_module_cannot_be_built(files, monkeypatch, tmp_path):
    lib, calls, log = files
    for cxx in (script(tmp_path / "fails", "echo no >&2\nexit 1\n"), str(tmp_path / "not_there")):
        monkeypatch.setenv("CXX", cxx)
        with pytest.raises(RuntimeError, match=os.path.basename(cxx)):
            build.build(force=True)
        assert lib.exists() and not calls.exists()
    assert log() == ["library"] * 2


def test_the_module_is_built_again_for_another_torch_or_python(files, monkeypatch):
    import torch
    lib, calls, log = files
    build.build()
    with monkeypatch.context() as m:
        m.setattr(torch, "__version__", "0.0.1")
        assert build.calls_mismatch()
        build.build()
        assert log() == ["library", "calls", "calls"] and not build.calls_mismatch()
    soabi = build.sysconfig.get_config_var
    with monkeypatch.context() as m:
        m.setattr(build.sysconfig, "get_config_var", lambda name: "cpython-1" if name == "SOABI" else soabi(name))
        build.build()
        assert log() == ["library"] + ["calls"] * 3
    assert "cpython-1" in build.calls_mismatch()
    build.build()
    assert log() == ["library"] + ["calls"] * 4 and build.calls_mismatch() == ""


def test_a_module_of_another_torch_is_not_loaded(files, monkeypatch):
    build.build()
    monkeypatch.setattr(binding, "load", lambda: None)         # (the stand-in is no library)
    with open(build.CALLS_BUILT_FOR, "w") as f:
        f.write("cpython-1, torch 0.0.1")
    with pytest.raises(ImportError, match="torch 0.0.1.*paper_2609_21264_b200.build"):
        binding._native()
