"""The build without what only the compiled part of the binding needs, and the binding's choice between that part and ctypes."""
import os
import subprocess
import types

import pytest

from paper_2511_09844_gb300 import build, sd2


@pytest.fixture
def compilers(monkeypatch, tmp_path):
    """A build into a folder of its own by compilers that write empty files; g++ fails for lack of a header until told otherwise."""
    state = types.SimpleNamespace(calls=[], gpp=1)

    def run(cmd, **kw):
        state.calls.append(os.path.basename(cmd[0]))
        if cmd[0] == "g++" and state.gpp:
            return subprocess.CompletedProcess(cmd, state.gpp, "", "fatal error: Python.h: No such file or directory")
        open(cmd[cmd.index("-o") + 1], "w").close()
        return subprocess.CompletedProcess(cmd, 0, "", "")
    monkeypatch.setattr(build.subprocess, "run", run)
    monkeypatch.setattr(build, "_nvcc", lambda: "/usr/local/cuda/bin/nvcc")
    monkeypatch.setattr(build, "OUT_DIR", str(tmp_path))
    monkeypatch.setattr(build, "LIB", str(tmp_path / "libsd2.so"))
    return state


def test_the_library_is_built_without_the_bindings_headers(compilers, capsys):
    assert build.build() == build.LIB and os.path.exists(build.LIB)
    assert "Python.h" in capsys.readouterr().err
    # what cannot be compiled here is not tried again for ever
    before = len(compilers.calls)
    assert not build.is_stale() and build.build() == build.LIB and len(compilers.calls) == before
    # but it is when asked for, and is then there
    compilers.gpp = 0
    build.build(force=True)
    assert os.path.exists(build.binding_path()) and not build.is_stale()
    # and a newer source is compiled again
    old = os.path.getmtime(build.LIB) - 1e6
    for f in os.listdir(build.OUT_DIR):
        os.utime(os.path.join(build.OUT_DIR, f), (old, old))
    assert build.is_stale()


def test_the_library_is_built_without_torch(compilers, monkeypatch):
    def missing(name):
        raise build.metadata.PackageNotFoundError(name)
    monkeypatch.setattr(build.metadata, "version", missing)
    assert build.binding_path() is None
    assert build.build() == build.LIB and not build.is_stale()
    assert "g++" not in compilers.calls


def test_a_library_that_fails_still_says_so(compilers, monkeypatch):
    monkeypatch.setattr(build.subprocess, "run", lambda cmd, **kw: subprocess.CompletedProcess(cmd, 1, "", "error"))
    with pytest.raises(RuntimeError, match="nvcc failed"):
        build.build()


def test_calls_go_through_ctypes_where_the_compiled_part_does_not_load(monkeypatch, tmp_path):
    build.build()
    junk = tmp_path / "sd2_binding.so"
    junk.write_bytes(b"not a library")
    monkeypatch.setattr(build, "binding_path", lambda: str(junk))
    monkeypatch.setattr(sd2, "_native", None)
    with pytest.warns(RuntimeWarning, match="sd2_binding"):
        assert sd2._connect() is False
    assert sd2._native is False


def test_a_compiled_part_of_another_torch_is_not_loaded(monkeypatch):
    build.build()
    mine = build.binding_path()
    monkeypatch.setattr(sd2, "_native", None)
    assert sd2._connect()
    monkeypatch.setattr(sd2, "_native", None)
    monkeypatch.setattr(build.metadata, "version", lambda name: "1.0.0+other")
    assert build.binding_path() != mine
    assert sd2._connect() is False
