"""When _calls.so is compiled, and what becomes of a build without the headers that it alone needs (a compiler that only records stands for hipcc)."""
import os
import subprocess

import pytest

from paper_2605_06057_amd import build


@pytest.fixture
def compiled(tmp_path, monkeypatch):
    """The commands run so far; the compiler writes its output, or fails once `error` is set."""
    runs = []

    def run(cmd, **_):
        runs.append(cmd)
        if run.error:
            return subprocess.CompletedProcess(cmd, 1, "", run.error)
        open(cmd[cmd.index("-o") + 1], "w").close()
        return subprocess.CompletedProcess(cmd, 0, "", "")
    run.error = ""
    monkeypatch.setattr(build, "CALLS", str(tmp_path / "_calls.so"))
    monkeypatch.setattr(build, "GEN", str(tmp_path))
    monkeypatch.setattr(build.subprocess, "run", run)
    runs_of = lambda: runs
    runs_of.fail = lambda message: setattr(run, "error", message)
    return runs_of


def test_compiled_once_and_again_for_another_torch(compiled, monkeypatch):
    assert build._build_calls(False).startswith("compiled") and build._build_calls(False).startswith("up to date")
    assert len(compiled()) == 1 and compiled()[0][0] == build.HIPCC and os.path.exists(build.CALLS)
    monkeypatch.setattr(build, "_calls_built_for", lambda: "another torch")
    assert build._build_calls(False).startswith("compiled") and build._build_calls(False).startswith("up to date")
    assert build._build_calls(True).startswith("compiled") and len(compiled()) == 3


def test_without_its_headers_the_library_is_what_is_built(compiled, monkeypatch):
    build._build_calls(False)
    monkeypatch.setattr(build, "_calls_missing", lambda: "Python.h")
    assert build._build_calls(False).startswith("up to date")
    monkeypatch.setattr(build, "_calls_built_for", lambda: "")
    assert "Python.h not found" in build._build_calls(False)
    assert not os.path.exists(build.CALLS) and len(compiled()) == 1  # (an older one for another torch does not stay)


def test_what_is_missing_is_named(monkeypatch):
    import importlib.util
    import sysconfig
    assert build._calls_missing() == ""
    monkeypatch.setattr(sysconfig, "get_paths", lambda: {"include": "/nowhere"})
    assert build._calls_missing() == "Python.h"
    monkeypatch.setattr(importlib.util, "find_spec", lambda name: None)
    assert build._calls_missing() == "torch"


def test_an_error_of_the_compiler_is_raised(compiled):
    compiled.fail("no such member")
    with pytest.raises(RuntimeError, match="no such member"):
        build._build_calls(False)
    assert not os.path.exists(build.CALLS)
