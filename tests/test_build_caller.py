"""The compiled caller follows the library: an older one is rebuilt, and none is left behind where it cannot be."""
import os

import pytest

from paper_2009_09271_b200 import build as scbuild


@pytest.fixture
def tree(tmp_path, monkeypatch):
    """A package folder with a library and a caller newer than all sources, and commands that are noted instead of run."""
    lib, calls, source = tmp_path / "libsparsecomm.so", tmp_path / "_sc_calls.so", tmp_path / "sc_calls.c"
    for path in (source, lib, calls):
        path.write_text("made before")
    now = max(os.path.getmtime(d) for d in scbuild._dependencies()) + 1000
    for path in (source, lib, calls):
        os.utime(path, (now, now))
    monkeypatch.setattr(scbuild, "LIB", str(lib))
    monkeypatch.setattr(scbuild, "CALLS", str(calls))
    monkeypatch.setattr(scbuild, "CALLS_SOURCE", str(source))
    ran = []

    class Done:
        def __init__(self, command, **_):
            out = command[command.index("-o") + 1]
            ran.append(os.path.basename(out))
            self.returncode, self.stdout, self.stderr = int(os.path.basename(out) in fails), "", ""
            if not self.returncode:
                with open(out, "w") as f:
                    f.write("made now")

        def communicate(self):
            return "", None

    fails = set()
    monkeypatch.setattr(scbuild.subprocess, "Popen", Done)
    monkeypatch.setattr(scbuild.subprocess, "run", Done)
    monkeypatch.setattr(scbuild, "_calls_wanted", lambda: True)
    return lib, calls, source, ran, fails, now


def test_nothing_is_built_where_everything_is_current(tree):
    lib, calls, source, ran, fails, now = tree
    scbuild.build()
    assert not ran and calls.read_text() == "made before"


def test_an_older_caller_is_rebuilt_beside_a_current_library(tree):
    lib, calls, source, ran, fails, now = tree
    os.utime(calls, (now - 10, now - 10))
    scbuild.build()
    assert "_sc_calls.so" in ran and calls.read_text() == "made now"


def test_a_failed_caller_leaves_none_and_is_tried_again(tree):
    lib, calls, source, ran, fails, now = tree
    fails.add("_sc_calls.so")
    with pytest.raises(RuntimeError, match="_sc_calls"):
        scbuild.build(force=True)
    assert not calls.exists()
    fails.clear()
    scbuild.build()
    assert calls.read_text() == "made now"


def test_a_failed_library_leaves_no_caller(tree):
    lib, calls, source, ran, fails, now = tree
    fails.add("sc_layer.o")
    with pytest.raises(RuntimeError, match="nvcc"):
        scbuild.build(force=True)
    assert not calls.exists()


def test_an_older_caller_that_cannot_be_rebuilt_is_not_left_over(tree, monkeypatch):
    lib, calls, source, ran, fails, now = tree
    monkeypatch.setattr(scbuild, "_calls_wanted", lambda: False)
    scbuild.build()
    assert not ran and calls.exists()               # current: stays, where there is no compiler too
    os.utime(calls, (now - 10, now - 10))
    scbuild.build()
    assert not calls.exists() and lib.read_text() == "made now"
    ran.clear()
    scbuild.build()
    assert not ran
