"""The compiled caller where torch's headers are missing or do not compile: the calls by pointers remain, those that take tensors do not."""
import importlib.util
import os
import subprocess
import sys

import pytest

import paper_2009_09271_b200 as sc
from paper_2009_09271_b200 import binding
from paper_2009_09271_b200 import build as scbuild

wanted = pytest.mark.skipif(not scbuild._calls_wanted(), reason="no Python headers or no C++ compiler")


def made(monkeypatch, tmp_path):
    """The commands, with the caller's place in a folder of its own."""
    monkeypatch.setattr(scbuild, "CALLS", str(tmp_path / os.path.basename(scbuild.CALLS)))
    return scbuild._calls_commands()


@wanted
def test_without_torchs_headers_the_caller_is_still_built(monkeypatch, tmp_path):
    monkeypatch.setattr(scbuild, "_torch_home", lambda: str(tmp_path / "nowhere"))
    commands = made(monkeypatch, tmp_path)
    assert scbuild._calls_wanted() and len(commands) == 1 and "-DSC_TENSORS" not in commands[0]
    subprocess.run(commands[0], check=True)
    spec = importlib.util.spec_from_file_location("_sc_calls", scbuild.CALLS)
    calls = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(calls)
    assert binding._tensor_calls(calls) is None
    for name in binding._LAYER_CALLS:
        assert callable(getattr(calls, name))
    with pytest.raises(TypeError):
        calls.bind()


def run_build(monkeypatch, tmp_path, fails):
    """A build whose commands are noted instead of run; those that `fails` names fail."""
    ran = []

    class Done:
        def __init__(self, command, **_):
            ran.append(command)
            out = command[command.index("-o") + 1]
            self.returncode, self.stdout, self.stderr = int(fails(command)), "", ""
            if not self.returncode:
                with open(out, "w") as f:
                    f.write("made")

        def communicate(self):
            return "", None

    monkeypatch.setattr(scbuild, "LIB", str(tmp_path / "libsparsecomm.so"))
    monkeypatch.setattr(scbuild.subprocess, "Popen", Done)
    monkeypatch.setattr(scbuild.subprocess, "run", Done)
    scbuild.build(force=True)
    return [c for c in ran if c[c.index("-o") + 1] == scbuild.CALLS]


@wanted
def test_a_caller_that_does_not_compile_with_tensors_is_built_without(monkeypatch, tmp_path):
    if len(made(monkeypatch, tmp_path)) < 2:
        pytest.skip("torch's headers are not here")
    tried = run_build(monkeypatch, tmp_path, lambda c: "-DSC_TENSORS" in c)
    assert ["-DSC_TENSORS" in c for c in tried] == [True, False] and os.path.exists(scbuild.CALLS)
    assert len(run_build(monkeypatch, tmp_path, lambda c: False)) == 1
    with pytest.raises(RuntimeError, match="_sc_calls"):
        run_build(monkeypatch, tmp_path, lambda c: c[c.index("-o") + 1] == scbuild.CALLS)


@wanted
def test_both_forms_reach_the_library(monkeypatch, tmp_path):
    """In a process of its own, which has the plain form in the place of the other."""
    monkeypatch.setattr(scbuild, "_torch_home", lambda: str(tmp_path / "nowhere"))
    subprocess.run(made(monkeypatch, tmp_path)[0], check=True)
    sc.load_library()
    code = ("import sys, importlib.util; from paper_2009_09271_b200 import binding as b; import paper_2009_09271_b200 as sc\n"
            f"spec = importlib.util.spec_from_file_location('paper_2009_09271_b200._sc_calls', {scbuild.CALLS!r})\n"
            "m = importlib.util.module_from_spec(spec); spec.loader.exec_module(m); sys.modules[spec.name] = m; sc._sc_calls = m\n"
            "calls = b._layer_calls(sc.load_library())\n"
            "assert calls is m and b._tensor_calls(calls) is None\n"
            "assert calls.sc_checkpoint_pack(None, 0, None, 0, 0, 0, None, None, None) == -1\n"
            "assert calls.sc_dropout(None, 0, None, 0, None, 0, 0.5, 1, 0, 0, None, 0, None) == -1\n")
    subprocess.run([sys.executable, "-c", code], check=True, cwd=os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
