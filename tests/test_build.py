"""What the build asks for: libss.so hipcc alone, ss_bind.so the host compiler and torch's headers (the commands are not run)."""
import os
import subprocess
import sys

import pytest
import torch

from paper_2402_11131_amd import build


@pytest.fixture
def commands(tmp_path, monkeypatch):
    """(names of the commands that a build runs, in order; a list: while it holds something, the host compiler fails).  The commands
    only make their output files, in a folder of the test's own."""
    ran, broken = [], []

    def run(cmd, **kw):
        ran.append(os.path.basename(cmd[0]))
        if broken and ran[-1] == "g++":
            return subprocess.CompletedProcess(cmd, 1, "no such header")
        open(cmd[cmd.index("-o") + 1], "w").close()
        return subprocess.CompletedProcess(cmd, 0, "")

    monkeypatch.setattr(build.subprocess, "run", run)
    monkeypatch.delenv("CXX", raising=False)
    monkeypatch.setattr(build, "HIPCC", "hipcc")
    monkeypatch.setattr(build, "OBJ_DIR", str(tmp_path / "_build"))
    for name in ("LIB_PATH", "BIND_PATH"):
        monkeypatch.setattr(build, name, str(tmp_path / os.path.basename(getattr(build, name))))
    return ran, broken


def test_the_library_needs_hipcc_alone(commands, monkeypatch):
    monkeypatch.setitem(sys.modules, "torch", None)     # not importable
    build.build_lib()
    assert os.path.exists(build.LIB_PATH) and set(commands[0]) == {"hipcc"}
    assert len(commands[0]) == len(build.sources()) + 1


def test_the_library_is_there_without_the_binding(commands):
    ran, broken = commands
    broken.append(True)
    with pytest.raises(RuntimeError, match="g\\+\\+ failed"):
        build.build_all()
    assert os.path.exists(build.LIB_PATH) and not os.path.exists(build.BIND_PATH)
    broken.clear()
    ran.clear()
    build.build_all(force=False)
    assert ran == ["g++"] and os.path.exists(build.BIND_PATH)


def test_the_binding_is_made_again_for_another_torch(commands, monkeypatch):
    ran, _ = commands
    build.build_bind(force=False)
    assert ran == ["g++"]
    build.build_bind(force=False)
    assert ran == ["g++"]
    monkeypatch.setattr(torch, "__version__", torch.__version__ + ".post1")
    build.build_bind(force=False)
    assert ran == ["g++"] * 2
    build.build_bind(force=False)
    assert ran == ["g++"] * 2
