"""What a build needs: the library nvcc and g++ alone, its binding for Python torch too.  The compilers are stood in for."""
import importlib.util
import os
import types

import pytest

from paper_2003_06513_gb300 import build as B


@pytest.fixture
def commands(monkeypatch, tmp_path_factory):
    """The commands of builds into an empty folder, each of which makes its output."""
    ran, out = [], tmp_path_factory.mktemp("out")

    def run(cmd, **kw):
        ran.append(cmd)
        if "-o" in cmd:
            open(cmd[cmd.index("-o") + 1], "w").close()
        return types.SimpleNamespace(returncode=0, stdout="", stderr="")
    for name, path in (("BUILD", ""), ("LIB", "libpatconv.so"), ("BINDING", "_patconv.so")):
        monkeypatch.setattr(B, name, str(out / path))
    monkeypatch.setattr(B, "_nvcc", lambda: "/cuda/bin/nvcc")
    monkeypatch.setattr(B.subprocess, "run", run)
    return ran


def _without_torch(monkeypatch):
    find = importlib.util.find_spec
    monkeypatch.setattr(importlib.util, "find_spec", lambda name, *a: None if name == "torch" else find(name, *a))


def test_the_library_builds_without_torch(commands, monkeypatch):
    _without_torch(monkeypatch)
    assert B.build() == B.LIB and os.path.exists(B.LIB) and not os.path.exists(B.BINDING)
    made = [c for c in commands if "-o" in c]
    assert len(made) == len(B.KERNELS) + 2 and not any("binding" in a or "torch" in a for c in made for a in c)
    commands.clear()
    assert B.build() == B.LIB and not commands
    with pytest.raises(RuntimeError, match="torch"):
        B.build(binding=True)


def test_library_and_binding_go_stale_each_by_its_own(commands, monkeypatch):
    B.build(binding=False)
    assert not os.path.exists(B.BINDING)
    commands.clear()
    B.build(binding=True)
    assert os.path.exists(B.BINDING) and [c[0] for c in commands] == ["g++", "g++"]
    commands.clear()
    B.build(binding=True)
    assert not commands
    monkeypatch.setattr(B, "_torch_version", lambda d: "another")
    B.build(binding=False)
    assert not commands
    B.build(binding=True)
    assert [c[0] for c in commands] == ["g++", "g++"]
    commands.clear()
    B.build(extra_nvcc=["-DX"], binding=True)
    assert len([c for c in commands if "-o" in c]) == len(B.KERNELS) + 2 and not any("binding" in a for c in commands for a in c)
