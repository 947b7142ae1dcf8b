"""libgrid.so needs g++ and hipcc only: where torch is not installed it is built without the module that needs it, and
the package compiles grammars.  The compilers are recorded, not run."""

import importlib.util
import subprocess
import sys
from pathlib import Path

import pytest

from paper_2607_11951_amd import build as B


@pytest.fixture
def commands(monkeypatch, tmp_path):
    """what build() would run, with outputs in a place of its own"""
    ran = []

    def output(cmd):
        Path(cmd[cmd.index("-o") + 1]).write_bytes(b"")

    class Popen:
        def __init__(self, cmd, **kw):
            ran.append(cmd)
            self.args = cmd
            output(cmd)

        def wait(self):
            return 0

    monkeypatch.setattr(B.subprocess, "Popen", Popen)
    monkeypatch.setattr(B.subprocess, "run", lambda cmd, **kw: (ran.append(cmd), output(cmd)))
    monkeypatch.setattr(B, "BUILD", tmp_path / "_build")
    monkeypatch.setattr(B, "OUT", tmp_path / "libgrid.so")
    monkeypatch.setattr(B, "MODULE", tmp_path / "_step.so")
    return ran


def test_without_torch(commands, monkeypatch):
    find = importlib.util.find_spec
    monkeypatch.setattr(B.importlib.util, "find_spec", lambda name, *a: None if name == "torch" else find(name, *a))
    assert B.build() == B.OUT and B.OUT.exists() and not B.MODULE.exists()
    sources = [Path(x).name for cmd in commands for x in cmd if x.endswith((".cpp", ".hip"))]
    assert sorted(sources) == sorted(B.HOST_SOURCES + B.HIP_SOURCES)
    assert not any(x.startswith("-ltorch") for cmd in commands for x in cmd)


def test_with_torch(commands):
    pytest.importorskip("torch")
    B.build()
    assert B.OUT.exists() and B.MODULE.exists()
    assert any("step_module.cpp" in x for cmd in commands for x in cmd)


def test_the_package_does_not_import_torch():
    code = "import sys; sys.modules['torch'] = None; import paper_2607_11951_amd as G; G.lib(); G.Grid; G.apply"
    if not B.OUT.exists():
        B.build()
    subprocess.run([sys.executable, "-c", code], check=True, cwd=B.PKG.parent)
