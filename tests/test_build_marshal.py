"""The extension module is rebuilt when it was built against another torch, not only when its sources are newer."""
import importlib.metadata
import subprocess

import pytest

from paper_2608_13057_b200 import build


@pytest.fixture
def compiled(monkeypatch):
    """The compiler's command lines, recorded instead of run."""
    build.build()
    lines = []
    monkeypatch.setattr(subprocess, "run", lambda cmd, **kw: lines.append(cmd) or subprocess.CompletedProcess(cmd, 0, "", ""))
    return lines


def test_the_module_of_this_torch_stays(compiled):
    build.build_marshal()
    assert compiled == []


def test_the_module_of_another_torch_is_rebuilt(compiled, monkeypatch):
    version = importlib.metadata.version
    monkeypatch.setattr(importlib.metadata, "version", lambda name: "1.2.3+other" if name == "torch" else version(name))
    build.build_marshal()
    assert len(compiled) == 1 and any("1.2.3+other" in a for a in compiled[0])


def test_the_module_of_a_torch_elsewhere_is_rebuilt(compiled, monkeypatch):
    monkeypatch.setattr(build, "_torch_dir", lambda: "/opt/elsewhere/torch")
    build.build_marshal()
    assert len(compiled) == 1 and any("/opt/elsewhere/torch" in a for a in compiled[0])
