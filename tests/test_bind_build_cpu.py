"""The compiled marshalling of the paged cache's calls is made anew for another PyTorch, Python or command, and refused where it
was made for another."""

import os
import subprocess
import sys
import types

import pytest
import torch

from paper_2608_08878_gb300 import build, dc


@pytest.fixture
def fake(tmp_path, monkeypatch):
    """The builder with a compiler that only writes its output: the commands it was given."""
    ran = []

    def run(cmd, **kw):
        ran.append(cmd)
        with open(cmd[cmd.index("-o") + 1], "w"):
            pass
        return types.SimpleNamespace(returncode=0, stdout="", stderr="")

    monkeypatch.setattr(build, "LIB_BIND", str(tmp_path / "_dc_bind.so"))
    monkeypatch.setattr(subprocess, "run", run)
    return ran


def test_built_once(fake):
    assert build._bind() == build.LIB_BIND and len(fake) == 1 and os.path.exists(build.LIB_BIND)
    build._bind()
    assert len(fake) == 1


def test_built_anew_for_another_torch(fake, monkeypatch):
    build._bind()
    monkeypatch.setattr(torch, "__version__", "9.9.9+cu999")
    build._bind()
    build._bind()
    assert len(fake) == 2
    monkeypatch.setattr(torch, "__path__", ["/elsewhere/torch"])
    build._bind()
    assert len(fake) == 3


def test_built_anew_for_another_python(fake, monkeypatch):
    build._bind()
    monkeypatch.setattr(build.sysconfig, "get_config_var", lambda name: "cpython-999-other")
    build._bind()
    assert len(fake) == 2


def test_without_torch(fake, monkeypatch):
    monkeypatch.setitem(sys.modules, "torch", None)
    with pytest.raises(RuntimeError, match="PyTorch cannot be imported"):
        build._bind()
    assert not fake


@pytest.mark.parametrize("version", ["2.0.0", "{}1", "{}"])
def test_loaded_for_the_right_torch_only(version, monkeypatch):
    build.build()
    monkeypatch.setattr(dc, "_bound", None)
    made_for = dc._bind().torch
    assert torch.__version__ == made_for
    monkeypatch.setattr(dc, "_bound", None)
    monkeypatch.setattr(torch, "__version__", version.format(made_for))
    if version == "{}":
        assert dc._bind().torch == made_for
        return
    with pytest.raises(OSError, match="built for PyTorch"):
        dc._bind()
