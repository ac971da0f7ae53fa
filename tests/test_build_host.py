"""What the build needs, and when it counts as done (nothing is compiled here)."""
import importlib.util
import os

import pytest

from paper_2407_19644_b200 import build as b


@pytest.fixture
def commands(monkeypatch):
    """The commands the build would run."""
    ran = []
    monkeypatch.setattr(b.subprocess, "run", lambda cmd, **k: ran.append(cmd))
    monkeypatch.setattr(b.os, "replace", lambda a, c: open(c, "a").close())
    return ran


def test_the_library_builds_without_torch(monkeypatch, commands):
    find = importlib.util.find_spec
    monkeypatch.setattr(importlib.util, "find_spec", lambda name, *a: None if name == "torch" else find(name, *a))
    monkeypatch.setattr(b, "build_torch_calls", lambda *a, **k: pytest.fail("the extension module needs torch"))
    monkeypatch.setattr(b, "_stale", lambda lib: False)
    assert b.build() == b.LIB and b.build(debug=True) == b.LIB_DEBUG


def test_the_library_is_built_before_the_extension_module(monkeypatch):
    order = []
    monkeypatch.setattr(b, "build_library", lambda *a: order.append("library") or b.LIB)
    monkeypatch.setattr(b, "build_torch_calls", lambda *a: order.append("extension"))
    assert b.build() == b.LIB and order == ["library", "extension"]


def test_another_torch_makes_the_extension_module_stale(monkeypatch, commands, tmp_path):
    import torch
    lib = tmp_path / "_torch_calls.so"
    lib.touch()
    monkeypatch.setattr(b, "TORCH_LIB", str(lib))
    monkeypatch.setattr(b, "TORCH_MADE_FOR", str(tmp_path / "build" / "torch_calls.txt"))
    assert b.build_torch_calls() == str(lib) and len(commands) == 1          # (nobody knows what it was built against)
    assert b.build_torch_calls() == str(lib) and len(commands) == 1          # up to date
    monkeypatch.setattr(torch, "__version__", "0.0.1")
    b.build_torch_calls()
    assert len(commands) == 2
    b.build_torch_calls()
    assert len(commands) == 2
    os.utime(b.TORCH_LIB, (0, 0))                                            # a newer source
    b.build_torch_calls()
    assert len(commands) == 3
    b.build_torch_calls(force=True)
    assert len(commands) == 4
