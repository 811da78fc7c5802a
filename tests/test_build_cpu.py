"""What the build needs and when it runs again; the compilers are faked."""
import importlib.util
import os

import pytest

from paper_2410_21271_b200 import build as b


@pytest.fixture
def commands(monkeypatch):
    ran = []

    class Done:
        returncode, stdout = 0, ""

        def __init__(self, cmd, **kw):
            ran.append(cmd)

        def communicate(self):
            return "", None

    b.build()                                                  # (for real, if it has to be)
    monkeypatch.setattr(b.subprocess, "Popen", Done)
    monkeypatch.setattr(b.subprocess, "run", Done)
    return ran


def without_torch(monkeypatch):
    real = importlib.util.find_spec
    monkeypatch.setattr(b.importlib.util, "find_spec", lambda name, *a: None if name.split(".")[0] == "torch" else real(name, *a))


def test_the_library_builds_without_torch(commands, monkeypatch):
    without_torch(monkeypatch)
    assert b.build(force=True) == b.LIB
    assert all(os.path.basename(c[0]) == "nvcc" for c in commands) and len(commands) == len(b.SOURCES) + 1
    assert b.LIB in commands[-1] and not any("torch" in part for c in commands for part in c)


def test_without_torch_what_is_built_counts_as_built(commands, monkeypatch):
    without_torch(monkeypatch)
    monkeypatch.setattr(b, "NATIVE", b.NATIVE + ".none")
    assert not b.needs_build() and b.build() == b.LIB and not commands


def test_a_torch_without_cuda_counts_as_none(commands, monkeypatch, tmp_path):
    (tmp_path / "lib").mkdir()
    (tmp_path / "__init__.py").write_text("")
    spec = importlib.util.spec_from_file_location("torch", str(tmp_path / "__init__.py"))
    real = importlib.util.find_spec
    monkeypatch.setattr(b.importlib.util, "find_spec", lambda name, *a: spec if name == "torch" else real(name, *a))
    b.build(force=True)
    assert all(os.path.basename(c[0]) == "nvcc" for c in commands)


def test_another_torch_builds_the_marshalling_again_and_nothing_else(commands, monkeypatch):
    assert not b.needs_build()
    monkeypatch.setattr(b, "_built_for", lambda *a: "torch 0.0, another python", raising=False)
    assert b.needs_build()
    b.build()
    assert commands and not any(os.path.basename(c[0]) == "nvcc" for c in commands) and b.NATIVE in commands[-1]
