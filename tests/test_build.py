"""What the build runs, without running it: the library needs hipcc alone; the binding's helper needs torch and g++, and comes behind it."""
import importlib
import subprocess
import sys

import pytest

build = importlib.import_module("paper_1410_7455_amd.build")


@pytest.fixture
def commands(monkeypatch):
    """The commands of a build; those whose program or argument is in `failing` fail."""
    class Commands(list):
        failing = ()

    made = Commands()

    def run(cmd, **_):
        made.append(cmd)
        failed = any(word in made.failing for word in cmd)
        return subprocess.CompletedProcess(cmd, 1 if failed else 0, "", "no such thing" if failed else "")

    monkeypatch.setattr(build.subprocess, "run", run)
    monkeypatch.setattr(build, "find_hipcc", lambda: "hipcc")
    return made


def linked(commands):
    return [c for c in commands if c[0] == "hipcc" and "-shared" in c and build.LIB_PATH in c]


def helpers(commands):
    return [c for c in commands if build.BINDING_SOURCE in c]


def test_builds_both(commands):
    pytest.importorskip("torch")
    assert build.build() == build.LIB_PATH
    assert len(linked(commands)) == 1 and len(helpers(commands)) == 1 and len(commands) == len(build.SOURCES) + 2


def test_builds_the_library_without_torch(commands, monkeypatch):
    monkeypatch.setitem(sys.modules, "torch", None)
    with pytest.warns(UserWarning, match="_tensors.so"):
        assert build.build() == build.LIB_PATH
    assert len(linked(commands)) == 1 and not helpers(commands)


def test_builds_the_library_without_a_host_compiler(commands, monkeypatch):
    monkeypatch.setattr(build.shutil, "which", lambda name: None)
    with pytest.warns(UserWarning, match="_tensors.so"):
        assert build.build() == build.LIB_PATH
    assert len(linked(commands)) == 1 and not helpers(commands)


def test_a_helper_that_does_not_compile_fails_behind_the_library(commands):
    pytest.importorskip("torch")
    commands.failing = (build.BINDING_SOURCE,)
    with pytest.raises(RuntimeError, match="no such thing"):
        build.build()
    assert len(linked(commands)) == 1


def test_a_source_that_does_not_compile_fails(commands):
    commands.failing = (build.SOURCES[1],)
    with pytest.raises(RuntimeError, match="no such thing"):
        build.build()
    assert not linked(commands)
