"""What is built, and when it is built again.  No GPU, and no compiler: stand-ins are called in its place."""
import importlib.metadata
import importlib.util
import os
import stat

import pytest

from paper_2609_00097_b200 import build as real


def load(name):
    spec = importlib.util.spec_from_file_location(name, real.__file__)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.fixture
def build(tmp_path, monkeypatch):
    """A build module of its own whose products go to a folder of their own, with an nvcc and a g++ that only leave a file."""
    module = load("build_under_test")
    tool = tmp_path / "tool"
    tool.write_text('#!/bin/sh\nwhile [ "$1" != -o ]; do shift; done\necho built > "$2"\n')
    tool.chmod(tool.stat().st_mode | stat.S_IXUSR)
    monkeypatch.setenv("NVCC", str(tool))
    monkeypatch.setenv("CXX", str(tool))
    monkeypatch.setattr(module, "LIB_PATH", str(tmp_path / "lib.so"))
    monkeypatch.setattr(module, "BINDING_PATH", str(tmp_path / "binding.so"))
    return module


def test_both_are_built_and_not_again(build):
    assert build.is_stale()
    assert build.build_library() == build.LIB_PATH
    assert os.path.exists(build.LIB_PATH) and os.path.exists(build.BINDING_PATH) and not build.is_stale()
    before = os.stat(build.LIB_PATH).st_mtime_ns, os.stat(build.BINDING_PATH).st_mtime_ns
    build.build_library()
    assert before == (os.stat(build.LIB_PATH).st_mtime_ns, os.stat(build.BINDING_PATH).st_mtime_ns)


@pytest.mark.parametrize("tool", ["/nonexistent/g++", "/bin/false"])
def test_the_library_needs_no_host_compiler_and_no_torch_headers(build, monkeypatch, tool):
    monkeypatch.setenv("CXX", tool)
    with open(build.BINDING_PATH, "w") as f:      # one that is older than its sources is not left in place
        f.write("old")
    os.utime(build.BINDING_PATH, (0, 0))
    with pytest.warns(RuntimeWarning, match="byte cache"):
        assert build.build_library() == build.LIB_PATH
    assert os.path.exists(build.LIB_PATH) and not os.path.exists(build.BINDING_PATH)
    with pytest.raises((OSError, RuntimeError, build.subprocess.CalledProcessError)):
        build.build_binding()


def test_a_library_that_cannot_be_built_is_an_error(build, monkeypatch):
    monkeypatch.setenv("NVCC", "/bin/false")
    with pytest.raises(build.subprocess.CalledProcessError):
        build.build_library()


def test_a_binding_belongs_to_one_version_of_torch(monkeypatch):
    import torch
    assert "torch-" + torch.__version__ in os.path.basename(real.BINDING_PATH)
    version = importlib.metadata.version
    monkeypatch.setattr(importlib.metadata, "version", lambda name: "99.1.0" if name == "torch" else version(name))
    other = load("build_of_another_torch")
    assert other.BINDING_PATH != real.BINDING_PATH and "torch-99.1.0" in other.BINDING_PATH and other.is_stale()
    assert other.LIB_PATH == real.LIB_PATH          # the library does not depend on it


def test_without_torch_there_is_no_binding_but_a_path_to_say_so(monkeypatch):
    def none(name):
        raise importlib.metadata.PackageNotFoundError(name)
    monkeypatch.setattr(importlib.metadata, "version", none)
    assert not os.path.exists(load("build_without_torch").BINDING_PATH)
