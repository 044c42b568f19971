"""The build script with stand-ins for the compilers: the library never depends on the binding, and a
binding is rebuilt for another PyTorch."""
import os
import stat
import sys

import pytest

from paper_2606_07713_gb300 import build

COMPILER = """#!/bin/sh
echo "$0 $@" >> {log}
while [ $# -gt 0 ]; do [ "$1" = -o ] && echo made > "$2"; shift; done
exit {rc}
"""


@pytest.fixture
def tools(tmp_path, monkeypatch):
    """Stand-ins for nvcc and g++ that log their calls and make what they are asked for."""
    log = tmp_path / "log"

    def tool(name, rc=0):
        path = tmp_path / name
        path.write_text(COMPILER.format(log=log, rc=rc))
        path.chmod(path.stat().st_mode | stat.S_IXUSR)
        return str(path)

    def calls():
        lines = log.read_text().splitlines() if log.exists() else []
        log.unlink(missing_ok=True)
        return [os.path.basename(line.split()[0]) for line in lines]

    out = tmp_path / "out"
    for name, file in (("BUILD", None), ("LIB", "libmoa_attn.so"), ("BINDING", "moa_torch.so"),
                       ("BINDING_TORCH", "moa_torch.so.torch")):
        monkeypatch.setattr(build, name, str(out / file) if file else str(out), raising=False)
    monkeypatch.setenv("NVCC", tool("nvcc"))
    monkeypatch.setenv("CXX", tool("g++"))
    return tool, calls


def without_torch(monkeypatch):
    find = build.importlib.util.find_spec
    monkeypatch.setattr(build.importlib.util, "find_spec", lambda name, *a: None if name == "torch" else find(name, *a))
    monkeypatch.setitem(sys.modules, "torch", None)     # importing it raises


def test_the_library_builds_without_torch(tools, monkeypatch, capfd):
    without_torch(monkeypatch)
    assert build.build() == build.LIB
    assert os.path.exists(build.LIB) and not os.path.exists(build.BINDING)
    assert "PyTorch" in capfd.readouterr().err


def test_the_library_builds_without_a_host_compiler(tools, monkeypatch, capfd):
    monkeypatch.delenv("CXX")
    which = build.shutil.which
    monkeypatch.setattr(build.shutil, "which", lambda n, *a, **k: None if n in ("g++", "c++") else which(n, *a, **k))
    assert build.build() == build.LIB
    assert os.path.exists(build.LIB) and not os.path.exists(build.BINDING)
    assert "host C++ compiler" in capfd.readouterr().err


def test_a_failing_binding_leaves_the_library(tools, monkeypatch):
    pytest.importorskip("torch")
    tool, _ = tools
    monkeypatch.setenv("CXX", tool("g++", rc=1))
    with pytest.raises(RuntimeError, match="binding failed"):
        build.build()
    assert os.path.exists(build.LIB) and not os.path.exists(build.BINDING)


def test_another_torch_rebuilds_the_binding_only(tools, monkeypatch):
    pytest.importorskip("torch")
    _, calls = tools
    build.build()
    assert "nvcc" in calls()
    build.build()
    assert calls() == []                                  # nothing to do
    version = build.importlib.metadata.version
    monkeypatch.setattr(build.importlib.metadata, "version", lambda n: "99.0" if n == "torch" else version(n))
    build.build()
    assert calls() == ["g++", "g++"]                      # compiled and linked
    build.build()
    assert calls() == []
