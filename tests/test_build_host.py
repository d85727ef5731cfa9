"""When _host.so and libmoara.so are built again: the compilers are fakes that write a file."""

import os
import subprocess

import pytest

pytest.importorskip("torch")


@pytest.fixture
def tree(tmp_path, monkeypatch):
    from paper_2609_15037_gb300 import build
    monkeypatch.setattr(build, "HOST", str(tmp_path / "_host.so"))
    monkeypatch.setattr(build, "HOST_SRC", str(tmp_path / "host.cpp"))
    monkeypatch.setattr(build, "LIB", str(tmp_path / "libmoara.so"))
    monkeypatch.setattr(build, "OUT_DIR", str(tmp_path / "x86_64"))
    monkeypatch.setattr(build, "_sources", lambda: [str(tmp_path / "a.cu")])
    monkeypatch.setattr(build, "_nvcc", lambda: "nvcc")
    for f in ("host.cpp", "a.cu"):
        (tmp_path / f).write_text("")
    calls = []

    def run(cmd, **_):
        out = cmd[cmd.index("-o") + 1]
        calls.append(os.path.basename(out))
        with open(out, "w") as f:
            f.write(build.platform.machine())
        return subprocess.CompletedProcess(cmd, 0, "", "")
    monkeypatch.setattr(build.subprocess, "run", run)

    def built():
        calls.clear()
        build.build()
        return sorted(calls)
    return build, tmp_path, built


EVERYTHING = ["_host.so.tmp", "a.cu.o", "libmoara.so.tmp"]


def test_nothing_is_built_twice(tree):
    _, _, built = tree
    assert built() == EVERYTHING and built() == []


def test_libraries_of_another_machine_are_replaced(tree, monkeypatch):
    """One tree, built here, on a second machine, and here again."""
    build, tmp, built = tree

    def machine(name):
        monkeypatch.setattr(build, "OUT_DIR", str(tmp / name))
        monkeypatch.setattr(build.platform, "machine", lambda: name)
    machine("first")
    assert built() == EVERYTHING
    machine("another")
    assert built() == EVERYTHING
    machine("first")
    assert built() == ["_host.so.tmp", "libmoara.so.tmp"]
    assert (tmp / "_host.so").read_text() == (tmp / "libmoara.so").read_text() == "first"


def test_a_library_that_another_build_left_is_replaced(tree):
    build, tmp, built = tree
    built()
    for f in ("_host.so", "libmoara.so"):
        (tmp / f).write_text("another machine's")
        os.utime(tmp / f, ns=(1, os.stat(os.path.join(build.OUT_DIR, "a.cu.o")).st_mtime_ns + 10 ** 9))
    assert built() == ["_host.so.tmp", "libmoara.so.tmp"]


def test_another_compiler_command_builds_the_module_again(tree, monkeypatch):
    build, _, built = tree
    built()
    command = build._host_command
    monkeypatch.setattr(build, "_host_command", lambda out: command(out) + ["-O3"])
    assert built() == ["_host.so.tmp"]


def test_another_source_builds_the_module_again(tree):
    build, tmp, built = tree
    built()
    os.utime(tmp / "host.cpp", ns=(1, 1))
    assert built() == ["_host.so.tmp"]
