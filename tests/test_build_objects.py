"""Which compiled sources a build uses again (no compiler: a script in its place writes down what it is asked for)."""
import os
import time

import pytest

from paper_2605_02218_b200 import build as B

NVCC = """#!/bin/sh
if [ "$1" = --version ]; then cat {dir}/version; exit 0; fi
echo "$@" >> {dir}/calls
if [ "$1" = -c ] && [ -f {dir}/meanwhile ]; then sh {dir}/meanwhile; fi
while [ $# -gt 0 ]; do if [ "$1" = -o ]; then echo made > "$2"; fi; last=$1; shift; done
echo "about $last"
"""


@pytest.fixture
def tree(tmp_path, monkeypatch):
    csrc = tmp_path / "csrc"
    csrc.mkdir()
    (tmp_path / "include").mkdir()
    (tmp_path / "include" / "covspec.h").write_text("")
    (csrc / "binding.cpp").write_text("")
    (csrc / "a.cu").write_text('#include "common.cuh"\n')
    (csrc / "b.cu").write_text("")
    (csrc / "common.cuh").write_text("")
    (tmp_path / "version").write_text("release 1")
    nvcc = tmp_path / "nvcc"
    nvcc.write_text(NVCC.format(dir=tmp_path))
    nvcc.chmod(0o755)
    for name, value in [("ROOT", tmp_path), ("CSRC", csrc), ("LIB", tmp_path / "lib.so"), ("LIB_DEBUG", tmp_path / "lib_debug.so"),
                        ("OBJECTS", tmp_path / "objects"), ("BINDING_SOURCE", csrc / "binding.cpp")]:
        monkeypatch.setattr(B, name, str(value))
    monkeypatch.setattr(B, "SOURCES", ["a.cu", "b.cu"])
    monkeypatch.setattr(B, "build_binding", lambda force=False: None)
    monkeypatch.setattr(B.needs_build, "__defaults__", (str(tmp_path / "lib.so"),))
    monkeypatch.setenv("NVCC", str(nvcc))
    return tmp_path


def age(tree):
    """Everything that is there becomes older."""
    for at, _, names in os.walk(tree):
        for name in names:
            path = os.path.join(at, name)
            t = os.path.getmtime(path) - 10
            os.utime(path, (t, t))


def compiled(tree, **kw):
    """Sources that a build compiles."""
    log = tree / "calls"
    if log.exists():
        log.unlink()
    B.build(**kw)
    lines = log.read_text().splitlines() if log.exists() else []
    return sorted(os.path.basename(line.split()[-1]) for line in lines if " -c " in f" {line} ")


def test_a_source_is_compiled_again_when_a_file_of_it_changes(tree):
    assert compiled(tree) == ["a.cu", "b.cu"] and compiled(tree) == []
    age(tree)
    (tree / "csrc" / "common.cuh").write_text("// new")
    assert compiled(tree) == ["a.cu"] and compiled(tree) == []


def test_another_compiler_or_command_compiles_everything_again(tree):
    compiled(tree)
    age(tree)
    (tree / "version").write_text("release 2")
    (tree / "csrc" / "b.cu").write_text("// new")
    assert compiled(tree) == ["a.cu", "b.cu"]                    # not an old a.o with a new b.o
    assert compiled(tree, debug_bounds=True) == ["a.cu", "b.cu"]
    age(tree)
    (tree / "csrc" / "b.cu").write_text("// newer")
    assert compiled(tree, debug_bounds=True) == ["b.cu"] and compiled(tree) == ["b.cu"]


def test_a_file_that_changes_while_it_is_compiled_is_compiled_again(tree):
    (tree / "meanwhile").write_text(f"sleep 0.05; echo '// changed' >> {tree}/csrc/b.cu; sleep 0.05")
    age(tree)
    compiled(tree)
    (tree / "meanwhile").unlink()
    time.sleep(0.02)
    os.utime(tree / "csrc" / "common.cuh")                       # the library is older than a file
    assert "b.cu" in compiled(tree)


def test_a_verbose_build_says_something_of_every_source(tree, capsys):
    compiled(tree)
    age(tree)
    (tree / "csrc" / "b.cu").write_text("// new")
    assert compiled(tree, verbose=True) == ["a.cu", "b.cu"]
    said = capsys.readouterr().err
    assert "about" in said and "a.cu" in said and "b.cu" in said
