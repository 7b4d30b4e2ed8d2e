"""What the build compiles again: with a stand-in for the compiler that writes its outputs and keeps a list of its calls."""
import os
import stat
import time

import pytest

from paper_2302_12510_b200 import _build

COMPILER = r'''#!/bin/sh
echo "$@" >> "%(log)s"
out= dep= src=
while [ $# -gt 0 ]; do
    case "$1" in
        -o) out=$2; shift;;
        -MF) dep=$2; shift;;
        *.cu) src=$1;;
    esac
    shift
done
echo built > "$out"
[ -z "$dep" ] || echo "x.o : $src" > "$dep"
'''


@pytest.fixture
def project(tmp_path, monkeypatch):
    sources = [str(tmp_path / n) for n in ("a.cu", "b.cu")]
    for s in sources:
        with open(s, "w") as f:
            f.write("//\n")
        os.utime(s, (time.time() - 100, time.time() - 100))
    nvcc, log = tmp_path / "nvcc", tmp_path / "calls"
    nvcc.write_text(COMPILER % {"log": log})
    nvcc.chmod(nvcc.stat().st_mode | stat.S_IXUSR)
    for name, value in (("_SOURCES", sources), ("_OBJECTS", str(tmp_path / "objects")), ("LIB_PATH", str(tmp_path / "lib.so")),
                        ("DEBUG_LIB_PATH", str(tmp_path / "lib_debug.so")), ("_nvcc", lambda: str(nvcc)), ("_deps", lambda: sources),
                        ("NVCC_FLAGS", ["-O3"])):
        monkeypatch.setattr(_build, name, value)

    def calls(**kw):
        """The compiler's calls of one build: sources compiled, and how often it linked."""
        if log.exists():
            log.unlink()
        _build.build_library(**kw)
        lines = log.read_text().splitlines() if log.exists() else []
        return sorted(os.path.basename(s) for s in sources for l in lines if l.split()[-1] == s), sum("-shared" in l for l in lines)

    return sources, calls


def test_nothing_changed_nothing_built(project):
    _, calls = project
    assert calls() == (["a.cu", "b.cu"], 1)
    assert calls() == ([], 0)
    assert calls(debug_bounds=True) == (["a.cu", "b.cu"], 1)
    assert calls(debug_bounds=True) == ([], 0) and calls() == ([], 0)
    assert calls(force=True) == (["a.cu", "b.cu"], 1)


def test_a_changed_source_alone(project):
    sources, calls = project
    calls()
    os.utime(sources[1], (time.time() + 100, time.time() + 100))
    assert calls() == (["b.cu"], 1)


def test_other_options_build_everything_again(project, monkeypatch):
    _, calls = project
    calls()
    calls(debug_bounds=True)
    monkeypatch.setattr(_build, "NVCC_FLAGS", ["-O3", "-lineinfo"])
    assert calls() == (["a.cu", "b.cu"], 1)
    assert calls() == ([], 0)
    assert calls(debug_bounds=True) == (["a.cu", "b.cu"], 1)
