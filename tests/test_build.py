"""What a build takes over from the one before it, with a compiler that only says what it was asked."""
import os
import stat
import time

import pytest

from paper_1802_00130_b200 import build as b

COMPILER = """#!/usr/bin/env python3
import os, sys, time
out = sys.argv[sys.argv.index("-o") + 1]
with open("../log", "a") as f:
    f.write(" ".join(sys.argv[1:]) + "\\n")
open(out, "w").write("part of it")
for a in sys.argv[1:]:
    if os.path.exists("../fail_" + a): sys.exit(1)
    if os.path.exists("../edit_" + a):
        os.remove("../edit_" + a)
        time.sleep(0.05)
        open(a, "a").write("// edited meanwhile")
        time.sleep(0.05)
open(out, "w").write("\\n".join(sys.argv[1:]))
"""


@pytest.fixture
def tree(tmp_path, monkeypatch):
    pkg = tmp_path / "pkg"
    (pkg / "csrc").mkdir(parents=True)
    (tmp_path / "include").mkdir()
    (tmp_path / "include" / "gn.h").write_text("")
    nvcc = tmp_path / "nvcc"
    nvcc.write_text(COMPILER)
    nvcc.chmod(nvcc.stat().st_mode | stat.S_IXUSR)
    for name in ("a.cu", "b.cu", "h.cuh"):
        (pkg / "csrc" / name).write_text("")
    for path in [tmp_path / "include" / "gn.h", *(pkg / "csrc").iterdir()]:
        os.utime(path, (time.time() - 100,) * 2)
    monkeypatch.setattr(b, "HERE", str(pkg))
    monkeypatch.setattr(b, "CSRC", str(pkg / "csrc"))
    monkeypatch.setattr(b, "LIB", str(pkg / "lib.so"))
    monkeypatch.setattr(b, "SOURCES", ["a.cu", "b.cu"])
    monkeypatch.setattr(b, "FLAGS", ["-shared", "-O3"])
    monkeypatch.setenv("NVCC", str(nvcc))
    monkeypatch.delenv("GN_NVTX", raising=False)
    return pkg


def compiled(pkg):
    """The sources that were compiled since the last look."""
    log = pkg / "log"
    lines = log.read_text().splitlines() if log.exists() else []
    log.write_text("")
    return sorted(line.split()[-1] for line in lines if "-c" in line.split())


def edit(path):
    time.sleep(0.02)
    path.write_text("// edited")


def test_what_is_newer_than_its_sources_is_taken_over(tree):
    b.build()
    assert compiled(tree) == ["a.cu", "b.cu"] and os.path.exists(b.LIB)
    b.build()
    assert (tree / "log").read_text() == ""
    edit(tree / "csrc" / "a.cu")
    b.build()
    assert compiled(tree) == ["a.cu"]
    edit(tree / "csrc" / "h.cuh")
    b.build()
    assert compiled(tree) == ["a.cu", "b.cu"]
    b.build(force=True)
    assert compiled(tree) == ["a.cu", "b.cu"]


def test_objects_of_another_command_are_not(tree, monkeypatch):
    monkeypatch.setenv("GN_NVTX", "1")
    b.build()
    assert compiled(tree) == ["a.cu", "b.cu"]
    monkeypatch.delenv("GN_NVTX")
    edit(tree / "csrc" / "a.cu")
    b.build()
    assert compiled(tree) == ["a.cu", "b.cu"]
    assert "GN_NVTX" not in (tree / "_build" / "b.cu.o").read_text()
    monkeypatch.setattr(b, "FLAGS", ["-shared", "-O2"])
    edit(tree / "csrc" / "b.cu")
    b.build()
    assert compiled(tree) == ["a.cu", "b.cu"]


def test_what_a_compiler_left_half_done_is_not(tree):
    (tree / "fail_b.cu").write_text("")
    with pytest.raises(RuntimeError, match="nvcc failed"):
        b.build()
    assert not os.path.exists(b.LIB) and [p.name for p in (tree / "_build").iterdir() if "b.cu" in p.name] == []
    (tree / "fail_b.cu").unlink()
    compiled(tree)
    b.build()
    assert compiled(tree) == ["b.cu"]


def test_an_edit_during_a_build_is_newer_than_it(tree):
    (tree / "edit_a.cu").write_text("")
    b.build()
    compiled(tree)
    assert b.is_stale()
    b.build()
    assert compiled(tree) == ["a.cu"] and not b.is_stale()
