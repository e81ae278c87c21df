"""A library is linked from objects of one compiler and one set of flags, whatever was built before it."""
import os
import stat

import pytest

from paper_2505_22179_amd import build

FAKE = """#!/bin/sh
# writes what it was given into its output, one line an object: the sources' text and the flags of a compilation, the objects of a link
all="$*"; out=; link=; rest=
while [ $# -gt 0 ]; do
    case "$1" in -o) out="$2"; shift;; -shared) link=1;; *.o|*.hip) rest="$rest $1";; esac
    shift
done
if [ -n "$link" ]; then cat $rest > "$out"; else echo "$(cat $rest) | $0 $all" > "$out"; fi
"""


@pytest.fixture
def tree(tmp_path, monkeypatch):
    csrc, include, lib = tmp_path / "csrc", tmp_path / "include", tmp_path / "lib"
    csrc.mkdir()
    include.mkdir()
    for name in ("a", "b", "c"):
        (csrc / f"{name}.hip").write_text(name)
        os.utime(csrc / f"{name}.hip", (1000, 1000))
    for n in ("one", "two"):
        (tmp_path / n).write_text(FAKE)
        (tmp_path / n).chmod(stat.S_IRWXU)
    for attribute, value in (("CSRC", csrc), ("INCLUDE", include), ("LIBDIR", lib), ("LIB", lib / "libw4a16.so")):
        monkeypatch.setattr(build, attribute, str(value))
    monkeypatch.setattr(build, "HIPCC_FLAGS", ["-DPLAIN"])
    monkeypatch.setenv("HIPCC", str(tmp_path / "one"))
    return tmp_path


def lines():
    return open(build.LIB).read().splitlines()


def edit(tree, name):
    path = tree / "csrc" / f"{name}.hip"
    path.write_text(path.read_text() + "+")   # its time is now: newer than what was built


def test_objects_of_other_flags_are_not_linked(tree):
    build.build()
    assert len(lines()) == 3
    build.build(extra_flags=["-DEXTRA"])
    assert all("-DEXTRA" in ln for ln in lines())
    edit(tree, "b")
    build.build(force=False)
    assert [ln.split(" | ")[0] for ln in lines()] == ["a", "b+", "c"] and not any("-DEXTRA" in ln for ln in lines())


def test_a_library_of_other_flags_is_not_taken_for_the_one_asked_for(tree):
    build.build(extra_flags=["-DEXTRA"])
    build.build(force=False)
    assert len(lines()) == 3 and not any("-DEXTRA" in ln for ln in lines())
    build.build(force=False, extra_flags=["-DEXTRA"])
    assert all("-DEXTRA" in ln for ln in lines())


def test_changed_flags_and_another_compiler_build_everything_anew(tree, monkeypatch):
    build.build()
    monkeypatch.setattr(build, "HIPCC_FLAGS", ["-DOTHER"])
    build.build(force=False)
    assert len(lines()) == 3 and all("-DOTHER" in ln for ln in lines())
    monkeypatch.setenv("HIPCC", str(tree / "two"))
    edit(tree, "c")
    build.build(force=False)
    assert [ln.split(" | ")[0] for ln in lines()] == ["a", "b", "c+"] and all(f"{tree}/two " in ln for ln in lines())


def test_only_what_changed_is_compiled(tree):
    build.build()
    first = {f.name: f.stat().st_mtime_ns for f in (tree / "lib").rglob("*.o")}
    assert len(first) == 3
    edit(tree, "a")
    build.build(force=False)
    again = {f.name: f.stat().st_mtime_ns for f in (tree / "lib").rglob("*.o")}
    assert [n for n in first if first[n] != again[n]] == ["w4a16_a.o"] and lines()[0].startswith("a+ ")
