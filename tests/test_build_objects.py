"""The build keeps objects between calls: one whose compilation was broken off is made again, whatever the source says now, and
so is the library."""
import os
import stat

import pytest

from paper_2606_03077_b200 import build

NVCC = """#!/bin/sh
# writes what it was given: the source after -c, or all objects linked together
out=""; src=""; objs=""
while [ $# -gt 0 ]; do
  case "$1" in
    -o) out="$2"; shift;;
    -c) src="$2"; shift;;
    *.o) objs="$objs $1";;
  esac
  shift
done
if [ -n "$src" ]; then
  if grep -q BROKEN "$src"; then echo half > "$out"; exit 1; fi
  cat "$src" > "$out"
else
  if cat $objs | grep -q UNLINKABLE; then echo half > "$out"; exit 1; fi
  cat $objs > "$out"
fi
"""


@pytest.fixture
def tree(tmp_path, monkeypatch):
    csrc, include = tmp_path / "csrc", tmp_path / "include"
    csrc.mkdir(); include.mkdir()
    nvcc = tmp_path / "nvcc"
    nvcc.write_text(NVCC)
    nvcc.chmod(nvcc.stat().st_mode | stat.S_IXUSR)
    for name, value in dict(CSRC=str(csrc), INCLUDE=str(include), LIB_PATH=str(tmp_path / "lib.so"), STAMP_PATH=str(tmp_path / "lib.stamp"),
                            OBJ_DIR=str(tmp_path / "objects"), SOURCES=["one.cu", "two.cu"], _nvcc=lambda: str(nvcc)).items():
        monkeypatch.setattr(build, name, value)
    (include / "libra.h").write_text("// header\n")
    (csrc / "one.cu").write_text('#include "part.cuh"\none\n')
    (csrc / "part.cuh").write_text("// part\n")
    (csrc / "two.cu").write_text("two\n")
    return csrc


def made():
    with open(build.build_library(verbose=False)) as f:
        return f.read()


def test_an_object_that_was_broken_off_is_made_again(tree):
    first = made()
    assert "one" in first and "two" in first
    (tree / "one.cu").write_text("BROKEN\n")
    with pytest.raises(RuntimeError):
        made()
    (tree / "one.cu").write_text('#include "part.cuh"\none\n')   # back to what the kept object was made from, and another change
    (tree / "two.cu").write_text("three\n")
    assert made() == '#include "part.cuh"\none\nthree\n'


def test_a_library_that_was_broken_off_is_linked_again(tree):
    first = made()
    (tree / "two.cu").write_text("UNLINKABLE\n")
    with pytest.raises(RuntimeError):
        made()
    (tree / "two.cu").write_text("two\n")
    assert made() == first


def test_only_what_changed_is_compiled_again(tree):
    made()
    obj = os.path.join(build.OBJ_DIR, "two.cu.o")
    with open(obj, "a") as f:
        f.write("kept\n")
    (tree / "part.cuh").write_text("// another part\n")          # included by one.cu alone
    (tree / "one.cu").write_text('#include "part.cuh"\nfour\n')
    assert made() == '#include "part.cuh"\nfour\ntwo\nkept\n'
