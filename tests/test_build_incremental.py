"""What a second build compiles again: everything that was made from what has changed, and nothing else."""
import os
import stat

import pytest

from paper_2603_20661_b200 import build as cuda_build


@pytest.fixture
def tree(tmp_path, monkeypatch):
    """A package of three small sources, one of which includes another, and a compiler that writes down what it is asked to compile."""
    csrc, include = tmp_path / "package" / "csrc", tmp_path / "include"
    csrc.mkdir(parents=True), include.mkdir()
    (include / "api.h").write_text("int api();\n")
    (csrc / "common.cuh").write_text("#pragma once\n#define COMMON 1\n")
    (csrc / "rows.cu").write_text('#include "common.cuh"\n#ifndef NAME\n#define NAME rows\n#endif\nextern "C" int NAME() { return COMMON; }\n')
    (csrc / "rows_tree.cu").write_text('#define NAME rows_tree\n#include "rows.cu"\n')
    (csrc / "other.cu").write_text('extern "C" int other() { return 2; }\n')
    log, nvcc = tmp_path / "log", tmp_path / "nvcc"
    nvcc.write_text(f'#!/bin/bash\nfor a in "$@"; do case "$a" in *.cu) echo "$(basename "$a")" >> {log};; esac; done\nexec {cuda_build.NVCC} "$@"\n')
    nvcc.chmod(nvcc.stat().st_mode | stat.S_IEXEC)
    monkeypatch.setattr(cuda_build, "HERE", str(tmp_path / "package"))
    monkeypatch.setattr(cuda_build, "CSRC", str(csrc))
    monkeypatch.setattr(cuda_build, "SO", str(tmp_path / "package" / "lib.so"))
    monkeypatch.setattr(cuda_build, "SO_CHECKED", str(tmp_path / "package" / "lib_checked.so"))
    monkeypatch.setenv("NVCC", str(nvcc))
    monkeypatch.delenv("WWWS_NVCC_EXTRA", raising=False)

    def compiled(**how):
        log.write_text("")
        cuda_build.build(**how)
        return sorted(log.read_text().split())

    def touch(name):
        path = csrc / name
        later = os.path.getmtime(cuda_build.SO) + 10         # (as if saved after the build, whatever the clock's steps)
        for p in (tmp_path / "package").rglob("*"):
            if p != path and p.stat().st_mtime > later - 5:
                os.utime(p, (later - 9, later - 9))
        os.utime(path, (later, later))

    return compiled, touch, csrc


EVERY = ["other.cu", "rows.cu", "rows_tree.cu"]


def test_a_source_that_another_includes(tree):
    compiled, touch, csrc = tree
    assert compiled() == EVERY
    assert compiled() == []
    touch("rows.cu")
    assert compiled() == ["rows.cu", "rows_tree.cu"]


def test_a_header_and_an_own_change(tree):
    compiled, touch, csrc = tree
    compiled()
    touch("common.cuh")
    assert compiled() == ["rows.cu", "rows_tree.cu"]
    (csrc.parent / "lib.so").unlink()
    (csrc / "other.cu").unlink()
    (csrc / "more.cu").write_text('extern "C" int more() { return 3; }\n')
    assert "other.cu" not in compiled()


def test_other_flags(tree, monkeypatch):
    """Objects and libraries made with other flags are not taken for these."""
    compiled, touch, csrc = tree
    compiled()
    monkeypatch.setenv("WWWS_NVCC_EXTRA", "-DMORE=1")
    assert compiled() == EVERY
    monkeypatch.delenv("WWWS_NVCC_EXTRA")
    assert cuda_build.needs_build()
    assert compiled() == []                                  # the first objects are still good: linked again
    assert not cuda_build.needs_build()
    monkeypatch.setattr(cuda_build, "NVCC_FLAGS", cuda_build.NVCC_FLAGS + ["-DCHANGED"])
    assert compiled() == EVERY
    assert compiled(checked=True) == EVERY
    assert compiled(checked=True) == []
