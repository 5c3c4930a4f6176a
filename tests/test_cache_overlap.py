"""Rows within a cache's keys or values are refused by every attention over one, as the header says, without a GPU (as test_window_api.py)."""
import os

import pytest

from tests.test_decode_api import CXX, HERE, _run


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    tmp_path = tmp_path_factory.mktemp("overlap")
    obj, stubs, exe = str(tmp_path / "api.o"), str(tmp_path / "stubs.c"), str(tmp_path / "api")
    san = ["-fsanitize=undefined", "-fno-sanitize-recover=undefined"]
    _run(CXX, "-std=c++17", "-O1", "-w", "-I/opt/rocm/include", *san, "-c", os.path.join(HERE, "cache_overlap_main.cpp"), "-o", obj)
    undefined = {line.split()[-1] for line in _run("nm", "-u", obj).splitlines()}
    with open(stubs, "w") as f:
        for s in sorted(undefined):
            if s.startswith("hip") or s.startswith("_ZN4otas"):
                f.write(f"long {s}(void) {{ return 0; }}\n")
    _run("gcc", "-w", "-c", stubs, "-o", stubs + ".o")
    _run(CXX, obj, stubs + ".o", *san, "-o", exe)
    return exe


@pytest.mark.parametrize("which", ["last tokens", "tree"])
def test_rows_within_a_cache_are_refused(program, which):
    assert "cache overlap ok" in _run(program, which)
