"""The host side of the entry points with norms of heads, windows and the cache in 4 bits without a GPU: refusals, edges and how calls are cut
up, under the undefined-behaviour sanitizer, with every HIP function and kernel launcher replaced by a stub that returns success."""
import os

from paper_2401_05031_amd import binding
from tests.test_decode_api import CXX, HERE, _run


def test_host_side_refuses_and_accepts_what_the_header_says(tmp_path):
    obj, stubs, exe = str(tmp_path / "api.o"), str(tmp_path / "stubs.c"), str(tmp_path / "api")
    san = ["-fsanitize=undefined", "-fno-sanitize-recover=undefined"]
    _run(CXX, "-std=c++17", "-O1", "-w", "-I/opt/rocm/include", *san, "-c", os.path.join(HERE, "window_api_main.cpp"), "-o", obj)
    undefined = {line.split()[-1] for line in _run("nm", "-u", obj).splitlines()}
    with open(stubs, "w") as f:
        for s in sorted(undefined):
            if s.startswith("hip") or s.startswith("_ZN4otas"):
                f.write(f"long {s}(void) {{ return 0; }}\n")
    _run("gcc", "-w", "-c", stubs, "-o", stubs + ".o")
    _run(CXX, obj, stubs + ".o", *san, "-o", exe)
    assert "window api ok" in _run(exe)


def test_limits_are_those_of_the_header():
    text = open(os.path.join(os.path.dirname(HERE), "include", "otas_decode.h")).read()
    assert f"#define OTAS_CACHE4_GROUP {binding.OTAS_CACHE4_GROUP}" in text
