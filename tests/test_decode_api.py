"""The host side of the decoder's C ABI without a GPU: refusals and edges, under the undefined-behaviour sanitizer, with every HIP
function and kernel launcher replaced by a stub that returns success."""
import os
import subprocess

from paper_2401_05031_amd import binding

CXX = "/opt/rocm/llvm/bin/clang++"
HERE = os.path.dirname(os.path.abspath(__file__))


def _run(*cmd):
    r = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert r.returncode == 0, r.stdout[-3000:]
    return r.stdout


def test_host_side_refuses_and_accepts_what_the_header_says(tmp_path):
    obj, stubs, exe = str(tmp_path / "api.o"), str(tmp_path / "stubs.c"), str(tmp_path / "api")
    san = ["-fsanitize=undefined", "-fno-sanitize-recover=undefined"]
    _run(CXX, "-std=c++17", "-O1", "-w", "-I/opt/rocm/include", *san, "-c", os.path.join(HERE, "decode_api_main.cpp"), "-o", obj)
    undefined = {l.split()[-1] for l in _run("nm", "-u", obj).splitlines()}
    with open(stubs, "w") as f:
        for s in sorted(undefined):
            if s.startswith("hip") or s.startswith("_ZN4otas"):
                f.write(f"long {s}(void) {{ return 0; }}\n")
    _run("gcc", "-w", "-c", stubs, "-o", stubs + ".o")
    _run(CXX, obj, stubs + ".o", *san, "-o", exe)
    assert "decode api ok" in _run(exe)


def test_limits_are_those_of_the_header():
    text = open(os.path.join(os.path.dirname(HERE), "include", "otas_decode.h")).read()
    for name in ("OTAS_DECODE_ARGUMENTS", "OTAS_MAX_LONG_SEQ", "OTAS_MAX_TREE_NODES"):
        assert f"#define {name} {getattr(binding, name)}" in text
