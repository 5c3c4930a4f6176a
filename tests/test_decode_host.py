"""Host arithmetic of the decoder's operators without a GPU (decode_host_main.cpp)."""
import os

from tests.test_decode_api import CXX, HERE, _run


def test_host_arithmetic(tmp_path):
    obj, stubs, exe = str(tmp_path / "host.o"), str(tmp_path / "stubs.c"), str(tmp_path / "host")
    san = ["-fsanitize=undefined", "-fno-sanitize-recover=undefined"]
    _run(CXX, "-std=c++17", "-O1", "-w", "-I/opt/rocm/include", *san, "-c", os.path.join(HERE, "decode_host_main.cpp"), "-o", obj)
    undefined = {line.split()[-1] for line in _run("nm", "-u", obj).splitlines()}
    with open(stubs, "w") as f:
        for s in sorted(undefined):
            if s.startswith("hip") or s.startswith("_ZN4otas"):
                f.write(f"long {s}(void) {{ return 0; }}\n")
    _run("gcc", "-w", "-c", stubs, "-o", stubs + ".o")
    _run(CXX, obj, stubs + ".o", *san, "-o", exe)
    assert "decode host ok" in _run(exe)
