"""Cross attention's kernels on the CPU in every tile shape that the library
launches (cpu_lanes/attn_shapes.cpp): indexes under a sanitizer, results in
whole numbers compared with the formulas."""
import os
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
CLANG = "/opt/rocm/llvm/bin/clang++"  # the kernels' vector types are clang's

pytestmark = pytest.mark.skipif(not os.path.exists(CLANG),
                                reason="no clang++")


def test_every_shape(tmp_path):
    parts = range(5)  # of the shapes, compiled side by side

    def program(i):
        return str(tmp_path / f"attn_shapes{i}")
    source = os.path.join(HERE, "cpu_lanes", "attn_shapes.cpp")
    compilers = [subprocess.Popen(
        [CLANG, "-x", "c++", "-std=c++20", "-O1", "-w", f"-DPART={i}",
         "-I/opt/rocm/include", "-pthread", "-fsanitize=address,bounds",
         "-fno-sanitize-recover=bounds", source, "-o", program(i)])
        for i in parts]
    assert [p.wait(timeout=300) for p in compilers] == [0] * len(parts)
    runs = [subprocess.Popen([program(i)], stdout=subprocess.PIPE,
                             stderr=subprocess.PIPE, text=True)
            for i in parts]
    lines = []
    for run in runs:
        out, err = run.communicate(timeout=300)
        assert run.returncode == 0, out + err[-2000:]
        lines += out.splitlines()
    assert len(lines) == 14 * 3
    assert all(line.endswith(": 0 wrong") for line in lines), lines
