"""The dense operators' kernels on the CPU, from their own source with threads
for lanes (cpu_lanes/lanes.h): every index into LDS arrays and every read of
the operands under a sanitizer, results on integers compared for equality.
Blocks go through several tiles of unaligned operands; the kernel for few rows
meets last blocks of fewer columns than a lane's vector."""
import os
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
CLANG = "/opt/rocm/llvm/bin/clang++"  # the kernels' vector types are clang's

pytestmark = pytest.mark.skipif(not os.path.exists(CLANG),
                                reason="no clang++")


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("dense") / "dense")
    subprocess.run([CLANG, "-x", "c++", "-std=c++20", "-O0", "-w",
                    "-I/opt/rocm/include", "-pthread",
                    "-fsanitize=address,bounds",
                    "-fno-sanitize-recover=bounds",
                    os.path.join(HERE, "cpu_lanes", "dense.cpp"), "-o", out],
                   check=True, timeout=240)
    return out


@pytest.mark.parametrize("cases,least", [("few", 18), ("tiles", 10)])
def test_indexes_and_results(program, cases, least):
    run = subprocess.run([program, cases], capture_output=True, text=True,
                         timeout=240)
    assert run.returncode == 0, run.stdout + run.stderr[-2000:]
    lines = run.stdout.splitlines()
    assert len(lines) == least
    assert all(line.endswith(": 0 wrong") for line in lines), run.stdout
