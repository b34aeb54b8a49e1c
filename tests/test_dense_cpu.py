"""The dense operators' kernels on the CPU, from their own source with threads
for lanes (cpu_lanes/lanes.h): every index into LDS arrays and every read of
the operands under a sanitizer, results compared with the formulas.  Blocks go
through several tiles of unaligned operands; the kernel for few rows meets
last blocks of fewer columns than a lane's vector; layer norm and the one-pass
backward meet rows and tables of less than a vector."""
import os
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
CLANG = "/opt/rocm/llvm/bin/clang++"  # the kernels' vector types are clang's

pytestmark = pytest.mark.skipif(not os.path.exists(CLANG),
                                reason="no clang++")


@pytest.fixture(scope="module")
def programs(tmp_path_factory):
    out = tmp_path_factory.mktemp("dense")
    # (without optimisation this compiler returns bfloat16 vectors wrongly)
    builds = {name: subprocess.Popen(
        [CLANG, "-x", "c++", "-std=c++20", "-O1", "-w",
         "-I/opt/rocm/include", "-pthread", "-fsanitize=address,bounds",
         "-fno-sanitize-recover=bounds",
         os.path.join(HERE, "cpu_lanes", name + ".cpp"),
         "-o", str(out / name)]) for name in ("dense", "rows")}
    assert all(p.wait(timeout=240) == 0 for p in builds.values())
    return out


@pytest.mark.parametrize("program,argument,cases",
                         [("dense", "few", 18), ("dense", "tiles", 10),
                          ("rows", "", 48)])
def test_indexes_and_results(programs, program, argument, cases):
    run = subprocess.run([str(programs / program), argument],
                         capture_output=True, text=True, timeout=240)
    assert run.returncode == 0, run.stdout + run.stderr[-2000:]
    lines = run.stdout.splitlines()
    assert len(lines) == cases
    assert all(line.endswith(": 0 wrong") for line in lines), run.stdout
