"""What cross attention launches, on the CPU from its own source: the launches
are recorded (cpu_lanes/attn_plan.cpp), from the smallest sizes to the largest
that the entry points take."""
import os
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
CLANG = "/opt/rocm/llvm/bin/clang++"  # the kernels' vector types are clang's

pytestmark = pytest.mark.skipif(not os.path.exists(CLANG),
                                reason="no clang++")


@pytest.fixture(scope="module")
def lines(tmp_path_factory):
    program = str(tmp_path_factory.mktemp("attn_plan") / "attn_plan")
    subprocess.run(
        [CLANG, "-x", "c++", "-std=c++20", "-O1", "-w", "-I/opt/rocm/include",
         "-pthread", os.path.join(HERE, "cpu_lanes", "attn_plan.cpp"), "-o",
         program], check=True, timeout=240)
    run = subprocess.run([program], capture_output=True, text=True,
                         timeout=240)
    assert run.returncode in (0, 1), run.stderr[-2000:]
    return run.stdout.splitlines()


def test_launches_fit(lines):
    """Threads along x stay below 2^32, as a launch needs."""
    assert any(x.startswith("launches of") and x.endswith(": fit")
               for x in lines), "\n".join(lines[:20])


def test_every_unit_has_one_block(lines):
    assert "units: one block each" in lines
