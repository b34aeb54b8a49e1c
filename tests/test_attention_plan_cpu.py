"""What cross attention launches, on the CPU from its own source: the launches
are recorded (cpu_lanes/attn_plan.cpp), from the smallest sizes to the largest
that the entry points take; and the workspaces that hold their parts."""
import os
import subprocess

import pytest

from paper_2512_00385_amd import ezsp

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


def test_workspaces_hold_the_parts(lines):
    """And calls that cannot come in parts ask for no sums of these."""
    assert "workspaces: fit" in lines, "\n".join(lines[:20])


@pytest.mark.skipif(not os.path.exists(ezsp.LIB_PATH),
                    reason="libezsp.so not built")
def test_workspace_of_few_keys():
    """70,001 rows to 3 keys come in one part forward; backward 64 of the
    keys' sums and D."""
    lib = ezsp.load()
    assert lib.ezsp_cross_attention_workspace_size(70_001, 3, 2, 2, 16) < 4096
    assert lib.ezsp_cross_attention_backward_workspace_size(
        70_001, 3, 2, 2, 16) < 4 * (70_001 * 2 + 64 * 3 * 2 * 64) + 4096
