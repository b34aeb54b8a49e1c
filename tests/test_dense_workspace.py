"""Workspaces of the dense operators: what a call keeps there and no more."""
import os

import pytest

from paper_2512_00385_amd import ezsp

pytestmark = pytest.mark.skipif(not os.path.exists(ezsp.LIB_PATH),
                                reason="libezsp.so not built")

SIZE = {0: 2, 1: 4}  # bytes of a bfloat16, of an fp32 value
WIDTHS = [1, 7, 16, 31, 32, 33, 64, 65, 100, 128, 129, 200, 256, 257, 500, 512,
          513, 4096]


def padded(d):
    return (d + 7) // 8 * 8


@pytest.mark.parametrize("name,products", [("linear", 1), ("gated_ff", 2)])
@pytest.mark.parametrize("ty", SIZE)
@pytest.mark.parametrize("n", [65_536, 1_300_000])
def test_backward(name, products, ty, n):
    # dz, and the larger of a split product's parts (at most 128 MiB), the
    # one-pass kernel's (1024 blocks' sums of at most 128 x 256 or 64 x 512
    # values, in fp32, with a row for the bias) and, from 512 columns on,
    # twice an aligned copy of x (at most 256 MiB a product)
    query = getattr(ezsp.load(), f"ezsp_{name}_backward_workspace_size")
    for d_in in WIDTHS:
        for d_out in WIDTHS:
            parts = max(128 << 20, 1024 * 4 * 65 * 512)
            if d_out * products >= 512:
                copy = (n + 256) * padded(d_in) * SIZE[ty]
                parts = max(parts, min(2 * copy, products << 28))
            dz = n * products * padded(d_out) * SIZE[ty]
            assert query(n, d_in, d_out, ty) <= dz + parts + 4096, \
                (d_in, d_out)


@pytest.mark.parametrize("name,products", [("linear", 1), ("gated_ff", 2)])
def test_forward_of_few_columns(name, products):
    # sums too short to be split, too few columns to pack x for: an aligned
    # copy of the weights in half of it, at most
    query = getattr(ezsp.load(), f"ezsp_{name}_workspace_size")
    for n in (1000, 1_300_000, 2 ** 31 - 256):
        for d_in in (1, 32, 224):
            for d_out in (1, 64, 191 // products):
                copy = products * d_in * padded(d_out) * 4
                assert query(n, d_in, d_out) <= 2 * copy + 4096
