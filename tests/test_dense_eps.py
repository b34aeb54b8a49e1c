"""Layer norm's eps is held in fp32: values that overflow there would give the
bias for every row, values that vanish NaN for a constant one."""
import ctypes
import os

import pytest

from paper_2512_00385_amd import ezsp

pytestmark = pytest.mark.skipif(not os.path.exists(ezsp.LIB_PATH),
                                reason="libezsp.so not built")

FAKE = ctypes.c_void_p(0x1000)


def norm(eps):
    return ezsp.load().ezsp_layer_norm(FAKE, 8, 0, 4, 8, None, None, eps,
                                       FAKE, 8, 1, None, None, None)


@pytest.mark.parametrize("eps", [1e39, 1.7e308, 1e-46, 5e-324])
def test_eps_that_fp32_cannot_hold(eps):
    assert norm(eps) == ezsp.ERR_INVALID_ARG
    assert "eps" in ezsp.last_error()
