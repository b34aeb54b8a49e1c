"""CPU-side checks of the dense operators' C entry points: bad arguments are
refused on the host before anything reaches the device, and workspace sizes
do not fall when an argument grows."""
import ctypes
import itertools
import os

import pytest

from paper_2512_00385_amd import ezsp

pytestmark = pytest.mark.skipif(not os.path.exists(ezsp.LIB_PATH),
                                reason="libezsp.so not built")

FAKE = ctypes.c_void_p(0x1000)  # never dereferenced: validation fails first
E, W = ezsp.ERR_INVALID_ARG, ezsp.ERR_WORKSPACE
BF, F32 = 0, 1


def norm(x=FAKE, ldx=8, tx=BF, n=4, d=8, eps=1e-5, y=FAKE, ldy=8, ty=F32):
    return ezsp.load().ezsp_layer_norm(x, ldx, tx, n, d, None, None, eps, y,
                                       ldy, ty, None, None, None)


def norm_backward(dy=FAKE, lddy=8, ty=BF, x=FAKE, ldx=8, tx=BF, n=4, d=8,
                  mean=FAKE, rstd=FAKE, dres=None, lddres=8, dx=FAKE, lddx=8,
                  dw=FAKE, db=FAKE, ws=FAKE, nbytes=1 << 40):
    return ezsp.load().ezsp_layer_norm_backward(
        dy, lddy, ty, x, ldx, tx, n, d, None, mean, rstd, dres, lddres, dx,
        lddx, dw, db, ws, nbytes, None)


@pytest.mark.parametrize("bad", [
    dict(x=None), dict(y=None), dict(n=0), dict(n=2 ** 31), dict(d=0),
    dict(d=16385, ldx=20000, ldy=20000), dict(ldx=7), dict(ldy=7),
    dict(tx=2), dict(ty=-1), dict(eps=-1e-5), dict(eps=float("nan")),
    dict(eps=float("inf"))])
def test_layer_norm_refuses(bad):
    assert norm(**bad) == E
    assert ezsp.last_error()


@pytest.mark.parametrize("bad", [
    dict(dy=None), dict(x=None), dict(mean=None), dict(rstd=None),
    dict(ws=None), dict(n=0), dict(d=0), dict(d=16385, ldx=1 << 20,
                                              lddy=1 << 20, lddx=1 << 20),
    dict(ldx=7), dict(lddy=7), dict(lddx=7), dict(dres=FAKE, lddres=7),
    dict(dres=FAKE, dx=None), dict(tx=5), dict(ty=9),
    dict(dx=None, dw=None, db=None)])
def test_layer_norm_backward_refuses(bad):
    assert norm_backward(**bad) == E
    assert ezsp.last_error()


def test_layer_norm_backward_workspace():
    assert norm_backward(nbytes=16) == W
    q = ezsp.load().ezsp_layer_norm_backward_workspace_size
    assert q(0, 8) == 0 and q(8, 0) == 0 and q(8, 16385) == 0
    assert q(2 ** 31, 8) == 0


NS = [1, 7, 64, 1000, 1024, 1025, 20_000, 300_000, 1_300_000, 40_000_000]
QUERIES = {
    "ezsp_layer_norm_backward_workspace_size":
        (NS, [1, 7, 8, 65, 1000, 2048, 2049, 16384]),
}


@pytest.mark.parametrize("name", QUERIES)
def test_sizes_grow(name):
    query = getattr(ezsp.load(), name)
    axes = QUERIES[name]
    for at in itertools.product(*(range(len(a)) for a in axes)):
        here = query(*(a[i] for a, i in zip(axes, at)))
        assert here > 0
        for j, i in enumerate(at):
            if i + 1 < len(axes[j]):
                more = list(at)
                more[j] += 1
                assert query(*(a[m] for a, m in zip(axes, more))) >= here
