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


def lin(x=FAKE, ldx=8, n=4, d_in=8, d_out=16, ty=BF, w=FAKE, act=0, res=None,
        ldr=16, y=FAKE, ldy=16, ty_y=BF, z=None, ldz=16, ws=FAKE,
        nbytes=1 << 40):
    return ezsp.load().ezsp_linear(x, ldx, n, d_in, d_out, ty, w, None, act,
                                   res, ldr, y, ldy, ty_y, z, ldz, ws, nbytes,
                                   None)


def lin_backward(dy=FAKE, lddy=16, ty_y=BF, x=FAKE, ldx=8, n=4, d_in=8,
                 d_out=16, ty=BF, w=FAKE, z=FAKE, ldz=16, act=3, dx=FAKE,
                 lddx=8, dw=FAKE, db=FAKE, ws=FAKE, nbytes=1 << 40):
    return ezsp.load().ezsp_linear_backward(
        dy, lddy, ty_y, x, ldx, n, d_in, d_out, ty, w, z, ldz, act, dx, lddx,
        dw, db, ws, nbytes, None)


def gated(x=FAKE, ldx=8, n=4, d_in=8, d_out=16, ty=BF, wg=FAKE, wu=FAKE,
          act=3, h=FAKE, ldh=16, g=None, u=None, lds=16, ws=FAKE,
          nbytes=1 << 40):
    return ezsp.load().ezsp_gated_ff(x, ldx, n, d_in, d_out, ty, wg, None, wu,
                                     None, act, h, ldh, g, u, lds, ws, nbytes,
                                     None)


def gated_backward(dh=FAKE, lddh=16, x=FAKE, ldx=8, n=4, d_in=8, d_out=16,
                   ty=BF, wg=FAKE, wu=FAKE, g=FAKE, u=FAKE, lds=16, act=3,
                   dx=FAKE, lddx=8, dw=FAKE, db=FAKE, ws=FAKE,
                   nbytes=1 << 40):
    return ezsp.load().ezsp_gated_ff_backward(
        dh, lddh, x, ldx, n, d_in, d_out, ty, wg, wu, g, u, lds, act, dx,
        lddx, dw, dw, db, db, ws, nbytes, None)


SHARED = [dict(x=None), dict(ws=None), dict(n=0), dict(n=2 ** 31),
          dict(d_in=0), dict(d_out=0),
          dict(d_in=65537, ldx=1 << 20, lddx=1 << 20),
          dict(ldx=7), dict(ty=2), dict(ty=-1), dict(act=4), dict(act=-1)]


def no_lddx(bad):
    return {k: v for k, v in bad.items() if k != "lddx"}


@pytest.mark.parametrize("bad", SHARED + [
    dict(w=None), dict(y=None), dict(ldy=15), dict(res=FAKE, ldr=15),
    dict(z=FAKE, ldz=15), dict(ty=F32, ty_y=BF), dict(ty_y=7)])
def test_linear_refuses(bad):
    assert lin(**no_lddx(bad)) == E
    assert ezsp.last_error()


@pytest.mark.parametrize("bad", SHARED + [
    dict(dy=None), dict(w=None), dict(z=None), dict(ldz=15), dict(lddy=15),
    dict(lddx=7), dict(ty=F32, ty_y=BF), dict(dx=None, dw=None, db=None)])
def test_linear_backward_refuses(bad):
    assert lin_backward(**bad) == E
    assert ezsp.last_error()


@pytest.mark.parametrize("bad", SHARED + [
    dict(wg=None), dict(wu=None), dict(h=None), dict(ldh=15),
    dict(g=FAKE, lds=15), dict(u=FAKE, lds=15)])
def test_gated_refuses(bad):
    assert gated(**no_lddx(bad)) == E
    assert ezsp.last_error()


@pytest.mark.parametrize("bad", SHARED + [
    dict(dh=None), dict(wg=None), dict(wu=None), dict(g=None), dict(u=None),
    dict(lddh=15), dict(lds=15), dict(lddx=7),
    dict(dx=None, dw=None, db=None)])
def test_gated_backward_refuses(bad):
    assert gated_backward(**bad) == E
    assert ezsp.last_error()


def test_product_workspaces():
    assert lin(nbytes=16) == W and lin_backward(nbytes=16) == W
    assert gated(nbytes=16) == W and gated_backward(nbytes=16) == W
    lib = ezsp.load()
    for name in ("ezsp_linear_workspace_size", "ezsp_gated_ff_workspace_size"):
        q = getattr(lib, name)
        assert q(0, 8, 8) == 0 and q(8, 0, 8) == 0 and q(8, 8, 65537) == 0
    for name in ("ezsp_linear_backward_workspace_size",
                 "ezsp_gated_ff_backward_workspace_size"):
        q = getattr(lib, name)
        assert q(0, 8, 8, 0) == 0 and q(8, 8, 8, 2) == 0


NS = [1, 7, 64, 1000, 1024, 1025, 20_000, 300_000, 1_300_000, 40_000_000]
WIDTHS = [1, 7, 8, 9, 32, 33, 128, 515, 4096, 8192, 65536]
QUERIES = {
    "ezsp_layer_norm_backward_workspace_size":
        (NS, [1, 7, 8, 65, 1000, 2048, 2049, 16384]),
    "ezsp_linear_workspace_size": (NS, WIDTHS, WIDTHS),
    "ezsp_linear_backward_workspace_size": (NS, WIDTHS, WIDTHS, [BF, F32]),
    "ezsp_gated_ff_workspace_size": (NS, WIDTHS, WIDTHS),
    "ezsp_gated_ff_backward_workspace_size": (NS, WIDTHS, WIDTHS, [BF, F32]),
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
