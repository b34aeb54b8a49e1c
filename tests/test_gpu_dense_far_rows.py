"""Tables of more than 2^32 bytes: rows far apart (also farther than the tile
kernel's 32-bit offsets reach) and many rows, inputs, outputs and workspace
matrices, through every kernel that serves.  On integers: sums are exact in
fp32, so results are compared for equality with 64-bit ones after one
rounding."""
import pytest
import torch

from dense_bounds import BF, F32, generator, integers
from paper_2512_00385_amd import ezsp

pytestmark = pytest.mark.gpu

CODE = {BF: 0, F32: 1}


@pytest.fixture(scope="module", autouse=True)
def gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    ezsp.load()
    yield
    torch.cuda.empty_cache()


def far(t, ld):
    """t as the first columns of rows ld apart, eight sevens after them."""
    n, d = t.shape
    table = torch.empty((n, ld), dtype=t.dtype, device=t.device)
    assert n * ld * t.element_size() > 2 ** 32
    table[:, :d] = t
    table[:, d:d + 8] = 7
    return table[:, :d]


def untouched(view):
    n, d = view.shape
    after = torch.as_strided(view, (n, 8), view.stride(),
                             view.storage_offset() + d)
    return bool((after == 7).all())


def call(name, query, sizes, *args):
    lib = ezsp.load()
    nb = getattr(lib, query)(*sizes)
    ws = torch.empty(nb, dtype=torch.uint8, device="cuda")
    rc = getattr(lib, name)(*args, ws.data_ptr(), nb,
                            ezsp._stream(ws.device))
    assert rc == ezsp.OK, ezsp.last_error()
    torch.cuda.synchronize()


# few rows, narrow, aligned tiles, unaligned tiles, packed; then farther apart
# than kFastLd (2^21 values)
FORWARD = [(50, 64, 40, 2 ** 26 + 1), (40_000, 24, 48, 60_000),
           (40_000, 128, 128, 60_000), (40_000, 100, 100, 60_001),
           (40_000, 1021, 515, 60_003), (2100, 100, 100, 2 ** 21 + 5),
           (1100, 24, 48, 2 ** 21 + 8)]


@pytest.mark.parametrize("ty", [BF, F32])
@pytest.mark.parametrize("n,k,m,ld", FORWARD)
def test_linear(n, k, m, ld, ty):
    g = generator(n + k)
    x, y = far(integers(g, (n, k), 2, ty), ld), \
        far(integers(g, (n, m), 4, ty), ld)  # y: first the residual
    w, b = integers(g, (k, m), 2, ty), integers(g, (m,), 5, F32)
    z = far(torch.zeros((n, m), dtype=ty, device="cuda"), ld)
    ref = x.double() @ w.double() + b.double()
    out = (ref.clamp_min(0) + y.double()).to(ty)
    assert torch.equal(ezsp.linear(x, w, b, "relu", y), out)
    call("ezsp_linear", "ezsp_linear_workspace_size", (n, k, m),
         x.data_ptr(), ld, n, k, m, CODE[ty], w.data_ptr(), b.data_ptr(), 1,
         y.data_ptr(), ld, y.data_ptr(), ld, CODE[ty], z.data_ptr(), ld)
    assert torch.equal(y, out) and torch.equal(z, ref.to(ty))
    assert untouched(y) and untouched(z)


# one pass, aligned tiles, unaligned tiles, packed; then beyond kFastLd
BACKWARD = [(40_000, 24, 48, 60_000), (40_000, 256, 128, 60_000),
            (40_000, 130, 100, 60_001), (40_000, 1021, 515, 60_003),
            (2100, 130, 100, 2 ** 21 + 5), (1100, 24, 48, 2 ** 21 + 8)]


@pytest.mark.parametrize("ty", [BF, F32])
@pytest.mark.parametrize("n,k,m,ld", BACKWARD)
def test_linear_backward(n, k, m, ld, ty):
    g = generator(n + k)
    x, dy, z = (far(integers(g, (n, d), 2, ty), ld) for d in (k, m, m))
    w = integers(g, (k, m), 2, ty)
    dz = dy.double() * (z > 0)
    dx = far(torch.zeros((n, k), dtype=ty, device="cuda"), ld)
    dw = torch.empty((k, m), dtype=ty, device="cuda")
    db = torch.empty(m, device="cuda")
    call("ezsp_linear_backward", "ezsp_linear_backward_workspace_size",
         (n, k, m, CODE[ty]), dy.data_ptr(), ld, CODE[ty], x.data_ptr(), ld, n,
         k, m, CODE[ty], w.data_ptr(), z.data_ptr(), ld, 1, dx.data_ptr(), ld,
         dw.data_ptr(), db.data_ptr())
    assert torch.equal(dx, (dz @ w.double().t()).to(ty)) and untouched(dx)
    assert torch.equal(dw, (x.double().t() @ dz).to(ty))
    assert torch.equal(db.double(), dz.sum(0))


@pytest.mark.parametrize("ty", [BF, F32])
@pytest.mark.parametrize("n,k,m,ld", BACKWARD)
def test_gated(n, k, m, ld, ty):
    g = generator(n + k)
    x, dh = (far(integers(g, (n, d), 1, ty), ld) for d in (k, m))
    w = [integers(g, (k, m), 2, ty) for _ in range(2)]
    s = [x.double() @ wi.double() for wi in w]
    h = far(torch.zeros((n, m), dtype=ty, device="cuda"), ld)
    call("ezsp_gated_ff", "ezsp_gated_ff_workspace_size", (n, k, m),
         x.data_ptr(), ld, n, k, m, CODE[ty], w[0].data_ptr(), None,
         w[1].data_ptr(), None, 1, h.data_ptr(), ld, None, None, 0)
    assert torch.equal(h, (s[0].clamp_min(0) * s[1]).to(ty)) and untouched(h)
    gate, up = (far(integers(g, (n, m), 2, ty), ld) for _ in range(2))
    dg = dh.double() * up.double() * (gate > 0)
    du = dh.double() * gate.double().clamp_min(0)
    ref = (dg @ w[0].double().t() + du @ w[1].double().t(),
           x.double().t() @ dg, x.double().t() @ du, dg.sum(0), du.sum(0))
    got = ezsp.gated_ff_backward(dh, x, *w, gate, up, act="relu")
    for name, p, r in zip(("dx", "dwg", "dwu", "dbg", "dbu"), got, ref):
        assert torch.equal(p, r.to(p.dtype)), name


@pytest.mark.parametrize("ty", [BF, F32])
@pytest.mark.parametrize("n,d,ld", [(40_000, 7, 60_000), (40_000, 100, 60_001),
                                    (40_000, 2049, 60_000),
                                    (2100, 520, 2 ** 21 + 5)])
def test_layer_norm(n, d, ld, ty):
    # against the same rows side by side
    g = generator(n + d)
    x, dy, dres = (torch.randn((n, d), generator=g, device="cuda").to(ty)
                   for _ in range(3))
    y, mean, rstd = ezsp.layer_norm(x, want_stats=True)
    ref = ezsp.layer_norm_backward(dy, x, mean, rstd, dres=dres)
    fx, fdy, fdres = (far(t, ld) for t in (x, dy, dres))
    got = ezsp.layer_norm_backward(fdy, fx, mean, rstd, dres=fdres)
    for p, q in zip(got, ref):
        assert torch.equal(p, q)
    call("ezsp_layer_norm_backward", "ezsp_layer_norm_backward_workspace_size",
         (n, d), fdy.data_ptr(), ld, CODE[ty], fx.data_ptr(), ld, CODE[ty], n,
         d, None, mean.data_ptr(), rstd.data_ptr(), fdres.data_ptr(), ld,
         fdres.data_ptr(), ld, None, None)
    assert torch.equal(fdres, ref[0]) and untouched(fdres)
    lib = ezsp.load()
    rc = lib.ezsp_layer_norm(fx.data_ptr(), ld, CODE[ty], n, d, None, None,
                             1e-5, fx.data_ptr(), ld, CODE[ty], None, None,
                             ezsp._stream(x.device))
    assert rc == ezsp.OK and torch.equal(fx, y) and untouched(fx)


@pytest.mark.parametrize("products", [1, 2])
def test_many_rows(products):
    # x, dx and dz beyond 2^32 bytes; a few rows at both ends are not zero
    n, k, m = 17_000_000, 136, 130
    g = generator(products)
    rows = torch.cat([torch.arange(3), torch.arange(n - 300, n)]).cuda()

    def table(d):
        t = torch.zeros((n, d), dtype=BF, device="cuda")
        t[rows] = integers(g, (len(rows), d), 2, BF)
        return t
    x, dy = table(k), table(m)
    assert x.numel() * 2 > 2 ** 32 and dy.numel() * 2 > 2 ** 32
    w = [integers(g, (k, m), 2, BF) for _ in range(products)]
    xs, ds = x[rows].double(), dy[rows].double()
    if products == 1:
        got = ezsp.linear_backward(dy, x, w[0])
        dz = [ds]
    else:
        gate, up = table(m), table(m)
        got = ezsp.gated_ff_backward(dy, x, *w, gate, up, act="relu")
        gs, us = gate[rows].double(), up[rows].double()
        dz = [ds * us * (gs > 0), ds * gs.clamp_min(0)]
    dx = sum(z @ wi.double().t() for z, wi in zip(dz, w))
    assert torch.equal(got[0][rows], dx.to(BF))
    got[0][rows] = 0
    assert not bool(got[0].any())
    for p in range(products):
        assert torch.equal(got[1 + p], (xs.t() @ dz[p]).to(BF))
        assert torch.equal(got[1 + products + p].double(), dz[p].sum(0))
    y = ezsp.linear(x, w[0])
    assert torch.equal(y[rows], (xs @ w[0].double()).to(BF))
    y[rows] = 0
    assert not bool(y.any())
