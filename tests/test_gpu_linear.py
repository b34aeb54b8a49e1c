"""ezsp_linear and its backward pass against the formulas in 64 bits (bounds
in dense_bounds), bit for bit where small integers make every sum exact."""
import pytest
import torch

from dense_bounds import (BF, F32, U, act64, act_error, act_grad64, check,
                          generator, integers, normal, sum_error)
from paper_2512_00385_amd import ezsp

pytestmark = pytest.mark.gpu

ACTS = ["none", "relu", "gelu", "silu"]
# (n, d_in, d_out): one token, single values, every tile of the kernels and
# one row or column off, lengths that fill no vector, long sums
SIZES = [
    (1, 1, 1), (1, 8, 8), (1, 4096, 512), (2, 7, 3), (3, 300, 1000),
    (8, 1024, 96), (16, 520, 128), (17, 64, 40), (31, 65, 33), (32, 128, 64),
    (33, 40, 31), (64, 256, 256), (65, 1000, 72), (100, 16, 16),
    (128, 64, 128), (129, 72, 136), (130, 4, 6), (257, 6, 32), (300, 515, 77),
    (500, 32, 65), (511, 136, 264), (1000, 33, 1), (1000, 1, 50),
    (1003, 128, 32), (2000, 24, 48), (4100, 64, 130),
    # few columns: each split of the one-pass backward
    (7, 12, 20), (8, 5, 3), (65, 31, 33), (700, 32, 128), (700, 20, 250),
    (700, 30, 400), (700, 60, 64), (700, 64, 500), (700, 100, 30),
    (700, 128, 100), (700, 97, 256), (20_000, 3, 7),
    # few rows: columns and sums that fill no step, wide tables of weights
    (1, 33, 9), (5, 70, 37), (48, 129, 333), (64, 8192, 16), (2, 4097, 70),
    (1, 40, 16_400), (17, 40, 33_000), (40, 24, 40_001),
]


@pytest.fixture(scope="module", autouse=True)
def gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    ezsp.load()
    yield


def tensors(n, k, m, ty, seed, make=normal):
    g = generator(seed)
    if make is integers:
        return (integers(g, (n, k), 2, ty), integers(g, (k, m), 2, ty),
                integers(g, (m,), 5, F32), integers(g, (n, m), 4, ty))
    return (normal(g, (n, k), ty), normal(g, (k, m), ty, k ** -0.5),
            normal(g, (m,), F32), normal(g, (n, m), ty))


def check_forward(x, w, b, act, res, out, z):
    xd, wd = x.double(), w.double()
    rz = xd @ wd
    mag = xd.abs() @ wd.abs()
    if b is not None:
        rz = rz + b.double()
        mag = mag + b.double().abs()
    ez = sum_error(x.shape[1], mag)
    if z is not None:
        check(z, rz, ez, "z")
    ry = act64(rz, act)
    ey = ez if act == "none" else act_error(rz, ez)
    if res is not None:
        ry = ry + res.double()
        ey = ey + 2 * U * (ry.abs() + res.double().abs() + ey)
    check(out, ry, ey, "y")


@pytest.mark.parametrize("ty,out", [(BF, BF), (BF, F32), (F32, F32)])
@pytest.mark.parametrize("n,k,m", SIZES)
def test_forward(n, k, m, ty, out):
    x, w, b, r = tensors(n, k, m, ty, n + k + m)
    act = ACTS[(n + k + m) % 4]
    y, z = ezsp.linear(x, w, b, act=act, residual=r.to(out), out_dtype=out,
                       want_z=True)
    assert y.dtype == out and z.dtype == ty
    check_forward(x, w, b, act, r.to(out), y, z)
    plain = ezsp.linear(x, w, out_dtype=out)
    check_forward(x, w, None, "none", None, plain, None)


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("ty", [BF, F32])
def test_forward_activations(act, ty):
    x, w, b, _ = tensors(200, 64, 80, ty, 3)
    x = (x * 6).to(ty)  # well into both tails
    y, z = ezsp.linear(x, w, b, act=act, want_z=True)
    check_forward(x, w, b, act, None, y, z)


# sums exact in fp32 whatever their order: results are the exact ones,
# rounded; sizes that reach the largest tiles and split sums too
EXACT = SIZES + [(4096, 64, 3200), (3333, 200, 4112), (70, 20_000, 40),
                 (1, 65_536, 24), (20, 30_001, 9), (50_021, 16, 24),
                 # large and unaligned: packed, whole and in chunks
                 (5001, 1021, 515), (190_001, 259, 264), (30_003, 67, 1030)]


@pytest.mark.parametrize("ty", [BF, F32])
@pytest.mark.parametrize("n,k,m", EXACT)
def test_forward_exact(n, k, m, ty):
    x, w, b, r = tensors(n, k, m, ty, 7, integers)
    z = x.double() @ w.double() + b.double()
    assert float(z.abs().max()) < 2 ** 24
    y, got_z = ezsp.linear(x, w, b, act="relu", residual=r, want_z=True)
    assert torch.equal(got_z, z.to(ty))
    assert torch.equal(y, (z.clamp_min(0) + r.double()).to(ty))
    if ty == BF:
        y = ezsp.linear(x, w, b, out_dtype=F32)
        assert torch.equal(y, z.float())


def check_backward(dy, x, w, z, act, got):
    n, k = x.shape
    m = w.shape[1]
    ty = x.dtype
    xd, wd, dyd = x.double(), w.double(), dy.double()
    dz = dyd
    edz = torch.zeros_like(dz)
    if act != "none":
        zd = z.double()
        dz = dyd * act_grad64(zd, act)
        edz = dyd.abs() * act_error(zd, 0.0)
    dx, dw, db = got
    check(db, dz.sum(0), edz.sum(0) + sum_error(n, dz.abs().sum(0)), "db")
    if ty == BF:  # the products take dz as bfloat16
        edz = edz + 2.0 ** -8 * (dz.abs() + edz)
    top = dz.abs() + edz
    check(dx, dz @ wd.t(), edz @ wd.abs().t() +
          sum_error(m, top @ wd.abs().t()), "dx")
    check(dw, xd.t() @ dz, xd.abs().t() @ edz +
          sum_error(n, xd.abs().t() @ top), "dw")


@pytest.mark.parametrize("ty,ty_y", [(BF, BF), (BF, F32), (F32, F32)])
@pytest.mark.parametrize("n,k,m", SIZES)
def test_backward(n, k, m, ty, ty_y):
    x, w, b, dy = tensors(n, k, m, ty, n * 3 + k + m)
    act = ACTS[(n + k) % 4]
    z = (x.float() @ w.float() + b).to(ty)
    dy = normal(generator(n), (n, m), ty_y)
    got = ezsp.linear_backward(dy, x, w, z, act=act)
    assert got[0].dtype == ty and got[1].dtype == ty and got[2].dtype == F32
    check_backward(dy, x, w, z, act, got)


@pytest.mark.parametrize("ty", [BF, F32])
@pytest.mark.parametrize("n,k,m", EXACT)
def test_backward_exact(n, k, m, ty):
    x, w, b, _ = tensors(n, k, m, ty, 11, integers)
    g = generator(5)
    dy = integers(g, (n, m), 2, ty)
    z = integers(g, (n, m), 2, ty)
    dz = dy.double() * (z.double() > 0)
    dx, dw, db = ezsp.linear_backward(dy, x, w, z, act="relu")
    assert torch.equal(dx, (dz @ w.double().t()).to(ty))
    assert torch.equal(dw, (x.double().t() @ dz).to(ty))
    assert torch.equal(db, dz.sum(0).float())
    dx, dw, db = ezsp.linear_backward(dy, x, w)
    dz = dy.double()
    assert torch.equal(dx, (dz @ w.double().t()).to(ty))
    assert torch.equal(dw, (x.double().t() @ dz).to(ty))
    assert torch.equal(db, dz.sum(0).float())


def test_gradients_asked_for_alone():
    x, w, b, dy = tensors(333, 48, 56, BF, 2)
    z = ezsp.linear(x, w, b, act="silu", want_z=True)[1]
    dx, dw, db = ezsp.linear_backward(dy, x, w, z, act="silu")
    for i, want in enumerate(("want_dx", "want_dw", "want_db")):
        opts = dict(want_dx=False, want_dw=False, want_db=False)
        opts[want] = True
        got = ezsp.linear_backward(dy, x, w, z, act="silu", **opts)
        assert torch.equal(got[i], (dx, dw, db)[i])
        assert all(got[j] is None for j in range(3) if j != i)


@pytest.mark.parametrize("act", ["none", "gelu", "silu"])
def test_gradient_against_differences(act):
    # central differences of sum(y * dy) in 64 bits
    x, w, b, dy = tensors(3, 5, 4, F32, 9)
    z = ezsp.linear(x, w, b, act=act, want_z=True)[1]
    grads = ezsp.linear_backward(dy, x, w, z, act=act)

    def loss(x, w, b):
        return float((act64(x @ w + b, act) * dy.double()).sum())
    h = 1e-5
    base = [t.double() for t in (x, w, b)]
    for which, grad in enumerate(grads):
        flat = base[which].flatten()
        for i in range(flat.numel()):
            val = []
            for s in (h, -h):
                moved = flat.clone()
                moved[i] += s
                args = list(base)
                args[which] = moved.reshape(base[which].shape)
                val.append(loss(*args))
            num = (val[0] - val[1]) / (2 * h)
            # differences: h^2 / 6 of the third derivative and 1e-15 / h;
            # the gradient itself: fp32 and z rounded to it
            assert abs(num - float(grad.flatten()[i])) < 2e-5


@pytest.mark.parametrize("ty", [BF, F32])
def test_strides_and_odd_alignment(ty):
    g = generator(4)
    wide = normal(g, (150, 131), ty)
    x = wide[:, 5:69]                      # odd offset, odd distance
    w, b = normal(g, (64, 48), ty, 0.125), normal(g, (48,), F32)
    r = normal(g, (150, 99), ty)[:, 1:49]
    ref = ezsp.linear(x.contiguous(), w, b, act="silu",
                      residual=r.contiguous(), want_z=True)
    got = ezsp.linear(x, w, b, act="silu", residual=r, want_z=True)
    for p, q in zip(got, ref):
        assert torch.equal(p, q)
    # other orders are copied
    got = ezsp.linear(x.t().contiguous().t(), w.t().contiguous().t(), b,
                      act="silu", residual=r, want_z=True)
    for p, q in zip(got, ref):
        assert torch.equal(p, q)
    dy, z = normal(g, (150, 60), ty)[:, 3:51], ref[1]
    zs = torch.cat([z, z], 1)[:, 48:]
    ref = ezsp.linear_backward(dy.contiguous(), x.contiguous(), w, z,
                               act="silu")
    got = ezsp.linear_backward(dy, x, w, zs, act="silu")
    for p, q in zip(got, ref):
        assert torch.equal(p, q)


@pytest.mark.parametrize("ty,code", [(BF, 0), (F32, 1)])
@pytest.mark.parametrize("n,k,m", [(37, 24, 40), (37, 25, 41), (1, 64, 8),
                                   (5, 8, 3), (200, 64, 100)])
def test_nothing_past_the_rows_is_written(n, k, m, ty, code):
    lib = ezsp.load()
    g = generator(8)
    x, w = normal(g, (n, k), ty), normal(g, (k, m), ty)
    b = normal(g, (m,), F32)
    ldy, ldz, ldx = m + 5, m + 3, k + 7
    y = torch.full((n + 2, ldy), 7.0, dtype=ty, device="cuda")
    z = torch.full((n + 2, ldz), 7.0, dtype=ty, device="cuda")
    nb = lib.ezsp_linear_workspace_size(n, k, m)
    ws = torch.empty(nb, dtype=torch.uint8, device="cuda")
    st = ezsp._stream(x.device)
    rc = lib.ezsp_linear(x.data_ptr(), k, n, k, m, code, w.data_ptr(),
                         b.data_ptr(), 3, None, 0, y.data_ptr(), ldy, code,
                         z.data_ptr(), ldz, ws.data_ptr(), nb, st)
    assert rc == ezsp.OK, ezsp.last_error()
    ry, rz = ezsp.linear(x, w, b, act="silu", want_z=True)
    for t, ref in ((y, ry), (z, rz)):
        assert torch.equal(t[:n, :m], ref)
        assert bool((t[:, m:] == 7.0).all()) and bool((t[n:] == 7.0).all())
    dx = torch.full((n + 2, ldx), 7.0, dtype=ty, device="cuda")
    dw = torch.full((k * m + 64,), 7.0, dtype=ty, device="cuda")
    nb = lib.ezsp_linear_backward_workspace_size(n, k, m, code)
    ws = torch.empty(nb, dtype=torch.uint8, device="cuda")
    rc = lib.ezsp_linear_backward(
        ry.data_ptr(), m, code, x.data_ptr(), k, n, k, m, code, w.data_ptr(),
        rz.data_ptr(), m, 3, dx.data_ptr(), ldx, dw.data_ptr(), None,
        ws.data_ptr(), nb, st)
    assert rc == ezsp.OK, ezsp.last_error()
    rdx, rdw, _ = ezsp.linear_backward(ry, x, w, rz, act="silu")
    assert torch.equal(dx[:n, :k], rdx) and torch.equal(dw[:k * m],
                                                        rdw.flatten())
    assert bool((dx[:, k:] == 7.0).all()) and bool((dx[n:] == 7.0).all())
    assert bool((dw[k * m:] == 7.0).all())


@pytest.mark.parametrize("n,k,m", [(40, 40, 40), (300, 72, 136),
                                   (13, 40, 48), (40, 33, 47)])
def test_infinities_and_nan_stay_where_they_belong(n, k, m):
    # a row of x reaches its row of y, a column of w its column, nothing else
    x, w, b, dy = tensors(n, k, m, BF, 6)
    clean = ezsp.linear(x, w, b)
    x2, w2 = x.clone(), w.clone()
    x2[n - 1, k - 1] = float("nan")
    w2[k - 1, m - 1] = float("inf")
    y = ezsp.linear(x2, w2, b)
    assert bool(y[n - 1].isnan().all())
    assert not bool(y[:n - 1, m - 1].isfinite().any())
    assert torch.equal(y[:n - 1, :m - 1], clean[:n - 1, :m - 1])
    dx, dw, db = ezsp.linear_backward(dy, x, w)
    dy2 = dy.clone()
    dy2[n - 1, m - 1] = float("nan")
    ex, ew, eb = ezsp.linear_backward(dy2, x, w)
    assert bool(ex[n - 1].isnan().all()) and bool(ew[:, m - 1].isnan().all())
    assert torch.equal(ex[:n - 1], dx[:n - 1])
    assert torch.equal(ew[:, :m - 1], dw[:, :m - 1])
    assert torch.equal(eb[:m - 1], db[:m - 1]) and bool(eb[m - 1].isnan())


def test_rows_beyond_32_bit_offsets():
    # x, y of more than 2^32 bytes: the last rows are as they should be
    n, k, m = 70_000_001, 8, 32
    x = torch.ones((n, k), dtype=BF, device="cuda")
    x[-3:] = 2.0
    w = integers(generator(3), (k, m), 2, BF)
    y = ezsp.linear(x, w)
    s = w.float().sum(0)
    assert torch.equal(y[-3:].float(), (2 * s).expand(3, m))
    assert torch.equal(y[-5:-3].float(), s.expand(2, m))
    assert torch.equal(y[:2].float(), s.expand(2, m))
    dx, dw, db = ezsp.linear_backward(y, x, w)
    ref = (y[-4:].double() @ w.double().t()).to(BF)
    assert torch.equal(dx[-4:], ref)


def test_same_results_every_run_and_on_a_side_stream():
    x, w, b, dy = tensors(40_001, 64, 96, BF, 3)
    z = ezsp.linear(x, w, b, act="gelu", want_z=True)[1]
    a = ezsp.linear_backward(dy, x, w, z, act="gelu")
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        c = ezsp.linear_backward(dy, x, w, z, act="gelu")
    side.synchronize()
    for p, q in zip(a, c):
        assert torch.equal(p, q)


def test_residual_may_be_the_output():
    x, w, b, r = tensors(300, 64, 48, BF, 12)
    ref = ezsp.linear(x, w, b, residual=r)
    lib = ezsp.load()
    nb = lib.ezsp_linear_workspace_size(300, 64, 48)
    ws = torch.empty(nb, dtype=torch.uint8, device="cuda")
    rc = lib.ezsp_linear(x.data_ptr(), 64, 300, 64, 48, 0, w.data_ptr(),
                         b.data_ptr(), 0, r.data_ptr(), 48, r.data_ptr(), 48,
                         0, None, 0, ws.data_ptr(), nb, ezsp._stream(x.device))
    assert rc == ezsp.OK and torch.equal(r, ref)


def test_captured_in_a_graph():
    x, w, b, dy = tensors(5000, 32, 64, BF, 13)

    def step():
        y, z = ezsp.linear(x, w, b, act="silu", want_z=True)
        return (y, z) + ezsp.linear_backward(dy, x, w, z, act="silu")
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for seed in (21, 22, 23):
        x.copy_(normal(generator(seed), x.shape, BF))
        ref = step()
        graph.replay()
        torch.cuda.synchronize()
        for p, q in zip(out, ref):
            assert torch.equal(p, q)


def test_refusals():
    x, w, b, r = tensors(4, 8, 8, BF, 1)
    for bad in (dict(x=x.cpu()), dict(x=x.half()), dict(w=w.float()),
                dict(bias=b.bfloat16()), dict(residual=r.float()),
                dict(out_dtype=torch.float16)):
        args = dict(x=x, w=w, bias=b)
        args.update(bad)
        with pytest.raises(TypeError):
            ezsp.linear(**args)
    for bad in (dict(w=w[:7]), dict(bias=b[:7]), dict(act="tanh"),
                dict(residual=r[:3]), dict(x=x[0])):
        args = dict(x=x, w=w, bias=b)
        args.update(bad)
        with pytest.raises(ValueError):
            ezsp.linear(**args)
    with pytest.raises(TypeError):  # fp32 inputs do not narrow
        ezsp.linear(x.float(), w.float(), out_dtype=BF)
    with pytest.raises(ezsp.EzspError):
        ezsp.linear(x[:0], w)
    with pytest.raises(ezsp.EzspError):  # the activation's z is missing
        ezsp.linear_backward(r, x, w, act="silu")
    with pytest.raises(ezsp.EzspError):
        ezsp.linear_backward(r, x, w, want_dx=False, want_dw=False,
                             want_db=False)
    with pytest.raises(ValueError):
        ezsp.linear_backward(r[:3], x, w)
