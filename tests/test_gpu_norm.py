"""Layer norm, forward and backward, against the formulas in 64 bits.

Tolerances.  u = 2^-24 is half an ulp of fp32, U the same of the output type
(2^-8 bfloat16).  A row of d values is summed in a tree over lanes, so the
sums carry at most (d / 64 + 16) u relative to the sum of magnitudes; the
centred variance and the products of a result add a few more.  C = 4 d / 64
+ 64 roundings cover each, and every element is compared with its own bound:
C u times the magnitudes that enter it, plus U of the result."""
import numpy as np
import pytest
import torch

from paper_2512_00385_amd import ezsp

pytestmark = pytest.mark.gpu

U32 = 2.0 ** -24
# of a type with p significant bits: 2^-p (bfloat16 has 8 of them)
HALF_ULP = {torch.float32: U32, torch.bfloat16: 2.0 ** -8}
BF, F32 = torch.bfloat16, torch.float32
EPS = 1e-5
# lengths: one value, a vector less one, exactly, plus one; every group of
# lanes; a block; the longest
WIDTHS = [1, 7, 8, 9, 16, 31, 32, 65, 127, 256, 511, 512, 520, 1000, 2048,
          2049, 4096, 5001, 8192, 16384]


@pytest.fixture(scope="module", autouse=True)
def gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    ezsp.load()
    yield


def make(n, d, tx, ty, seed):
    g = torch.Generator().manual_seed(seed)
    x = (torch.randn(n, d, generator=g) * 2 + 0.7).to(tx)
    dy = torch.randn(n, d, generator=g).to(ty)
    w = 1 + 0.3 * torch.randn(d, generator=g)
    b = torch.randn(d, generator=g)
    return x, dy, w, b


def forward64(x, w, b, eps):
    x = x.double()
    mean = x.mean(1, keepdim=True)
    xc = x - mean
    rstd = ((xc * xc).mean(1, keepdim=True) + eps) ** -0.5
    y = xc * rstd
    if w is not None:
        y = y * w.double()
    if b is not None:
        y = y + b.double()
    return y, mean[:, 0], rstd[:, 0]


def within(got, ref, mag, dtype, c):
    got = got.double().cpu()
    err = (got - ref).abs()
    tol = c * U32 * mag + HALF_ULP[dtype] * (ref.abs() + c * U32 * mag) + 1e-37
    assert bool((err <= tol).all()), float((err / tol).max())


def check_forward(x, w, b, got, c, eps=EPS):
    y, mean, rstd = got
    ry, rm, rr = forward64(x, w, b, eps)
    xd = x.double()
    big = xd.abs().mean(1)
    within(mean, rm, big, F32, c)
    # relative error of the variance: roundings of the centred values, which
    # inherit the mean's error
    amp = 1 + big * rr
    within(rstd, rr, rr * amp, F32, c)
    wd = torch.ones(x.shape[1]).double() if w is None else w.double()
    bd = torch.zeros(x.shape[1]).double() if b is None else b.double()
    mag = (((xd.abs() + big[:, None]) * rr[:, None]) * wd.abs() * amp[:, None]
           + bd.abs())
    within(y, ry, mag, y.dtype, c)


@pytest.mark.parametrize("tx,ty", [(BF, BF), (F32, BF), (F32, F32),
                                   (BF, F32)])
@pytest.mark.parametrize("d", WIDTHS)
def test_forward(d, tx, ty):
    n = 1 if d > 8192 else 67
    x, _, w, b = make(n, d, tx, ty, d)
    got = ezsp.layer_norm(x.cuda(), w.cuda(), b.cuda(), EPS, out_dtype=ty,
                          want_stats=True)
    check_forward(x, w, b, got, 4 * d / 64 + 64)


@pytest.mark.parametrize("n", [1, 2, 63, 64, 65, 1000, 70_001])
def test_forward_rows(n):
    x, _, w, b = make(n, 24, F32, F32, n)
    check_forward(x, w, b, ezsp.layer_norm(x.cuda(), w.cuda(), b.cuda(),
                                           want_stats=True), 66)
    # without the affine part, and without the statistics
    y = ezsp.layer_norm(x.cuda())
    ry, _, rr = forward64(x, None, None, EPS)
    xd = x.double()
    big = xd.abs().mean(1)
    within(y, ry, (xd.abs() + big[:, None]) * rr[:, None] *
           (1 + big * rr)[:, None], F32, 66)


def backward64(dy, x, mean, rstd, w, dres):
    x, dy = x.double(), dy.double()
    r = rstd.double()[:, None]
    xh = (x - mean.double()[:, None]) * r
    g = dy * (1.0 if w is None else w.double())
    dx = (g - g.mean(1, keepdim=True) -
          xh * (g * xh).mean(1, keepdim=True)) * r
    mag = (g.abs() + g.abs().mean(1, keepdim=True) +
           xh.abs() * (g * xh).abs().mean(1, keepdim=True)) * r
    # xh's own rounding is that of x and mean before their difference
    amp = 1 + (x.abs() + mean.double()[:, None].abs()) * r
    mag = mag * amp
    if dres is not None:
        dx = dx + dres.double()
        mag = mag + dres.double().abs()
    return (dx, mag, (dy * xh).sum(0), (dy.abs() * (xh.abs() + amp)).sum(0),
            dy.sum(0), dy.abs().sum(0))


@pytest.mark.parametrize("tx,ty", [(BF, BF), (F32, BF), (F32, F32),
                                   (BF, F32)])
@pytest.mark.parametrize("d", WIDTHS)
def test_backward(d, tx, ty):
    n = 3 if d > 8192 else 67
    x, dy, w, _ = make(n, d, tx, ty, 100 + d)
    _, mean, rstd = forward64(x, None, None, EPS)
    mean, rstd = mean.float(), rstd.float()
    for dres in (None, torch.randn(n, d).to(tx)):
        dx, dw, db = ezsp.layer_norm_backward(
            dy.cuda(), x.cuda(), mean.cuda(), rstd.cuda(), w.cuda(),
            None if dres is None else dres.cuda())
        rdx, mag, rdw, mw, rdb, mb = backward64(dy, x, mean, rstd, w, dres)
        c = 4 * d / 64 + 64
        within(dx, rdx, mag, tx, c)
        within(dw, rdw, mw, F32, n / 16 + 64)
        within(db, rdb, mb, F32, n / 16 + 64)


@pytest.mark.parametrize("n,d", [(1, 5), (1, 1), (7, 1), (7, 3), (8, 1),
                                 (9, 7), (4099, 40), (50_001, 16),
                                 (9001, 512), (3001, 1500), (1100, 3001),
                                 (1200, 6000)])
def test_backward_rows(n, d):
    x, dy, _, _ = make(n, d, F32, F32, n)
    _, mean, rstd = forward64(x, None, None, EPS)
    mean, rstd = mean.float(), rstd.float()
    dx, dw, db = ezsp.layer_norm_backward(dy.cuda(), x.cuda(), mean.cuda(),
                                          rstd.cuda())
    rdx, mag, rdw, mw, rdb, mb = backward64(dy, x, mean, rstd, None, None)
    within(dx, rdx, mag, F32, 4 * d / 64 + 64)
    within(dw, rdw, mw, F32, n / 16 + 64)
    within(db, rdb, mb, F32, n / 16 + 64)
    only = ezsp.layer_norm_backward(dy.cuda(), x.cuda(), mean.cuda(),
                                    rstd.cuda(), want_sums=False)
    assert torch.equal(only[0], dx) and only[1] is None and only[2] is None
    sums = ezsp.layer_norm_backward(dy.cuda(), x.cuda(), mean.cuda(),
                                    rstd.cuda(), want_dx=False)
    assert sums[0] is None
    assert torch.equal(sums[1], dw) and torch.equal(sums[2], db)


def test_gradient_against_differences():
    # central differences of sum(y * dy) in 64 bits
    x, dy, w, b = make(3, 11, F32, F32, 5)
    _, mean, rstd = forward64(x, w, b, EPS)
    dx, dw, db = ezsp.layer_norm_backward(dy.cuda(), x.cuda(),
                                          mean.float().cuda(),
                                          rstd.float().cuda(), w.cuda())

    def loss(x, w, b):
        return float((forward64(x, w, b, EPS)[0] * dy.double()).sum())
    h = 1e-5
    for t, grad in ((x, dx), (w, dw), (b, db)):
        flat = t.double().flatten()
        for i in range(flat.numel()):
            args = []
            for s in (h, -h):
                moved = flat.clone()
                moved[i] += s
                moved = moved.reshape(t.shape)
                args.append([moved if q is t else q.double()
                             for q in (x, w, b)])
            num = (loss(*args[0]) - loss(*args[1])) / (2 * h)
            # differences: h^2 / 6 of the third derivative and 1e-16 / h
            assert abs(num - float(grad.flatten()[i])) < 2e-5


def test_strides_and_odd_alignment():
    # columns of a wider table, at an odd offset, and a transposed order
    g = torch.Generator().manual_seed(1)
    for ty in (BF, F32):
        wide = torch.randn(70, 61, generator=g).to(ty).cuda()
        x = wide[:, 3:52]
        same = ezsp.layer_norm(x.contiguous(), want_stats=True)
        for got, ref in zip(ezsp.layer_norm(x, want_stats=True), same):
            assert torch.equal(got, ref)
        xt = x.t().contiguous().t()
        assert torch.equal(ezsp.layer_norm(xt), same[0])
        dy = torch.randn(70, 61, generator=g).to(ty).cuda()[:, 7:56]
        a = ezsp.layer_norm_backward(dy, x, same[1], same[2], dres=x)
        b = ezsp.layer_norm_backward(dy.contiguous(), x.contiguous(), same[1],
                                     same[2], dres=x.contiguous())
        for p, q in zip(a, b):
            assert torch.equal(p, q)


def test_nothing_past_the_rows_is_written():
    # outputs inside larger buffers of a known value, through the C ABI
    lib = ezsp.load()
    n, d, ld = 19, 13, 17
    x = torch.randn(n, d, device="cuda")
    y = torch.full((n, ld), 7.0, device="cuda")
    rc = lib.ezsp_layer_norm(x.data_ptr(), d, 1, n, d, None, None, EPS,
                             y.data_ptr(), ld, 1, None, None,
                             ezsp._stream(x.device))
    assert rc == ezsp.OK
    assert torch.equal(y[:, :d], ezsp.layer_norm(x))
    assert bool((y[:, d:] == 7.0).all())


def test_infinities_and_nan_stay_in_their_row():
    x = torch.randn(9, 100, device="cuda")
    clean = ezsp.layer_norm(x)
    x[2, 5] = float("nan")
    x[4, 99] = float("inf")
    y = ezsp.layer_norm(x)
    assert bool(y[2].isnan().all()) and bool(y[4].isnan().all())
    keep = [r for r in range(9) if r not in (2, 4)]
    assert torch.equal(y[keep], clean[keep])


def test_constant_rows():
    # zero variance: rstd = eps^-1/2, y = bias
    x = torch.full((5, 64), 3.25, device="cuda")
    b = torch.randn(64, device="cuda")
    y, mean, rstd = ezsp.layer_norm(x, None, b, 1e-5, want_stats=True)
    assert torch.equal(y, b.expand(5, 64))
    assert bool((mean == 3.25).all())
    np.testing.assert_allclose(rstd.cpu().numpy(), 1e-5 ** -0.5, rtol=1e-6)


def test_same_results_every_run_and_on_a_side_stream():
    x, dy, w, _ = make(30_001, 48, F32, F32, 3)
    x, dy, w = x.cuda(), dy.cuda(), w.cuda()
    _, mean, rstd = ezsp.layer_norm(x, w, want_stats=True)
    a = ezsp.layer_norm_backward(dy, x, mean, rstd, w)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        b = ezsp.layer_norm_backward(dy, x, mean, rstd, w)
    side.synchronize()
    for p, q in zip(a, b):
        assert torch.equal(p, q)


def test_refusals():
    x = torch.randn(4, 8, device="cuda")
    v = torch.ones(8, device="cuda")
    with pytest.raises(TypeError):
        ezsp.layer_norm(x.cpu())
    with pytest.raises(TypeError):
        ezsp.layer_norm(x.half())
    with pytest.raises(TypeError):
        ezsp.layer_norm(x, v.double())
    with pytest.raises(TypeError):
        ezsp.layer_norm(x, out_dtype=torch.float16)
    with pytest.raises(ValueError):
        ezsp.layer_norm(x, torch.ones(7, device="cuda"))
    with pytest.raises(ValueError):
        ezsp.layer_norm(x[0])
    for bad in (float("nan"), -1.0, float("inf")):
        with pytest.raises(ezsp.EzspError):
            ezsp.layer_norm(x, eps=bad)
    with pytest.raises(ezsp.EzspError):
        ezsp.layer_norm(x[:0])
    _, mean, rstd = ezsp.layer_norm(x, want_stats=True)
    with pytest.raises(ValueError):
        ezsp.layer_norm_backward(x[:3], x, mean, rstd)
    with pytest.raises(TypeError):
        ezsp.layer_norm_backward(x, x, mean, rstd, dres=x.bfloat16())
    with pytest.raises(ezsp.EzspError):
        ezsp.layer_norm_backward(x, x, mean, rstd, want_dx=False,
                                 want_sums=False)
