"""ezsp_gated_ff and its backward pass against the formulas in 64 bits
(bounds in dense_bounds), bit for bit where small integers make every sum
exact."""
import pytest
import torch

from dense_bounds import (BF, F32, U, act64, act_error, act_grad64, check,
                          generator, integers, normal, sum_error)
from paper_2512_00385_amd import ezsp

pytestmark = pytest.mark.gpu

ACTS = ["relu", "gelu", "silu", "none"]
SIZES = [
    (1, 1, 1), (1, 8, 8), (1, 4096, 512), (2, 7, 3), (3, 300, 1000),
    (8, 1024, 96), (16, 520, 128), (17, 64, 40), (31, 65, 33), (32, 128, 64),
    (33, 40, 31), (64, 256, 256), (65, 1000, 72), (128, 64, 128),
    (129, 72, 136), (130, 4, 6), (257, 6, 32), (300, 515, 77), (500, 32, 65),
    (511, 136, 264), (1000, 33, 1), (1003, 32, 128), (2000, 24, 48),
    (4100, 64, 130),
    # few columns: each split of the one-pass backward
    (7, 12, 20), (8, 5, 3), (65, 31, 33), (700, 32, 40), (700, 20, 250),
    (700, 60, 30), (700, 64, 64), (700, 57, 200), (700, 100, 30),
    (700, 128, 64), (700, 97, 100), (20_000, 3, 7),
    # few rows: columns and sums that fill no step, wide tables of weights
    (1, 33, 9), (5, 70, 37), (48, 129, 333), (64, 8192, 16), (2, 4097, 70),
    (1, 40, 16_400), (17, 40, 33_000), (40, 24, 40_001),
]
EXACT = SIZES + [(4096, 64, 1600), (3333, 200, 2056), (70, 20_000, 40),
                 (20, 30_001, 9), (50_021, 16, 24),
                 # large and unaligned: packed, whole and in chunks
                 (5001, 1021, 515), (190_001, 259, 264), (30_003, 67, 1030)]


@pytest.fixture(scope="module", autouse=True)
def gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    ezsp.load()
    yield


def tensors(n, k, m, ty, seed, exact=False):
    g = generator(seed)
    if exact:
        return (integers(g, (n, k), 2, ty),
                [integers(g, (k, m), 2, ty) for _ in range(2)],
                [integers(g, (m,), 5, F32) for _ in range(2)],
                integers(g, (n, m), 2, ty))
    return (normal(g, (n, k), ty),
            [normal(g, (k, m), ty, k ** -0.5) for _ in range(2)],
            [normal(g, (m,), F32) for _ in range(2)], normal(g, (n, m), ty))


def check_forward(x, w, b, act, h, saved):
    xd = x.double()
    sums, errs = [], []
    for wi, bi in zip(w, b):
        r = xd @ wi.double()
        mag = xd.abs() @ wi.double().abs()
        if bi is not None:
            r = r + bi.double()
            mag = mag + bi.double().abs()
        sums.append(r)
        errs.append(sum_error(x.shape[1], mag))
    if saved:
        check(saved[0], sums[0], errs[0], "gate")
        check(saved[1], sums[1], errs[1], "up")
    a, ea = act64(sums[0], act), act_error(sums[0], errs[0])
    ref = a * sums[1]
    err = ea * (sums[1].abs() + errs[1]) + a.abs() * errs[1] + \
        2 * U * ref.abs()
    check(h, ref, err, "h")


@pytest.mark.parametrize("ty", [BF, F32])
@pytest.mark.parametrize("n,k,m", SIZES)
def test_forward(n, k, m, ty):
    x, w, b, _ = tensors(n, k, m, ty, n + k + m)
    act = ACTS[(n + k + m) % 4]
    h, g, u = ezsp.gated_ff(x, *w, *b, act=act, want_saved=True)
    check_forward(x, w, b, act, h, (g, u))
    assert torch.equal(ezsp.gated_ff(x, *w, *b, act=act), h)
    check_forward(x, w, (None, None), act, ezsp.gated_ff(x, *w, act=act),
                  None)


@pytest.mark.parametrize("ty", [BF, F32])
@pytest.mark.parametrize("n,k,m", EXACT)
def test_forward_exact(n, k, m, ty):
    # without an activation the sums are exact, their product is rounded once
    # (as long as it fits fp32's 24 bits)
    x, w, b, _ = tensors(n, k, m, ty, 7, exact=True)
    h, g, u = ezsp.gated_ff(x, *w, *b, act="relu", want_saved=True)
    rg, ru = (x.double() @ wi.double() + bi.double() for wi, bi in zip(w, b))
    assert torch.equal(g, rg.to(ty)) and torch.equal(u, ru.to(ty))
    ref = rg.clamp_min(0) * ru
    fits = ref.abs() < 2 ** 24
    assert torch.equal(h[fits], ref.to(ty)[fits])


def check_backward(dh, x, w, g, u, act, got):
    n, k = x.shape
    m = w[0].shape[1]
    xd, gd, ud, d = x.double(), g.double(), u.double(), dh.double()
    wd = [t.double() for t in w]
    ea = act_error(gd, 0.0)
    dz = [d * ud * act_grad64(gd, act), d * act64(gd, act)]
    err = [(d * ud).abs() * ea + 4 * U * dz[0].abs(),
           d.abs() * ea + 2 * U * dz[1].abs()]
    dx, dwg, dwu, dbg, dbu = got
    for p, db in ((0, dbg), (1, dbu)):
        check(db, dz[p].sum(0), err[p].sum(0) +
              sum_error(n, dz[p].abs().sum(0)), f"db{p}")
    if x.dtype == BF:  # the products take dg and du as bfloat16
        err = [e + 2.0 ** -8 * (z.abs() + e) for e, z in zip(err, dz)]
    top = [z.abs() + e for z, e in zip(dz, err)]
    check(dx, dz[0] @ wd[0].t() + dz[1] @ wd[1].t(),
          err[0] @ wd[0].abs().t() + err[1] @ wd[1].abs().t() +
          sum_error(2 * m, top[0] @ wd[0].abs().t() +
                    top[1] @ wd[1].abs().t()), "dx")
    for p, dw in ((0, dwg), (1, dwu)):
        check(dw, xd.t() @ dz[p], xd.abs().t() @ err[p] +
              sum_error(n, xd.abs().t() @ top[p]), f"dw{p}")


@pytest.mark.parametrize("ty", [BF, F32])
@pytest.mark.parametrize("n,k,m", SIZES)
def test_backward(n, k, m, ty):
    x, w, b, dh = tensors(n, k, m, ty, n * 3 + k + m)
    act = ACTS[(n + k) % 4]
    g, u = ((x.float() @ wi.float() + bi).to(ty) for wi, bi in zip(w, b))
    got = ezsp.gated_ff_backward(dh, x, *w, g, u, act=act)
    assert [t.dtype for t in got] == [ty, ty, ty, F32, F32]
    check_backward(dh, x, w, g, u, act, got)


@pytest.mark.parametrize("ty", [BF, F32])
@pytest.mark.parametrize("n,k,m", EXACT)
def test_backward_exact(n, k, m, ty):
    x, w, b, dh = tensors(n, k, m, ty, 11, exact=True)
    gen = generator(5)
    g, u = integers(gen, (n, m), 2, ty), integers(gen, (n, m), 2, ty)
    dx, dwg, dwu, dbg, dbu = ezsp.gated_ff_backward(dh, x, *w, g, u,
                                                    act="relu")
    d, gd, ud = dh.double(), g.double(), u.double()
    dg, du = d * ud * (gd > 0), d * gd.clamp_min(0)
    xt = x.double().t()
    assert torch.equal(dx, (dg @ w[0].double().t() +
                            du @ w[1].double().t()).to(ty))
    assert torch.equal(dwg, (xt @ dg).to(ty))
    assert torch.equal(dwu, (xt @ du).to(ty))
    assert torch.equal(dbg, dg.sum(0).float())
    assert torch.equal(dbu, du.sum(0).float())


def test_gradients_asked_for_alone():
    x, w, b, dh = tensors(333, 48, 56, BF, 2)
    _, g, u = ezsp.gated_ff(x, *w, *b, want_saved=True)
    full = ezsp.gated_ff_backward(dh, x, *w, g, u)
    for want, kept in (("want_dx", (0,)), ("want_dw", (1, 2)),
                       ("want_db", (3, 4))):
        opts = dict(want_dx=False, want_dw=False, want_db=False)
        opts[want] = True
        got = ezsp.gated_ff_backward(dh, x, *w, g, u, **opts)
        for i in range(5):
            if i in kept:
                assert torch.equal(got[i], full[i])
            else:
                assert got[i] is None


@pytest.mark.parametrize("act", ["gelu", "silu"])
def test_gradient_against_differences(act):
    x, w, b, dh = tensors(3, 5, 4, F32, 9)
    _, g, u = ezsp.gated_ff(x, *w, *b, act=act, want_saved=True)
    grads = ezsp.gated_ff_backward(dh, x, *w, g, u, act=act)

    def loss(x, wg, wu, bg, bu):
        return float((act64(x @ wg + bg, act) * (x @ wu + bu) *
                      dh.double()).sum())
    h = 1e-5
    base = [t.double() for t in (x, *w, *b)]
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
            assert abs(num - float(grad.flatten()[i])) < 5e-5


@pytest.mark.parametrize("ty", [BF, F32])
def test_strides_and_odd_alignment(ty):
    g = generator(4)
    x = normal(g, (150, 131), ty)[:, 5:69]
    w = [normal(g, (64, 48), ty, 0.125) for _ in range(2)]
    b = [normal(g, (48,), F32) for _ in range(2)]
    ref = ezsp.gated_ff(x.contiguous(), *w, *b, want_saved=True)
    for p, q in zip(ezsp.gated_ff(x, *w, *b, want_saved=True), ref):
        assert torch.equal(p, q)
    xt, wt = x.t().contiguous().t(), [t.t().contiguous().t() for t in w]
    for p, q in zip(ezsp.gated_ff(xt, *wt, *b, want_saved=True), ref):
        assert torch.equal(p, q)
    dh = normal(g, (150, 60), ty)[:, 3:51]
    both = torch.cat([ref[1], ref[2]], 1)   # gate and up side by side
    a = ezsp.gated_ff_backward(dh.contiguous(), x.contiguous(), *w, ref[1],
                               ref[2])
    c = ezsp.gated_ff_backward(dh, x, *w, both[:, :48], both[:, 48:])
    for p, q in zip(a, c):
        assert torch.equal(p, q)


@pytest.mark.parametrize("n,k,m", [(40, 40, 40), (300, 72, 136),
                                   (13, 40, 48), (40, 33, 47)])
def test_infinities_and_nan_stay_where_they_belong(n, k, m):
    x, w, b, dh = tensors(n, k, m, BF, 6)
    h, g, u = ezsp.gated_ff(x, *w, *b, want_saved=True)
    x2, wu = x.clone(), w[1].clone()
    x2[n - 1, k - 1] = float("nan")
    wu[k - 1, m - 1] = float("inf")
    h2, g2, u2 = ezsp.gated_ff(x2, w[0], wu, *b, want_saved=True)
    assert bool(h2[n - 1].isnan().all())
    assert torch.equal(h2[:n - 1, :m - 1], h[:n - 1, :m - 1])
    assert torch.equal(g2[:n - 1], g[:n - 1])
    assert not bool(u2[:n - 1, m - 1].isfinite().any())
    full = ezsp.gated_ff_backward(dh, x, *w, g, u)
    dh2 = dh.clone()
    dh2[n - 1, m - 1] = float("nan")
    got = ezsp.gated_ff_backward(dh2, x, *w, g, u)
    assert bool(got[0][n - 1].isnan().all())
    assert torch.equal(got[0][:n - 1], full[0][:n - 1])
    for p in (1, 2):
        assert bool(got[p][:, m - 1].isnan().all())
        assert torch.equal(got[p][:, :m - 1], full[p][:, :m - 1])
    for p in (3, 4):
        assert bool(got[p][m - 1].isnan())
        assert torch.equal(got[p][:m - 1], full[p][:m - 1])


def test_same_results_every_run_and_on_a_side_stream():
    x, w, b, dh = tensors(40_001, 32, 96, BF, 3)
    _, g, u = ezsp.gated_ff(x, *w, *b, want_saved=True)
    a = ezsp.gated_ff_backward(dh, x, *w, g, u)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        c = ezsp.gated_ff_backward(dh, x, *w, g, u)
    side.synchronize()
    for p, q in zip(a, c):
        assert torch.equal(p, q)


def test_refusals():
    x, w, b, dh = tensors(4, 8, 8, BF, 1)
    with pytest.raises(TypeError):
        ezsp.gated_ff(x.float(), *w)
    with pytest.raises(TypeError):
        ezsp.gated_ff(x, w[0], w[1].float())
    with pytest.raises(TypeError):
        ezsp.gated_ff(x, *w, b[0].double())
    with pytest.raises(ValueError):
        ezsp.gated_ff(x, w[0], w[1][:, :7])
    with pytest.raises(ValueError):
        ezsp.gated_ff(x, *w, b[0][:7])
    with pytest.raises(ValueError):
        ezsp.gated_ff(x, *w, act="sigmoid")
    with pytest.raises(ezsp.EzspError):
        ezsp.gated_ff(x[:0], *w)
    _, g, u = ezsp.gated_ff(x, *w, *b, want_saved=True)
    with pytest.raises(ValueError):
        ezsp.gated_ff_backward(dh[:3], x, *w, g, u)
    with pytest.raises(TypeError):
        ezsp.gated_ff_backward(dh, x, *w, g.float(), u)
    with pytest.raises(ezsp.EzspError):
        ezsp.gated_ff_backward(dh, x, *w, g, u, want_dx=False, want_dw=False,
                               want_db=False)
