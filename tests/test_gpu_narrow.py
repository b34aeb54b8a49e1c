"""Products over many rows with few columns, both directions, in the
widths where its tiles change, on integers: sums of products of small integers
are exact in fp32 in any order, so results are compared for equality with
64-bit ones (dW and dx in bfloat16 after one rounding).  The tables lie in
wider ones whose other columns, and the rows around them, are NaN: nothing of
them may be taken."""
import pytest
import torch

from paper_2512_00385_amd import ezsp

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32
WIDTHS = [(1, 1), (2, 3), (3, 16), (16, 4), (17, 15), (5, 33), (33, 5),
          (32, 31), (31, 64), (64, 65), (63, 17), (65, 16), (128, 3), (96, 63),
          (13, 127), (128, 32), (64, 128)]
ROWS = [8, 9, 16, 63, 64, 65, 129, 2500]


def inset(t, pad):
    """t as a view into a table of NaN, pad columns apart and a row down."""
    n, d = t.shape
    big = torch.full((n + 2, d + pad), float("nan"), dtype=t.dtype,
                     device=t.device)
    big[1:n + 1, :d] = t
    return big[1:n + 1, :d]


def ints(g, shape, lim, ty):
    return torch.randint(-lim, lim + 1, shape, generator=g).to(ty).cuda()


@pytest.mark.parametrize("ty", [F32, BF])
@pytest.mark.parametrize("k,m", WIDTHS)
def test_linear(k, m, ty):
    for i, n in enumerate(ROWS):
        g = torch.Generator().manual_seed(n + k + m)
        pad = (0, 1, 8)[i % 3]
        x, dy, z = (inset(ints(g, (n, d), 2, ty), pad) for d in (k, m, m))
        w = ints(g, (k, m), 2, ty)
        dx, dw, db = ezsp.linear_backward(dy, x, w, z, act="relu")
        dz = dy.double() * (z > 0)
        assert torch.equal(dx, (dz @ w.double().t()).to(ty)), (n, pad)
        assert torch.equal(dw, (x.double().t() @ dz).to(ty)), (n, pad)
        assert torch.equal(db.double(), dz.sum(0)), (n, pad)


@pytest.mark.parametrize("ty", [F32, BF])
@pytest.mark.parametrize("k,m", WIDTHS)
def test_gated(k, m, ty):
    for i, n in enumerate(ROWS):
        g = torch.Generator().manual_seed(n + k + m)
        pad = (0, 1, 8)[i % 3]
        x, dh = (inset(ints(g, (n, d), 2, ty), pad) for d in (k, m))
        gate, up = (inset(ints(g, (n, m), 2, ty), pad) for _ in range(2))
        w = [ints(g, (k, m), 2, ty) for _ in range(2)]
        got = ezsp.gated_ff_backward(dh, x, *w, gate, up, act="relu")
        dg = dh.double() * up.double() * (gate > 0)
        du = dh.double() * gate.double().clamp_min(0)
        ref = [dg @ w[0].double().t() + du @ w[1].double().t(),
               x.double().t() @ dg, x.double().t() @ du, dg.sum(0), du.sum(0)]
        for name, a, b in zip(("dx", "dwg", "dwu", "dbg", "dbu"), got, ref):
            assert torch.equal(a, b.to(a.dtype)), (name, n, pad)


@pytest.mark.parametrize("ty", [F32, BF])
@pytest.mark.parametrize("k,m", [(6, 4), (33, 16), (64, 64)])
def test_one_row_of_infinities_stays_its_own(k, m, ty):
    n, bad = 300, 137
    g = torch.Generator().manual_seed(1)
    x, dy = ints(g, (n, k), 2, ty), ints(g, (n, m), 2, ty)
    w = ints(g, (k, m), 2, ty)
    dy[bad, m - 1] = float("inf")
    dx, dw, db = ezsp.linear_backward(dy, x, w)
    ref = (dy.double() @ w.double().t()).to(ty)
    keep = torch.arange(n) != bad
    assert torch.equal(dx[keep], ref[keep])
    assert not torch.isfinite(dx[bad]).all()
    ref = (x.double().t() @ dy.double()).to(ty)
    assert torch.equal(dw[:, :m - 1], ref[:, :m - 1])
    assert torch.isfinite(db[:m - 1]).all() and torch.isinf(db[m - 1])


@pytest.mark.parametrize("ty", [F32, BF])
def test_results_alone_match_all(ty):
    g = torch.Generator().manual_seed(3)
    x, dy = ints(g, (400, 20), 2, ty), ints(g, (400, 12), 2, ty)
    w = ints(g, (20, 12), 2, ty)
    full = ezsp.linear_backward(dy, x, w)
    for i in range(3):
        want = [i == 0, i == 1, i == 2]
        got = ezsp.linear_backward(dy, x, w, None, "none", *want)
        for j in range(3):
            assert (got[j] is None) == (not want[j])
        assert torch.equal(got[i], full[i])


@pytest.mark.parametrize("ty", [F32, BF])
@pytest.mark.parametrize("k,m", [(1, 1), (3, 7), (6, 4), (7, 33), (8, 16),
                                 (15, 17), (16, 32), (16, 33), (17, 8),
                                 (31, 64), (32, 63), (33, 65)])
def test_forward(k, m, ty):
    for i, n in enumerate((8, 1023, 1024, 1055, 1153, 9000)):
        g = torch.Generator().manual_seed(n + k + m)
        pad = (0, 1, 8)[i % 3]
        x, res = (inset(ints(g, (n, d), 2, ty), pad) for d in (k, m))
        w = [ints(g, (k, m), 2, ty) for _ in range(2)]
        b = [ints(g, (m,), 5, F32) for _ in range(2)]
        s = [x.double() @ wi.double() + bi.double() for wi, bi in zip(w, b)]
        y, z = ezsp.linear(x, w[0], b[0], "relu", res, want_z=True)
        assert torch.equal(z, s[0].to(ty)), (n, pad)
        assert torch.equal(y, (s[0].clamp_min(0) + res.double()).to(ty))
        h, gate, up = ezsp.gated_ff(x, *w, *b, act="relu", want_saved=True)
        assert torch.equal(gate, s[0].to(ty)) and torch.equal(up, s[1].to(ty))
        assert torch.equal(h, (s[0].clamp_min(0) * s[1]).to(ty)), (n, pad)
        assert torch.equal(ezsp.gated_ff(x, *w, *b, act="relu"), h)


@pytest.mark.parametrize("ty", [F32, BF])
def test_forward_keeps_rows_apart(ty):
    g = torch.Generator().manual_seed(2)
    x, w = ints(g, (3000, 6), 2, ty), ints(g, (6, 12), 2, ty)
    ref = ezsp.linear(x, w)
    x[1500] = float("nan")
    y = ezsp.linear(x, w)
    keep = torch.arange(3000) != 1500
    assert torch.equal(y[keep], ref[keep]) and torch.isnan(y[1500]).all()
