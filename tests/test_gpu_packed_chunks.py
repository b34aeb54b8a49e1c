"""Unaligned products of 384 or 512 columns or more: the long operand is packed,
in chunks where its copy is larger than the workspace allows, and their results
and sums put together.  On integers, for equality with 64 bits."""
import pytest
import torch

from dense_bounds import BF, F32, generator, integers
from paper_2512_00385_amd import ezsp

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    ezsp.load()
    yield
    torch.cuda.empty_cache()


# one chunk; several, the last of them short
SIZES = [(20_011, 130, 515), (600_000, 130, 515), (330_007, 515, 512),
         (200_003, 201, 390), (400_003, 201, 384)]


@pytest.mark.parametrize("ty", [BF, F32])
@pytest.mark.parametrize("n,k,m", SIZES)
def test_linear(n, k, m, ty):
    g = generator(n + k + m)
    x, dy = (integers(g, (n, d), 2, ty) for d in (k, m))
    w, b = integers(g, (k, m), 2, ty), integers(g, (m,), 5, F32)
    y = ezsp.linear(x, w, b, "relu", dy)
    dx, dw, db = ezsp.linear_backward(dy, x, w)
    sums = torch.zeros((k, m), dtype=torch.float64, device="cuda")
    for i in range(0, n, 65_536):  # (the whole in 64 bits would be large)
        xs, ds = (t[i:i + 65_536].double() for t in (x, dy))
        z = (xs @ w.double() + b.double()).clamp_min(0) + ds
        assert torch.equal(y[i:i + 65_536], z.to(ty))
        assert torch.equal(dx[i:i + 65_536], (ds @ w.double().t()).to(ty))
        sums += xs.t() @ ds
    assert torch.equal(dw, sums.to(ty))
    assert torch.equal(db.double(), dy.double().sum(0))


@pytest.mark.parametrize("ty", [BF, F32])
@pytest.mark.parametrize("n,k,m", [(20_011, 130, 260), (500_000, 131, 260),
                                   (330_007, 515, 256), (200_003, 201, 195)])
def test_gated(n, k, m, ty):
    g = generator(n + k + m)
    x, dh, gate, up = (integers(g, (n, d), 2, ty) for d in (k, m, m, m))
    w = [integers(g, (k, m), 2, ty) for _ in range(2)]
    h, sg, su = ezsp.gated_ff(x, *w, act="relu", want_saved=True)
    got = ezsp.gated_ff_backward(dh, x, *w, gate, up, act="relu")
    sums = [torch.zeros((k, m), dtype=torch.float64, device="cuda")
            for _ in range(2)]
    bias = [torch.zeros(m, dtype=torch.float64, device="cuda")
            for _ in range(2)]
    for i in range(0, n, 65_536):
        at = slice(i, i + 65_536)
        xs, ds, gs, us = (t[at].double() for t in (x, dh, gate, up))
        s = [xs @ wi.double() for wi in w]
        assert torch.equal(sg[at], s[0].to(ty))
        assert torch.equal(su[at], s[1].to(ty))
        assert torch.equal(h[at], (s[0].clamp_min(0) * s[1]).to(ty))
        dz = [ds * us * (gs > 0), ds * gs.clamp_min(0)]
        dx = dz[0] @ w[0].double().t() + dz[1] @ w[1].double().t()
        assert torch.equal(got[0][at], dx.to(ty))
        for p in range(2):
            sums[p] += xs.t() @ dz[p]
            bias[p] += dz[p].sum(0)
    for p in range(2):
        assert torch.equal(got[1 + p], sums[p].to(ty))
        assert torch.equal(got[3 + p].double(), bias[p])
