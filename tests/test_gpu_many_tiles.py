"""Products whose operands are not aligned to 16 bytes, too small to be packed
and too large to give every tile a block of its own, so that a block goes from
tile to tile: sums of k that end inside a step, lines that end inside a
vector, columns of wider tables whose other columns are NaN.  On integers:
sums of products of small integers are exact in fp32 in any order, so results
are compared for equality with 64-bit ones after one rounding."""
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


def inset(t, pad):
    """t as columns of a table of NaN: an odd offset, pad columns more."""
    if pad == 0:
        return t
    n, d = t.shape
    big = torch.full((n + 2, d + pad), float("nan"), dtype=t.dtype,
                     device=t.device)
    big[1:n + 1, 1:d + 1] = t
    return big[1:n + 1, 1:d + 1]


@pytest.mark.parametrize("n,k,m,ty,pad", [
    (100_000, 100, 100, BF, 0), (100_000, 100, 100, BF, 3),
    (100_000, 33, 65, BF, 0), (200_000, 100, 64, BF, 0),
    (200_000, 128, 64, BF, 7), (150_001, 96, 96, BF, 3),
    (10_000, 9, 1024, BF, 0), (282_169, 6, 384, BF, 0),
    (300_000, 200, 20, BF, 5), (100_000, 130, 100, F32, 0),
    (100_000, 96, 96, F32, 3), (23_053, 64, 1023, F32, 0),
    (200_000, 70, 20, F32, 1)])
def test_linear(n, k, m, ty, pad):
    g = generator(n + k + m)
    x, res = (inset(integers(g, (n, d), 2, ty), pad) for d in (k, m))
    w, b = integers(g, (k, m), 2, ty), integers(g, (m,), 5, F32)
    z = x.double() @ w.double() + b.double()
    y, got = ezsp.linear(x, w, b, "relu", res, want_z=True)
    assert torch.equal(got, z.to(ty))
    assert torch.equal(y, (z.clamp_min(0) + res.double()).to(ty))


@pytest.mark.parametrize("n,k,m,ty,pad", [
    (100_000, 32, 100, BF, 0), (100_000, 33, 65, BF, 0),
    (150_001, 96, 48, BF, 3), (150_001, 200, 20, BF, 0),
    (20_000, 9, 515, BF, 0), (540, 24, 8191, F32, 0),
    (100_000, 40, 50, F32, 3)])
def test_gated(n, k, m, ty, pad):
    g = generator(n + k + m)
    x = inset(integers(g, (n, k), 2, ty), pad)
    w = [integers(g, (k, m), 2, ty) for _ in range(2)]
    b = [integers(g, (m,), 5, F32) for _ in range(2)]
    s = [x.double() @ wi.double() + bi.double() for wi, bi in zip(w, b)]
    h, gate, up = ezsp.gated_ff(x, *w, *b, act="relu", want_saved=True)
    assert torch.equal(gate, s[0].to(ty)) and torch.equal(up, s[1].to(ty))
    assert torch.equal(h, (s[0].clamp_min(0) * s[1]).to(ty))
    assert torch.equal(ezsp.gated_ff(x, *w, *b, act="relu"), h)


@pytest.mark.parametrize("n,k,m,ty,pad", [
    (100_000, 130, 100, BF, 0), (100_000, 130, 101, F32, 0),
    (200_000, 130, 33, BF, 3), (100_000, 140, 40, F32, 1)])
def test_linear_backward(n, k, m, ty, pad):
    g = generator(n + k + m)
    x, dy, z = (inset(integers(g, (n, d), 2, ty), pad) for d in (k, m, m))
    w = integers(g, (k, m), 2, ty)
    dz = dy.double() * (z > 0)
    got = ezsp.linear_backward(dy, x, w, z, act="relu")
    for p, ref in zip(got, (dz @ w.double().t(), x.double().t() @ dz,
                            dz.sum(0))):
        assert torch.equal(p, ref.to(p.dtype))
    dz = dy.double()
    got = ezsp.linear_backward(dy, x, w)
    for p, ref in zip(got, (dz @ w.double().t(), x.double().t() @ dz,
                            dz.sum(0))):
        assert torch.equal(p, ref.to(p.dtype))


@pytest.mark.parametrize("n,k,m,ty,pad", [
    (70_000, 130, 42, BF, 0), (70_000, 130, 42, F32, 0),
    (100_000, 131, 30, BF, 3)])
def test_gated_backward(n, k, m, ty, pad):
    g = generator(n + k + m)
    x, dh = (inset(integers(g, (n, d), 2, ty), pad) for d in (k, m))
    gate, up = (inset(integers(g, (n, m), 2, ty), pad) for _ in range(2))
    w = [integers(g, (k, m), 2, ty) for _ in range(2)]
    dg = dh.double() * up.double() * (gate > 0)
    du = dh.double() * gate.double().clamp_min(0)
    ref = (dg @ w[0].double().t() + du @ w[1].double().t(),
           x.double().t() @ dg, x.double().t() @ du, dg.sum(0), du.sum(0))
    got = ezsp.gated_ff_backward(dh, x, *w, gate, up, act="relu")
    for name, p, r in zip(("dx", "dwg", "dwu", "dbg", "dbu"), got, ref):
        assert torch.equal(p, r.to(p.dtype)), name


def test_embedding_network_of_a_hundred_hidden_channels():
    # one block's gated product as the example network calls it, against the
    # same rows in pieces that give every tile its own block
    g = generator(1)
    n, k, m = 100_000, 32, 100
    x = torch.randn((n, k), generator=g, device="cuda").to(BF)
    w = [torch.randn((k, m), generator=g, device="cuda").mul(0.2).to(BF)
         for _ in range(2)]
    whole = ezsp.gated_ff(x, *w, want_saved=True)
    parts = [ezsp.gated_ff(x[i:i + 20_000], *w, want_saved=True)
             for i in range(0, n, 20_000)]
    for p, q in zip(whole, zip(*parts)):
        assert torch.equal(p, torch.cat(q))
