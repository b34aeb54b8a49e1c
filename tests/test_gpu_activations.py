"""Activations and their derivatives alone, through products with the matrix
[[1]], results in fp32, against 64 bits.

u = 2^-24.  The hardware's 2^x and reciprocal are within one ulp (2 u).
  SiLU: exp(-z) carries |z| u from its argument's two roundings and 2 u of its
  own, the sum, the reciprocal and the product 4 u more: the value is within
  (8 + 2 |z|) u of itself, as far as fp32 holds exp(-z).
  GELU: exp(-z^2 / 2) carries 3 z^2 / 2 u from three roundings of its argument
  and 2 u; t, its complement and their products 7 u, which the polynomial
  (slope at most 1 relative to itself on the way) and its last steps bring to
  12: the tail is within (14 + 2 z^2) u of itself; 16 (1 + z^2) u covers it at
  every z.  Against 1 + |z| the worst place is 0, where Phi is 1/2: the value
  is within 2 (1 + |z|) u, the derivative, with a second product and a sum,
  within 4."""
import pytest
import torch

from dense_bounds import F32, U, act64, act_grad64
from paper_2512_00385_amd import ezsp

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    ezsp.load()
    yield


ONE = [[1.0]]


def value(z, act):
    return ezsp.linear(z[:, None], torch.tensor(ONE, device="cuda"),
                       act=act)[:, 0].double()


def derivative(z, act):
    ones = torch.ones_like(z)[:, None]
    return ezsp.linear_backward(
        ones, ones, torch.tensor(ONE, device="cuda"), z[:, None].contiguous(),
        act=act, want_dw=False, want_db=False)[0][:, 0].double()


def span(lo, hi, n=200_001):
    return torch.linspace(lo, hi, n, dtype=torch.float64,
                          device="cuda").float()


def test_gelu_tail_relative():
    z = span(-13.0, 0.0)
    # (Phi through erfc: 1 + erf has nothing left of it out there)
    ref = z.double() * torch.special.erfc(-z.double() * 0.5 ** 0.5) / 2
    off = (value(z, "gelu") - ref).abs()
    assert bool((off <= 16 * U * (1 + z.double() ** 2) * ref.abs()).all())


def test_gelu():
    for z in (span(-14.0, 14.0), span(-0.2, 0.2)):
        zd = z.double()
        off = (value(z, "gelu") - act64(zd, "gelu")).abs()
        assert bool((off <= 2 * U * (1 + zd.abs())).all())
        off = (derivative(z, "gelu") - act_grad64(zd, "gelu")).abs()
        assert bool((off <= 4 * U * (1 + zd.abs())).all())


def test_gelu_of_bfloat16_products_in_fp32():
    z = span(-9.0, 9.0).to(torch.bfloat16)
    y = ezsp.linear(z[:, None], torch.tensor(ONE, device="cuda").to(z.dtype),
                    act="gelu", out_dtype=F32)[:, 0].double()
    zd = z.double()
    ref = zd * torch.special.erfc(-zd * 0.5 ** 0.5) / 2
    assert bool(((y - ref).abs() <= 16 * U * (1 + zd ** 2) * ref.abs()).all())


def test_silu_tail_relative():
    z = span(-80.0, 80.0)
    ref = act64(z.double(), "silu")
    off = (value(z, "silu") - ref).abs()
    assert bool((off <= (8 + 2 * z.double().abs()) * U * ref.abs()).all())


@pytest.mark.parametrize("act", ["gelu", "silu", "relu"])
def test_far_values(act):
    big = torch.tensor([50.0, 1e4, 1e19, 3e38, float("inf")], device="cuda")
    assert torch.equal(value(big, act), big.double())
    assert bool((value(-big[1:4], act) == 0).all())
    assert torch.equal(derivative(big[:4], act),
                       torch.ones(4, device="cuda").double())
    assert bool((derivative(-big[1:4], act) == 0).all())
    nan = torch.tensor([float("nan"), 1.0], device="cuda")
    assert value(nan, act).isnan().tolist() == [True, False]
