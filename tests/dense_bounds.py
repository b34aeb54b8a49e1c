"""Bounds that the tests of the matrix-product operators share.

u = 2^-24 is half an ulp of fp32.  A sum of K products accumulated in fp32 in
any order, each step rounded or truncated, is within (2 K + 16) u of the sum
of the magnitudes.  A result is then rounded once to its type, by at most
2^-p relative (p = 8 significant bits for bfloat16, 24 for fp32)."""
import torch

U = 2.0 ** -24
BF, F32 = torch.bfloat16, torch.float32
HALF_ULP = {F32: U, BF: 2.0 ** -8}


def sum_error(k, magnitude):
    return (2 * k + 16) * U * magnitude


def check(got, ref, err, name):
    """got against ref, which it may miss by err before its one rounding."""
    assert got.shape == ref.shape, name
    half = HALF_ULP[got.dtype]
    off = (got.double() - ref).abs()
    tol = err + half * (ref.abs() + err) + 1e-37
    bad = ~(off <= tol)
    assert not bool(bad.any()), \
        (name, int(bad.sum()), float((off / tol).nan_to_num(9e9).max()))


def act64(z, act):
    if act == "relu":
        return z.clamp_min(0.0)
    if act == "gelu":
        return z * torch.special.ndtr(z)
    if act == "silu":
        return z * torch.sigmoid(z)
    return z


def act_grad64(z, act):
    if act == "relu":
        return (z > 0).double()
    if act == "gelu":
        return torch.special.ndtr(z) + z * torch.exp(-z * z / 2) * \
            0.3989422804014327
    if act == "silu":
        s = torch.sigmoid(z)
        return s * (1 + z * (1 - s))
    return torch.ones_like(z)


# An activation's value and derivative are evaluated in fp32 with a handful of
# operations of a few u each, relative to 1 + |z|; their slopes stay below 1.2.
def act_error(z, err_z):
    return 1.2 * err_z + 32 * U * (1 + z.abs())


def integers(g, shape, lim, dtype):
    """Small integers: every sum of their products is exact in fp32."""
    return torch.randint(-lim, lim + 1, shape, generator=g,
                         device="cuda").to(dtype)


def normal(g, shape, dtype, scale=1.0):
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(dtype)


def generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g
