"""Cross attention in whole numbers: no key and no row is lost or met twice.

q has values in the even places of d alone, k in the odd ones, so S = 0.  All
values are -1, 0 or 1.  Forward P = 1 before it is divided by the number n of
keys, so the sums are whole numbers below 2^24, exact in fp32 in any order and
parts, and
  out = sum v / n: 1 / n and the product are rounded, 2 2^-24 of it, then the
        result to its type;
  lse = log n: the base 2 logarithm (one ulp, 2 2^-24 of it), ln 2 and the
        product, 4 2^-24 of it; a key too few moves it by 1 / n, 40 times as
        far and more at these lengths.
Backward lse = 0 is handed in, so P = 1, and any out, so that D is a whole
number too: dS = dout . v - D is one of at most 2 d_head = 256, which bfloat16
holds, and with a scale of 1/4 every gradient is exact up to the one rounding
to its type."""
import math

import pytest
import torch

from paper_2512_00385_amd import ezsp

BF, F32 = torch.bfloat16, torch.float32
U = 2.0 ** -24
HALF_ULP = {F32: U, BF: 2.0 ** -8}
INF = math.inf
SCALE = 0.25


def make(nq, nk, heads, kv, dh, ty, seed, masked=False, device="cuda"):
    g = torch.Generator().manual_seed(seed)

    def ints(n, h):
        return torch.randint(-1, 2, (n, h, dh), generator=g).double()
    t = dict(q=ints(nq, heads), k=ints(nk, kv), v=ints(nk, kv),
             dout=ints(nq, heads), out=ints(nq, heads))
    t["q"][:, :, 1::2] = 0
    t["k"][:, :, 0::2] = 0
    t = {k: x.reshape(x.shape[0], -1).to(device, ty) for k, x in t.items()}
    t["bias"] = torch.zeros(nk)
    if masked:
        t["bias"][torch.rand(nk, generator=g) < 0.2] = -INF
    t["bias"] = t["bias"].to(device)
    return t


def oracle(t, heads, kv, dh, drop_key=None, drop_row=None):
    """Of one cloud, in 64 bits: out's sums, the number of keys, dq, dk, dv.
    A dropped key or row is what a kernel that loses it would do."""
    def split(x, n):
        return x.double().reshape(x.shape[0], n, dh).permute(1, 0, 2)
    group = heads // kv
    live = t["bias"] > -INF
    seen = live.clone()
    if drop_key is not None:
        seen[drop_key] = False
    rows = torch.ones(t["q"].shape[0], dtype=torch.float64,
                      device=t["q"].device)
    if drop_row is not None:
        rows[drop_row] = 0
    q, do, o = (split(t[x], heads) for x in ("q", "dout", "out"))
    k, v = (split(t[x], kv).repeat_interleave(group, 0) for x in ("k", "v"))
    ks, vs = (x * seen[:, None] for x in (k, v))
    d = (do * o).sum(2, keepdim=True)
    dq = SCALE * (do @ (vs.transpose(1, 2) @ ks) -
                  d * ks.sum(1, keepdim=True))
    if not bool(live.any()):
        dq = torch.zeros_like(dq)
    r = rows[None, :, None]

    def shared(x):
        return (x.reshape(kv, group, *x.shape[1:]).sum(1) *
                live[:, None]).permute(1, 0, 2).flatten(1)
    dk = SCALE * shared(v @ ((do * r).transpose(1, 2) @ q) -
                        (d * r * q).sum(1, keepdim=True))
    dv = shared((do * r).sum(1, keepdim=True).expand(-1, k.shape[1], -1))
    total = vs.sum(1, keepdim=True).expand(-1, q.shape[1], -1)

    def flat(x):
        return x.permute(1, 0, 2).flatten(1)
    return flat(total), int(seen.sum()), flat(dq), dk, dv


def pieces(t, q_off, k_off):
    """The call's clouds, those without the other side among them."""
    if q_off is None:
        yield slice(0, t["q"].shape[0]), slice(0, t["k"].shape[0])
        return
    for a, b, c, d in zip(q_off, q_off[1:], k_off, k_off[1:]):
        yield slice(a, b), slice(c, d)


def check(t, heads, kv, dh, q_off=None, k_off=None):
    ty = t["q"].dtype
    kw = dict(key_bias=t["bias"], scale=SCALE)
    if q_off is not None:
        kw["q_offsets"], kw["k_offsets"] = (
            torch.tensor(o, dtype=torch.int32, device="cuda")
            for o in (q_off, k_off))
    out, lse = ezsp.cross_attention(t["q"], t["k"], t["v"], heads, kv,
                                    want_lse=True, **kw)
    # P = 1 wherever a row has keys
    one = torch.where(lse == -INF, -INF, 0.0)
    dq, dk, dv = ezsp.cross_attention_backward(
        t["dout"], t["q"], t["k"], t["v"], t["out"], one, heads, kv, **kw)
    for rows, keys in pieces(t, q_off, k_off):
        part = {x: t[x][rows] for x in ("q", "dout", "out")}
        part.update({x: t[x][keys] for x in ("k", "v", "bias")})
        nq, nk = part["q"].shape[0], part["k"].shape[0]
        assert 2 * dh * max(nq * heads // kv, nk) < 1 << 24
        total, n, rdq, rdk, rdv = oracle(part, heads, kv, dh)
        if n:
            ref = total / n
            off = (out[rows].double() - ref).abs()
            assert bool((off <= (2 * U + HALF_ULP[ty]) * 1.01 * ref.abs())
                        .all()), "out"
            assert bool(((lse[:, rows].double() - math.log(n)).abs()
                         <= 5 * U * math.log(n)).all()), "lse"
        else:
            assert bool((out[rows] == 0).all())
            assert bool((lse[:, rows] == -INF).all())
        assert torch.equal(dq[rows], rdq.to(ty)), "dq"
        assert torch.equal(dk[keys], rdk.to(ty)), "dk"
        assert torch.equal(dv[keys], rdv.to(ty)), "dv"


@pytest.mark.parametrize("ty", [BF, F32])
@pytest.mark.parametrize("dh", [16, 64])
@pytest.mark.parametrize("nq,nk", [(60, 23_001), (20_000, 40)])
def test_a_lost_line_would_show(nq, nk, dh, ty):
    """The oracle that loses one key or one row differs beyond what check
    allows, at lengths where a bound on roundings hides it.  (Forward a key
    shows in lse; a lost key is one whose k and v hold something, as all but
    3^-dh do.)"""
    t = make(nq, nk, 1, 1, dh, ty, nq, device="cpu")
    whole = oracle(t, 1, 1, dh)
    for lost in (0, nk // 2, nk - 1):
        short = oracle(t, 1, 1, dh, drop_key=lost)
        assert abs(math.log(short[1]) - math.log(nk)) > 10 * U * math.log(nk)
        assert not torch.equal(whole[2].to(ty), short[2].to(ty))
    for lost in (0, nq // 2, nq - 1):
        short = oracle(t, 1, 1, dh, drop_row=lost)
        for i in (3, 4):
            assert not torch.equal(whole[i].to(ty), short[i].to(ty))


@pytest.fixture
def gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    ezsp.load()


WIDTHS = [16, 31, 48, 64, 80, 93, 128]


@pytest.mark.gpu
@pytest.mark.parametrize("ty", [BF, F32])
@pytest.mark.parametrize("dh", WIDTHS)
@pytest.mark.parametrize("masked", [False, True])
def test_edges_of_tiles(gpu, masked, dh, ty):
    for n in (1, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 191, 192,
              193, 255, 256, 257, 511, 513):
        check(make(n, 100, 2, 2, dh, ty, n, masked), 2, 2, dh)
        check(make(70, n, 4, 2, dh, ty, n + 1, masked), 4, 2, dh)


@pytest.mark.gpu
@pytest.mark.parametrize("ty", [BF, F32])
@pytest.mark.parametrize("dh", WIDTHS)
@pytest.mark.parametrize("nq,nk,heads,kv", [
    (1, 9001, 8, 2), (3, 23_001, 2, 2), (759, 23_001, 8, 8),
    (200, 4097, 6, 3), (20_000, 40, 2, 2), (13_400, 613, 8, 8),
    (20_000, 613, 4, 1), (60_001, 3, 2, 2)])
def test_lines_in_parts(gpu, nq, nk, heads, kv, dh, ty):
    if 2 * dh * nq * heads // kv >= 1 << 24:
        nq = (1 << 24) // (2 * dh * heads // kv) - 1
    check(make(nq, nk, heads, kv, dh, ty, nq + nk, True), heads, kv, dh)


@pytest.mark.gpu
@pytest.mark.parametrize("ty", [BF, F32])
@pytest.mark.parametrize("dh", WIDTHS)
def test_many_columns(gpu, dh, ty):
    # blocks of whole waves on both sides, without parts of lines
    check(make(4111, 300, 16, 16, dh, ty, dh), 16, 16, dh)
    check(make(300, 4111, 16, 16, dh, ty, dh), 16, 16, dh)


@pytest.mark.gpu
@pytest.mark.parametrize("ty", [BF, F32])
@pytest.mark.parametrize("dh", [16, 48, 64, 128])
@pytest.mark.parametrize("heads,kv", [(2, 2), (6, 2), (16, 8)])
def test_uneven_clouds(gpu, heads, kv, dh, ty):
    # without rows, without keys, without both, single ones, long ones
    rows = [3, 3, 40, 41, 41, 300, 428, 429, 5000, 5001, 9100]
    keys = [2, 70, 70, 71, 71, 200, 264, 2500, 2501, 2700, 9201]
    check(make(9110, 9211, heads, kv, dh, ty, dh + heads, True), heads, kv,
          dh, rows, keys)
    check(make(9211, 9110, heads, kv, dh, ty, dh + heads, True), heads, kv,
          dh, keys, rows)
