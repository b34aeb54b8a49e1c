"""Cross attention at the largest numbers of clouds and of rows and heads that
it takes: more blocks, or more rows of D, than one row of a launch has."""
import pytest
import torch

from paper_2512_00385_amd import ezsp

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32
MOST = 1 << 24


@pytest.fixture(scope="module", autouse=True)
def gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    ezsp.load()
    yield


@pytest.mark.parametrize("kv,clouds", [(1, MOST), (2, MOST // 2)])
def test_most_clouds(kv, clouds):
    # a few of them hold rows and keys; the results are those of a batch of
    # these alone, bit for bit
    at = [0, 5, clouds // 2 - 1, clouds // 2, clouds - 2, clouds - 1]
    rows = [3, 70, 1, 200, 65, 9]
    keys = [4, 66, 130, 3, 17, 1]
    dh, heads = 16, 2
    g = torch.Generator(device="cuda")
    g.manual_seed(clouds)

    def normal(n, h):
        return torch.randn((n, h * dh), generator=g, device="cuda").to(BF)
    nq, nk = sum(rows) + 2, sum(keys) + 1
    q, dout = normal(nq, heads), normal(nq, heads)
    k, v = normal(nk, kv), normal(nk, kv)

    def offsets(counts, places, n):
        c = torch.zeros(n + 1, dtype=torch.int32, device="cuda")
        c[torch.tensor(places, device="cuda") + 1] = torch.tensor(
            counts, dtype=torch.int32, device="cuda")
        return c.cumsum(0).int()

    def both(places, n):
        kw = dict(q_offsets=offsets(rows, places, n),
                  k_offsets=offsets(keys, places, n))
        out, lse = ezsp.cross_attention(q, k, v, heads, kv, want_lse=True,
                                        **kw)
        return (out, lse, *ezsp.cross_attention_backward(
            dout, q, k, v, out, lse, heads, kv, **kw))
    for name, x, y in zip(("out", "lse", "dq", "dk", "dv"),
                          both(at, clouds), both(list(range(6)), 6)):
        assert torch.equal(x, y), name
    assert bool((x != 0).any())


def test_most_rows_and_heads():
    # 2^30 rows and heads; one key, S = 0 and so P = 1, whole numbers
    heads, nq = 32, (1 << 25) + 3
    q = torch.zeros((nq, heads), dtype=BF, device="cuda")
    k = torch.zeros((1, heads), dtype=BF, device="cuda")
    v = torch.arange(heads, device="cuda").to(BF)[None] + 1
    out, lse = ezsp.cross_attention(q, k, v, heads, want_lse=True)
    assert bool((out == v).all()) and bool((lse == 0).all())
    del lse
    out.zero_()
    dout = torch.zeros_like(q)
    for i, row in enumerate((0, 77, nq // 2, nq - 2, nq - 1)):
        q[row], dout[row], out[row] = i + 1, 2, i - 3
    # lse = 0 says P = 1
    lse = torch.zeros((heads, nq), device="cuda")
    dq, dk, dv = ezsp.cross_attention_backward(
        dout, q, k, v, out, lse, heads, want_dq=False)
    ds = [2 * v.double() - 2 * (i - 3) for i in range(5)]
    assert torch.equal(dk.double(), sum((i + 1) * d
                                        for i, d in enumerate(ds)).to(
        BF).double())
    assert bool((dv == 10).all())
