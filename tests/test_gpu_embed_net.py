"""The example network: its gradients against the same network in 64 bits
(weights as rounded, by torch's differentiation), and that training lowers
the edge loss."""
import numpy as np
import pytest
import torch

from paper_2512_00385_amd import ezsp, scenes
from paper_2512_00385_amd.embed_net import EmbedNet

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    ezsp.load()
    yield


def forward64(net, p, x):
    def norm(s, w, b):
        c = s - s.mean(1, keepdim=True)
        return c * ((c * c).mean(1, keepdim=True) + 1e-5) ** -0.5 * w + b
    s = x.double() @ p["w_in"] + p["b_in"]
    for i in range(net.blocks):
        n = norm(s, p[f"n{i}_w"], p[f"n{i}_b"])
        g = n @ p[f"g{i}_w"] + p[f"g{i}_b"]
        u = n @ p[f"u{i}_w"] + p[f"u{i}_b"]
        s = s + (g * torch.sigmoid(g) * u) @ p[f"d{i}_w"] + p[f"d{i}_b"]
    return norm(s, p["n_w"], p["n_b"]) @ p["w_out"] + p["b_out"]


@pytest.mark.parametrize("n,d_in,width,hidden", [(500, 6, 32, 128),
                                                 (1003, 9, 40, 100),
                                                 (300, 16, 200, 520)])
def test_against_64_bits(n, d_in, width, hidden):
    net = EmbedNet(d_in, d_out=16, width=width, hidden=hidden, seed=n)
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    x = torch.randn((n, d_in), generator=g, device="cuda").bfloat16()
    de = torch.randn((n, 16), generator=g, device="cuda")
    e, saved = net.forward(x, train=True)
    assert torch.equal(e, net.forward(x))
    grad = net.backward(de, saved)
    p = {k: v.double().cpu().requires_grad_() for k, v in net.p.items()}
    ref = forward64(net, p, x.cpu())
    (ref * de.double().cpu()).sum().backward()
    # about ten bfloat16 roundings (2^-8 each at most, errors of either
    # sign) lie between the inputs and a result; in the norm of a whole
    # tensor they stay below 10 * 2^-8 / sqrt(3) = 0.023
    def off(a, b):
        return float((a.double().cpu() - b).norm() / b.norm())
    assert off(e, ref.detach()) < 0.023
    for k, v in grad.items():
        assert v.shape == p[k].shape
        assert off(v, p[k].grad) < 0.023, k
    assert set(grad) == set(net.p)


def test_training_lowers_the_edge_loss():
    sc = scenes.random_cloud(20_001, 8, seed=3, n_obj=12)
    xyz = torch.from_numpy(sc.xyz).cuda()
    cls = torch.from_numpy(sc.obj.astype(np.int32)).cuda()
    rng = np.random.default_rng(0)
    tone = rng.uniform(0, 1, (12, 3))[sc.obj] + \
        0.05 * rng.standard_normal((sc.n, 3))
    x = torch.cat([xyz, torch.from_numpy(tone.astype(np.float32)).cuda()],
                  1).bfloat16()
    nbr = ezsp.knn(xyz, 8)
    g = torch.Generator(device="cuda")
    g.manual_seed(4)
    net = EmbedNet(6, d_out=16, seed=5)
    losses = []
    for _ in range(60):
        word = torch.randint(-2 ** 31, 2 ** 31, nbr.shape, generator=g,
                             dtype=torch.int64, device="cuda").int()
        losses.append(net.step(x, nbr, cls, word))
    assert np.isfinite(losses).all()
    assert np.mean(losses[-5:]) < 0.7 * np.mean(losses[:5]), losses
    labels, nc, _ = ezsp.partition(xyz, net.forward(x), 8, [0.1])
    assert 1 <= int(nc[0]) <= sc.n
