"""A trainable point-embedding network on the library's dense operators.

The partition works on per-point embeddings that a network is trained to
produce with the contrastive edge loss (Sec. 3.1).  This one is a stack of
pre-norm residual blocks of gated feed-forward products,

  s_0 = x W_in + b_in
  s_i = s_{i-1} + (silu(n W_g + b_g) * (n W_u + b_u)) W_d + b_d,
        n = layer_norm(s_{i-1})
  e   = layer_norm(s_L) W_out + b_out,

with bfloat16 weights and activations and an fp32 residual stream; the
embeddings e are fp32.  ``forward`` and ``backward`` are sequences of library
calls (ezsp_linear, ezsp_layer_norm, ezsp_gated_ff and their backward
passes, ezsp_edge_loss for the gradient at the end), ``step`` one step of
gradient descent with momentum on fp32 copies of the weights.

  python -m paper_2512_00385_amd.embed_net [--points N] [--steps N]

trains one on a synthetic cloud and partitions it with the embeddings before
and after.
"""
from __future__ import annotations

import torch

from . import ezsp


class EmbedNet:
    def __init__(self, d_in: int, d_out: int = 32, width: int = 32,
                 hidden: int = 128, blocks: int = 2, seed: int = 0,
                 device="cuda"):
        g = torch.Generator(device=device)
        g.manual_seed(seed)
        self.blocks = blocks

        def mat(k, m, scale=1.0):
            w = torch.rand((k, m), generator=g, device=device)
            return (2 * w - 1) * (scale / k ** 0.5)

        def vec(m, value=0.0):
            return torch.full((m,), value, device=device)
        master = {"w_in": mat(d_in, width), "b_in": vec(width)}
        for i in range(blocks):
            master.update({
                f"n{i}_w": vec(width, 1.0), f"n{i}_b": vec(width),
                f"g{i}_w": mat(width, hidden), f"g{i}_b": vec(hidden),
                f"u{i}_w": mat(width, hidden), f"u{i}_b": vec(hidden),
                f"d{i}_w": mat(hidden, width), f"d{i}_b": vec(width)})
        master.update({"n_w": vec(width, 1.0), "n_b": vec(width),
                       "w_out": mat(width, d_out), "b_out": vec(d_out)})
        self.master = master
        self.speed = {k: torch.zeros_like(v) for k, v in master.items()}
        self._round()

    def _round(self):
        """The parameters as the operators take them: matrices rounded to
        bfloat16, vectors as they are."""
        self.p = {k: v.bfloat16() if v.dim() == 2 else v
                  for k, v in self.master.items()}

    def forward(self, x: torch.Tensor, train: bool = False):
        """Embeddings [n, d_out] fp32 of features x [n, d_in] bfloat16; with
        train also what backward needs."""
        p, f32 = self.p, torch.float32
        s = ezsp.linear(x, p["w_in"], p["b_in"], out_dtype=f32)
        saved = []
        for i in range(self.blocks):
            n, mean, rstd = ezsp.layer_norm(
                s, p[f"n{i}_w"], p[f"n{i}_b"], out_dtype=torch.bfloat16,
                want_stats=True)
            h = ezsp.gated_ff(n, p[f"g{i}_w"], p[f"u{i}_w"], p[f"g{i}_b"],
                              p[f"u{i}_b"], want_saved=train)
            if train:
                h, gate, up = h
                saved.append((s, mean, rstd, n, h, gate, up))
            s = ezsp.linear(h, p[f"d{i}_w"], p[f"d{i}_b"], residual=s,
                            out_dtype=f32)
        n, mean, rstd = ezsp.layer_norm(s, p["n_w"], p["n_b"],
                                        out_dtype=torch.bfloat16,
                                        want_stats=True)
        e = ezsp.linear(n, p["w_out"], p["b_out"], out_dtype=f32)
        return (e, (x, saved, s, mean, rstd, n)) if train else e

    def backward(self, de: torch.Tensor, saved):
        """Gradients of all parameters from the embeddings' (fp32)."""
        p = self.p
        x, blocks, s, mean, rstd, n = saved
        grad = {}
        dn, grad["w_out"], grad["b_out"] = ezsp.linear_backward(
            de, n, p["w_out"])
        ds, grad["n_w"], grad["n_b"] = ezsp.layer_norm_backward(
            dn, s, mean, rstd, p["n_w"])
        for i in reversed(range(self.blocks)):
            s, mean, rstd, n, h, gate, up = blocks[i]
            dh, grad[f"d{i}_w"], grad[f"d{i}_b"] = ezsp.linear_backward(
                ds, h, p[f"d{i}_w"])
            dn, grad[f"g{i}_w"], grad[f"u{i}_w"], grad[f"g{i}_b"], \
                grad[f"u{i}_b"] = ezsp.gated_ff_backward(
                    dh, n, p[f"g{i}_w"], p[f"u{i}_w"], gate, up)
            # the residual branch joins the norm's gradient
            ds, grad[f"n{i}_w"], grad[f"n{i}_b"] = ezsp.layer_norm_backward(
                dn, s, mean, rstd, p[f"n{i}_w"], dres=ds)
        _, grad["w_in"], grad["b_in"] = ezsp.linear_backward(
            ds, x, p["w_in"], want_dx=False)
        return grad

    def step(self, x, nbr, cls, word, lr: float = 0.05,
             momentum: float = 0.9, tau: float = 1.0, rho: float = 0.3):
        """One training step on the pairs of a neighbour table (arguments as
        ezsp.edge_loss); the loss per sampled pair."""
        e, saved = self.forward(x, train=True)
        stats, _, de, _ = ezsp.edge_loss(e, nbr, cls, word, tau, rho,
                                         want_affinity=False,
                                         want_sampled=False)
        pairs = max(1, stats["n_inter"] + stats["n_intra_kept"])
        grad = self.backward(de / pairs, saved)
        for k, w in self.master.items():
            v = self.speed[k].mul_(momentum).add_(grad[k].float())
            w.sub_(v, alpha=lr)
        self._round()
        return stats["loss"] / pairs


def main():
    import argparse

    import numpy as np

    from . import scenes
    ap = argparse.ArgumentParser()
    ap.add_argument("--points", type=int, default=100_000)
    ap.add_argument("--steps", type=int, default=100)
    args = ap.parse_args()
    sc = scenes.random_cloud(args.points, 8, seed=0, n_obj=24)
    dev = torch.device("cuda")
    xyz = torch.from_numpy(sc.xyz).to(dev)
    cls = torch.from_numpy(sc.obj.astype(np.int32)).to(dev)
    # features: position, and an intensity of each object with noise
    rng = np.random.default_rng(1)
    tone = rng.uniform(0, 1, (24, 3))[sc.obj] + \
        0.05 * rng.standard_normal((sc.n, 3))
    x = torch.cat([xyz, torch.from_numpy(tone.astype(np.float32)).to(dev)],
                  1).bfloat16()
    nbr = ezsp.knn(xyz, 10)
    g = torch.Generator(device=dev)
    g.manual_seed(2)
    net = EmbedNet(6, d_out=16)

    def score():
        labels, nc, _ = ezsp.partition(xyz, net.forward(x), 10, [0.1])
        stats, _, _ = ezsp.purity(labels[0], int(nc[0]), cls, 24)
        return int(nc[0]), stats["purity"]
    print("before: %d superpoints, purity %.4f" % score(), flush=True)
    for i in range(args.steps):
        word = torch.randint(-2 ** 31, 2 ** 31, nbr.shape, generator=g,
                             dtype=torch.int64, device=dev).int()
        loss = net.step(x, nbr, cls, word)
        if i % 20 == 0 or i + 1 == args.steps:
            print(f"step {i}: loss per pair {loss:.4f}", flush=True)
    print("after:  %d superpoints, purity %.4f" % score(), flush=True)


if __name__ == "__main__":
    main()
