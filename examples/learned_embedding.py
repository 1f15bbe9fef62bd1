"""Clusters raw measurements in an embedding that an autoencoder learns.

    python examples/learned_embedding.py [--n 8192] [--steps 60] [--dtype bfloat16]

The measurements are blobs seen through a random nonlinear map, beside
columns of noise.  The encoder is an input layer, a gated block with its
residual and a projection to 16 coordinates; the decoder mirrors it with one
hidden layer.  Training uses the package's layers and their gradients, the
weight matrices move by gpic_muon_step, the biases by plain descent.  Then
power iteration clustering runs over the embedded points, and single points
go through the encoder as a service would send them.
"""
from __future__ import annotations

import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_1604_02700_amd as g  # noqa: E402


def measurements(n, clusters=5, latent=6, seen=96, noise=64, seed=0, device="cuda"):
    """(X float32 [n, seen + noise], true cluster of each point)."""
    gen = torch.Generator().manual_seed(seed)
    centres = 6.0 * torch.randn((clusters, latent), generator=gen)
    label = torch.randint(clusters, (n,), generator=gen)
    z = centres[label] + torch.randn((n, latent), generator=gen)
    A = torch.randn((latent, seen), generator=gen) / latent ** 0.5
    X = torch.cat([torch.tanh(0.3 * (z @ A)), 0.1 * torch.randn((n, noise), generator=gen)], 1)
    return X.to(device), label.to(device)


class Autoencoder:
    """Weights, their momenta, and one training step."""

    def __init__(self, inputs, width, hidden, out, dtype, seed=1, device="cuda"):
        gen = torch.Generator().manual_seed(seed)

        def weight(m, k):
            return (torch.randn((m, k), generator=gen) / k ** 0.5).to(device=device, dtype=dtype)

        self.W = {"in": weight(width, inputs), "gate": weight(2 * hidden, width),
                  "down": weight(width, hidden), "embed": weight(out, width),
                  "up": weight(width, out), "out": weight(inputs, width)}
        self.b = {k: torch.zeros(self.W[k].shape[0], dtype=dtype, device=device)
                  for k in ("in", "embed", "up", "out")}
        self.M = {k: torch.zeros(w.shape, dtype=torch.float32, device=device)
                  for k, w in self.W.items()}

    def encode(self, X):
        W, b = self.W, self.b
        h = g.gpic_linear(X, W["in"], b["in"], "gelu")
        h = g.gpic_linear(g.gpic_gated(h, W["gate"]), W["down"], None, "none", residual=h)
        return g.gpic_linear(h, W["embed"], b["embed"])

    def step(self, X, lr):
        """One pass forward and back over X and one update; the loss (a
        tensor: nothing waits for it here)."""
        W, b = self.W, self.b
        h0, z0 = g.gpic_linear(X, W["in"], b["in"], "gelu", want_pre=True)
        a, za = g.gpic_gated(h0, W["gate"], want_pre=True)
        h1 = g.gpic_linear(a, W["down"], None, "none", residual=h0)
        e = g.gpic_linear(h1, W["embed"], b["embed"])
        h2, z2 = g.gpic_linear(e, W["up"], b["up"], "gelu", want_pre=True)
        y = g.gpic_linear(h2, W["out"], b["out"])
        r = y.float() - X.float()
        loss = r.square().mean()

        dy = (r * (2.0 / X.shape[0])).to(X.dtype)
        d_out = g.gpic_linear_backward(dy, h2, W["out"])
        d_up = g.gpic_linear_backward(d_out.dX, e, W["up"], z2, "gelu")
        d_embed = g.gpic_linear_backward(d_up.dX, h1, W["embed"])
        d_down = g.gpic_linear_backward(d_embed.dX, a, W["down"], want_bias=False)
        d_gate = g.gpic_gated_backward(d_down.dX, h0, W["gate"], za)
        # h0 feeds the gated block and, as the residual, its end
        d_in = g.gpic_linear_backward(d_gate.dX + d_embed.dX, X, W["in"], z0, "gelu", want_x=False)

        grads = {"in": d_in, "gate": d_gate, "down": d_down, "embed": d_embed, "up": d_up,
                 "out": d_out}
        for k, d in grads.items():
            g.gpic_muon_step(W[k], d.dW, self.M[k], lr, momentum=0.9)
            if k in b:
                b[k].sub_(d.db, alpha=lr)
        return loss


def run(n=8192, steps=60, dtype=torch.bfloat16, seed=0, say=print):
    X, label = measurements(n, seed=seed)
    net = Autoencoder(X.shape[1], 128, 192, 16, dtype)
    data = X.to(dtype)
    losses = []
    t = time.perf_counter()
    for i in range(steps):
        losses.append(net.step(data, 0.05 * (1.0 - i / steps)))
    losses = [float(v) for v in losses]
    say(f"{steps} steps over {n} points: loss {losses[0]:.4f} -> {losses[-1]:.4f} "
        f"({time.perf_counter() - t:.2f} s with the first launches)")

    E = net.encode(data).float()
    # the width of the affinity: a fifth of the typical distance
    a, c = E[torch.randperm(n, device=E.device)[:1024]], E[:1024]
    sigma = 0.2 * float(torch.cdist(a, c).median())
    k = int(label.max()) + 1
    out = g.pic_dense(E, sigma, k, "converge", 1000, 1e-5 / n)
    got = out.km.labels.long()
    # purity: the share of points in the majority class of their cluster
    table = torch.zeros((k, k), device=E.device)
    table.index_put_((got, label), torch.ones(n, device=E.device), accumulate=True)
    purity = float(table.max(1).values.sum()) / n
    say(f"clusters of the embedding: {out.pi.iterations} updates, sigma {sigma:.3f}, "
        f"purity {purity:.3f}")
    one = torch.cat([net.encode(data[i:i + 1]) for i in range(8)])
    return {"losses": losses, "embedding": E, "sigma": sigma, "clusters": out, "k": k,
            "purity": purity, "one": one.float()}


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__,
                                 formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--n", type=int, default=8192)
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--dtype", default="bfloat16", choices=("float32", "float16", "bfloat16"))
    o = ap.parse_args()
    run(o.n, o.steps, getattr(torch, o.dtype))
