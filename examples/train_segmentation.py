"""Train a small lattice network to label the points of a synthetic cloud.

    python examples/train_segmentation.py [--points 20000] [--steps 30] [--dtype f32|bf16]

Every step runs on the library's kernels, forward and backward:

    splat -> conv -> layer normalisation -> ReLU -> conv -> slice -> classifier and loss

The convolutions' weights move along the orthogonalised form of their (momentum)
gradients, the other parameters along the gradients themselves.
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2108_03917_amd import Dense, Lattice  # noqa: E402

CLASSES, CHANNELS, F_IN = 8, 64, 4


def cloud(points, seed):
    """Points on a few blobs, labelled by octant; one in ten has no label."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    centre = torch.rand(16, 3, generator=g, device="cuda") * 2 - 1
    which = torch.randint(0, 16, (points,), generator=g, device="cuda")
    pos = centre[which] + 0.15 * torch.randn(points, 3, generator=g, device="cuda")
    label = ((pos > 0) * torch.tensor([1, 2, 4], device="cuda")).sum(1)
    label[torch.rand(points, generator=g, device="cuda") < 0.1] = -100
    feat = torch.cat([pos, torch.ones(points, 1, device="cuda")], 1).contiguous()
    return pos.contiguous(), feat, label


class Net:
    def __init__(self, taps, dtype, seed=0):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)

        def weight(*shape):
            fan = math.prod(shape[1:])
            return torch.randn(*shape, generator=g, device="cuda") / math.sqrt(fan)

        self.dtype = dtype
        self.p = {"w1": weight(CHANNELS, taps, F_IN), "w2": weight(CHANNELS, taps, CHANNELS),
                  "gamma": torch.ones(CHANNELS, device="cuda"), "beta": torch.zeros(CHANNELS, device="cuda"),
                  "cls": weight(CLASSES, CHANNELS), "bias": torch.zeros(CLASSES, device="cuda")}
        self.momentum = {k: torch.zeros_like(v) for k, v in self.p.items()}

    def step(self, L, ops, pos, feat, label, lr):
        p = self.p
        x0, _ = L.splat(pos, feat, normalize=True)
        w1, w2 = (L.weights_to_bf16(p[k]) if self.dtype == "bf16" else p[k] for k in ("w1", "w2"))
        x1 = L.conv(x0, w1, self.dtype)
        n1, mean, rstd = ops.layer_norm(x1, p["gamma"], p["beta"], lattice=L, want_stats=True)
        x2 = torch.relu(n1)
        x3 = L.conv(x2, w2, self.dtype)
        f = L.slice(x3)
        loss, g_f, g_cls, g_bias = ops.linear_cross_entropy(f, p["cls"], label, p["bias"], want_grad=True)
        g3 = L.slice_backward(g_f)
        g2, g_w2, _ = L.conv_backward(g3, w2, x2, self.dtype)
        g_n1 = torch.where(n1 > 0, g2, 0.0)
        g1, g_gamma, g_beta = ops.layer_norm_backward(g_n1, x1, mean, rstd, p["gamma"], lattice=L)
        _, g_w1, _ = L.conv_backward(g1, w1, x0, self.dtype, want_input=False)
        grads = {"w1": g_w1, "w2": g_w2, "gamma": g_gamma, "beta": g_beta, "cls": g_cls, "bias": g_bias}
        for k, g in grads.items():
            m = self.momentum[k].mul_(0.9).add_(g)
            if k in ("w1", "w2"):    # as a matrix of outputs x (taps and inputs)
                rows, cols = m.shape[0], m[0].numel()
                o = ops.orthogonalize(m.view(rows, cols))
                p[k].view(rows, cols).add_(o, alpha=-lr * math.sqrt(max(1.0, rows / cols)))
            else:
                p[k].add_(m, alpha=-lr)
        return loss


def train(points=20000, steps=30, dtype="f32", lr=0.03, log=print):
    pos, feat, label = cloud(points, seed=1)
    L = Lattice(3, 0.1, max_points=points)
    ops = Dense()
    net = Net(L.taps, dtype)
    losses = []
    for i in range(steps):
        losses.append(net.step(L, ops, pos, feat, label, lr))
        if log and (i % 5 == 0 or i + 1 == steps):
            log(f"step {i:3d}  loss {losses[-1].item():.4f}")
    losses = torch.stack(losses).tolist()
    ops.close()
    L.close()
    return losses


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--points", type=int, default=20000)
    ap.add_argument("--steps", type=int, default=30)
    ap.add_argument("--dtype", choices=("f32", "bf16"), default="f32")
    a = ap.parse_args()
    train(a.points, a.steps, a.dtype)
