"""Train a small attention network to label the points of packed synthetic clouds.

    python examples/train_attention.py [--clouds 8] [--points 600] [--steps 30] [--dtype f32|bf16]

Every point attends to all points of its own cloud; queries and keys are normalised
and turned by the point's coordinates. The clouds have different lengths and lie one
behind the other:

    linear -> layer normalisation -> queries, keys, values -> rotation -> attention
    -> linear, added -> layer normalisation -> classifier and loss

All gradients are clipped by their common norm; the matrices then move along the
orthogonalised form of their momentum, the other parameters along it.
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2108_03917_amd import Dense  # noqa: E402

CLASSES, F_IN, WIDTH, HEADS, KV_HEADS, DIM = 8, 4, 64, 4, 2, 16
SECTIONS = (3, 3, 2)                      # pairs of a head's channels that turn with x, y and z
MATRICES = ("w_in", "w_qkv", "w_out", "cls")


def clouds(count, points, seed):
    """Points on blobs, packed: coordinates, features, labels (the octant about the
    cloud's first point; one in ten has none) and the clouds' starts."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    lengths = [max(1, points * (i + 1) // count) for i in range(count)]
    starts = torch.tensor([0] + lengths).cumsum(0).to(torch.int32).to("cuda")
    n = sum(lengths)
    pos = torch.randn(n, 3, generator=g, device="cuda")
    first = torch.repeat_interleave(starts[:-1].long(), torch.tensor(lengths, device="cuda"))
    label = ((pos > pos[first]) * torch.tensor([1, 2, 4], device="cuda")).sum(1)
    label[torch.rand(n, generator=g, device="cuda") < 0.1] = -100
    mark = (torch.arange(n, device="cuda") == first).float()     # which point is the first
    return pos, torch.cat([pos, mark[:, None]], 1), label, starts


class Net:
    def __init__(self, dtype="f32", seed=0):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)

        def weight(*shape):
            return torch.randn(*shape, generator=g, device="cuda") / math.sqrt(shape[-1])

        def ones(n):
            return torch.ones(n, device="cuda")

        self.type = torch.bfloat16 if dtype == "bf16" else torch.float32
        self.p = {"w_in": weight(WIDTH, F_IN), "gamma1": ones(WIDTH), "beta1": 0 * ones(WIDTH),
                  "w_qkv": weight((HEADS + 2 * KV_HEADS) * DIM, WIDTH), "gain_q": ones(DIM), "gain_k": ones(DIM),
                  "w_out": weight(WIDTH, HEADS * DIM), "gamma2": ones(WIDTH), "beta2": 0 * ones(WIDTH),
                  "cls": weight(CLASSES, WIDTH), "bias": 0 * ones(CLASSES)}
        self.freq = torch.cat([2.0 ** torch.arange(s, device="cuda") for s in SECTIONS]).float()
        self.momentum = {k: torch.zeros_like(v) for k, v in self.p.items()}

    def gradients(self, ops, pos, feat, label, starts):
        """The loss and the gradients of all parameters."""
        p = {k: v.to(self.type) if k in MATRICES else v for k, v in self.p.items()}
        n = feat.shape[0]
        feat = feat.to(self.type)
        x0 = feat @ p["w_in"].t()
        n1, mean1, rstd1 = ops.layer_norm(x0, p["gamma1"], p["beta1"], want_stats=True)
        qkv = (n1 @ p["w_qkv"].t()).view(n, HEADS + 2 * KV_HEADS, DIM)
        q0, k0, v = qkv.split((HEADS, KV_HEADS, KV_HEADS), 1)
        turn = (pos, self.freq, SECTIONS, p["gain_q"], p["gain_k"])
        q, k = ops.rotate_heads(q0, k0, *turn)
        o, lse = ops.attention(q, k, v, starts, want_lse=True)
        x1 = x0 + o.view(n, -1) @ p["w_out"].t()
        n2, mean2, rstd2 = ops.layer_norm(x1, p["gamma2"], p["beta2"], want_stats=True)
        loss, g_n2, g_cls, g_bias = ops.linear_cross_entropy(n2, p["cls"], label, p["bias"], want_grad=True)

        g_x1, g_gamma2, g_beta2 = ops.layer_norm_backward(g_n2, x1, mean2, rstd2, p["gamma2"])
        g_o = (g_x1 @ p["w_out"]).view(n, HEADS, DIM)
        g_q, g_k, g_v = ops.attention_backward(g_o, q, k, v, o, lse, starts)
        g_q0, g_k0, g_gain_q, g_gain_k = ops.rotate_heads_backward(g_q, g_k, q0, k0, *turn)
        g_qkv = torch.cat([g_q0, g_k0, g_v], 1).view(n, -1)
        g_x0, g_gamma1, g_beta1 = ops.layer_norm_backward(g_qkv @ p["w_qkv"], x0, mean1, rstd1, p["gamma1"])
        g_x0 = g_x0 + g_x1
        return loss, {"w_in": g_x0.t() @ feat, "gamma1": g_gamma1, "beta1": g_beta1, "w_qkv": g_qkv.t() @ n1,
                      "gain_q": g_gain_q, "gain_k": g_gain_k, "w_out": g_x1.t() @ o.view(n, -1), "gamma2": g_gamma2,
                      "beta2": g_beta2, "cls": g_cls, "bias": g_bias}

    def step(self, ops, batch, lr, most):
        loss, grads = self.gradients(ops, *batch)
        clipped = {k: torch.empty_like(self.p[k]) for k in grads}
        norm = ops.clip_gradients([g.contiguous() for g in grads.values()], most, out=list(clipped.values()))
        for k, g in clipped.items():
            m = self.momentum[k].mul_(0.9).add_(g)
            if k in MATRICES:
                self.p[k].add_(ops.orthogonalize(m), alpha=-lr * math.sqrt(max(1.0, m.shape[0] / m.shape[1])))
            else:
                self.p[k].add_(m, alpha=-lr)
        return loss, norm


def train(count=8, points=600, steps=30, dtype="f32", lr=0.02, most=1.0, log=print):
    batch = clouds(count, points, seed=1)
    ops = Dense()
    net = Net(dtype)
    losses = []
    for i in range(steps):
        loss, norm = net.step(ops, batch, lr, most)
        losses.append(loss)
        if log and (i % 5 == 0 or i + 1 == steps):
            log(f"step {i:3d}  loss {loss.item():.4f}  norm of the gradients {norm.item():.4f}")
    losses = torch.stack(losses).tolist()
    ops.close()
    return losses


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--clouds", type=int, default=8)
    ap.add_argument("--points", type=int, default=600)
    ap.add_argument("--steps", type=int, default=30)
    ap.add_argument("--dtype", choices=("f32", "bf16"), default="f32")
    a = ap.parse_args()
    train(a.clouds, a.points, a.steps, a.dtype)
