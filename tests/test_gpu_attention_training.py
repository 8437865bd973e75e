"""The operators together, as a training step uses them: the example's gradients
against those of the same network in 64 bits, from its formulas by autograd.

Tolerance: the relative 2-norm of each parameter's gradient.  Some 16 operators and
products lie between a parameter and the loss and back, each off by at most 1e-5 of
what it adds up in fp32 (REL_F32), and 2^-8 of it in bf16 (a rounding or two); the sizes
of what is added up are within 6 times those of the results: 16 x 6 x 1e-5 = 1e-3, and
in bf16 16 x 2^-8 = 0.0625 for roundings of random sign, which add up as the root
of their number at most times 6 / 4.
"""
import importlib.util
import math
import os

import pytest
import torch

from tests.test_gpu_dense import DEV, _gpu, ops  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def example():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "train_attention.py")
    spec = importlib.util.spec_from_file_location("train_attention", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def reference(example, net, pos, feat, label, starts):
    """Loss and gradients in 64 bits."""
    E = example
    p = {k: v.double().requires_grad_() for k, v in net.p.items()}
    n = feat.shape[0]

    def norm(x, gamma, beta):
        d = x - x.mean(1, keepdim=True)
        return d / (d.square().mean(1, keepdim=True) + 1e-5).sqrt() * gamma + beta

    axis = torch.repeat_interleave(torch.arange(3), torch.tensor(E.SECTIONS)).to(DEV)
    angle = (pos.double()[:, axis] * net.freq.double())[:, None]

    def turn(x, gain):
        x = x / (x.square().mean(-1, keepdim=True) + 1e-6).sqrt() * gain
        h = angle.shape[-1]
        a, b = x[..., :h], x[..., h:2 * h]
        return torch.cat([a * angle.cos() - b * angle.sin(), b * angle.cos() + a * angle.sin(), x[..., 2 * h:]], -1)

    x0 = feat.double() @ p["w_in"].t()
    qkv = (norm(x0, p["gamma1"], p["beta1"]) @ p["w_qkv"].t()).view(n, -1, E.DIM)
    q, k, v = qkv.split((E.HEADS, E.KV_HEADS, E.KV_HEADS), 1)
    q, k = turn(q, p["gain_q"]), turn(k, p["gain_k"])
    at, out = starts.tolist(), []
    for a, b in zip(at, at[1:]):
        heads = []
        for h in range(E.HEADS):
            kh = h * E.KV_HEADS // E.HEADS
            heads.append(torch.softmax(q[a:b, h] @ k[a:b, kh].t() / math.sqrt(E.DIM), 1) @ v[a:b, kh])
        out.append(torch.stack(heads, 1))
    x1 = x0 + torch.cat(out).reshape(n, -1) @ p["w_out"].t()
    z = norm(x1, p["gamma2"], p["beta2"]) @ p["cls"].t() + p["bias"]
    loss = torch.nn.functional.cross_entropy(z, label)
    loss.backward()
    return loss.detach(), {k: t.grad for k, t in p.items()}


@pytest.mark.parametrize("dtype,most", [("f32", 1e-3), ("bf16", 0.0625 * 6 / 4)])
@pytest.mark.parametrize("count,points", [(1, 50), (5, 300), (40, 90)])
def test_gradients_of_a_training_step(ops, example, count, points, dtype, most):  # noqa: F811
    net = example.Net(dtype, seed=3)
    batch = example.clouds(count, points, seed=count)
    loss, grads = net.gradients(ops, *batch)
    ref_loss, ref = reference(example, net, *batch)
    assert abs(loss.item() - ref_loss.item()) <= most * abs(ref_loss.item())
    for k, r in ref.items():
        off = (grads[k].double() - r).norm() / r.norm()
        assert off <= most, (k, off.item())
    clipped = {k: torch.empty_like(net.p[k]) for k in grads}
    norm = ops.clip_gradients([g.contiguous() for g in grads.values()], 0.1, out=list(clipped.values()))
    whole = math.sqrt(sum(r.square().sum().item() for r in ref.values()))
    assert abs(norm.item() - whole) <= most * whole
    for k, r in ref.items():
        assert (clipped[k].double() - r * min(1.0, 0.1 / whole)).norm() <= 2 * most * r.norm() * min(1.0, 0.1 / whole), k


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_example_runs(example, dtype):
    losses = example.train(count=3, points=200, steps=4, dtype=dtype, log=None)
    assert len(losses) == 4 and all(math.isfinite(v) for v in losses)
