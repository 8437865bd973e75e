"""Clipping by the norm over many tensors, against a plain 64-bit implementation.

Tolerances, fixed from the arithmetic: the norm is a sum in fp64, rounded to fp32
once (2^-24 of itself); the factor is rounded once and the product once more (2
times 2^-24), or to bf16 (2^-8) in place of the latter.
"""
import math

import pytest
import torch

from tests.test_gpu_dense import DEV, HALF, T, _gpu, ops, rand  # noqa: F401

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


def check(ops, grads, most, eps=1e-6, out=None):  # noqa: F811
    before = [g.clone() for g in grads]
    norm = ops.clip_gradients(grads, most, eps, out)
    ref = math.sqrt(sum(g.double().square().sum().item() for g in before))
    assert abs(norm.item() - ref) <= U * 1.01 * ref, (norm.item(), ref)
    factor = min(1.0, most / (ref + eps)) if ref else 1.0
    for i, (a, b) in enumerate(zip(before, grads if out is None else out)):
        want = a.double() * factor
        half = HALF if b.dtype == torch.bfloat16 else U
        err = (b.double() - want).abs()
        # values below the least normal one are spaced evenly
        assert torch.all(err <= (half + 2 * U) * want.abs() + 2.0 ** -126 * half), i
        if out is not None:
            assert torch.equal(grads[i], a)
    return norm


SIZES = [[1], [7], [8, 1, 0, 33], [16384], [16385, 3, 16383], [100003], [5] * 200, [1000, 2000001], list(range(100))]


@pytest.mark.parametrize("sizes", SIZES, ids=[f"{len(s)}x{max(s)}" for s in SIZES])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "both"])
@pytest.mark.parametrize("share", [0.3, 3.0])
def test_clip(ops, sizes, dtype, share):  # noqa: F811
    kinds = ["f32", "bf16"] if dtype == "both" else [dtype]
    grads = [rand(i, n, dtype=kinds[i % len(kinds)]) * 10.0 ** (i % 3 - 1) for i, n in enumerate(sizes)]
    norm = math.sqrt(sum(g.double().square().sum().item() for g in grads))
    out = [torch.full_like(g, 7.0) for g in grads]
    check(ops, grads, share * norm, out=out)
    wide = [torch.full(g.shape, 7.0, device=DEV) for g in grads]
    check(ops, grads, share * norm, out=wide)
    if dtype == "f32":
        check(ops, grads, share * norm, out=[torch.full(g.shape, 7.0, device=DEV, dtype=T["bf16"]) for g in grads])
    before = [g.clone() for g in grads]
    check(ops, grads, share * norm)
    if share > 1:
        assert all(torch.equal(a, b) for a, b in zip(before, grads))


def test_more_than_2_31_values(ops):  # noqa: F811
    """The norm and the scaled values are exact here: 2^32 squares of 1/4, and a factor of
    2^-10; two values behind the 2^31st one are not as the others."""
    x = torch.full((1 << 32,), 0.5, device=DEV, dtype=torch.bfloat16)
    x[(1 << 31) + 5], x[-1] = -0.5, -0.5
    want = x * 2.0 ** -10
    norm = ops.clip_gradients([x[:5], x[5:]], 2.0 ** 5, 0.0)
    assert norm.item() == 2.0 ** 15 and torch.equal(x, want)


def test_shapes_and_odd_addresses(ops):  # noqa: F811
    flat = rand(1, 10000)
    half = rand(2, 10000, dtype="bf16")
    check(ops, [flat[1:1000], flat[1003:1003 + 24].view(2, 3, 4), half[1:18], half[19:5000].view(-1, 17), flat[5000]], 0.5)


def test_very_large_and_very_small_values(ops):  # noqa: F811
    """Squares that fp32 does not hold."""
    check(ops, [rand(1, 1000) * 1e30, rand(2, 1000)], 1.0)
    check(ops, [rand(1, 1000) * 1e-30], 1e-29, eps=0.0)


def test_zeros(ops):  # noqa: F811
    for most in (0.0, 1.0):
        for eps in (0.0, 1e-6):
            g = [torch.zeros(100, device=DEV), torch.zeros(3, device=DEV, dtype=T["bf16"])]
            assert ops.clip_gradients(g, most, eps).item() == 0
            assert all(torch.all(x == 0) for x in g)
    g = [rand(1, 100)]
    ops.clip_gradients(g, 0.0)
    assert torch.all(g[0] == 0)


def test_nothing_to_clip(ops):  # noqa: F811
    assert ops.clip_gradients([], 1.0).item() == 0
    assert ops.clip_gradients([torch.empty(0, 5, device=DEV)], 1.0).item() == 0
    assert ops.clip_gradients([torch.empty(0, device=DEV)] * 300 + [torch.full((4,), 1.0, device=DEV)], 9.0).item() == 2


def test_not_finite(ops):  # noqa: F811
    g = [rand(1, 100), rand(2, 5000)]
    g[1][77] = float("nan")
    assert torch.isnan(ops.clip_gradients(g, 1.0)) and all(torch.isnan(x).all() for x in g)
    g = [rand(1, 100), rand(2, 5000)]
    g[0][3] = float("inf")
    assert torch.isinf(ops.clip_gradients(g, 1.0))
    assert torch.isnan(g[0][3]) and torch.all(g[1] == 0) and torch.isnan(g[0]).sum() == 1
    g = [rand(1, 100)]
    before = g[0].clone()
    ops.clip_gradients(g, math.inf)
    assert torch.equal(g[0], before)


def test_refusals(ops):  # noqa: F811
    from paper_2108_03917_amd import LatticeError

    a, b = rand(1, 64), rand(2, 64)
    for bad in (lambda: ops.clip_gradients([a.half()], 1.0), lambda: ops.clip_gradients([a.cpu()], 1.0),
                lambda: ops.clip_gradients([rand(1, 8, 8).t()], 1.0), lambda: ops.clip_gradients([a], 1.0, out=[]),
                lambda: ops.clip_gradients([a], 1.0, out=[b[:32]])):
        with pytest.raises(ValueError):
            bad()
    c = rand(3, 128)
    before = a.clone(), b.clone(), c.clone()
    for bad in (lambda: ops.clip_gradients([a, a], 1.0), lambda: ops.clip_gradients([a, a[10:20]], 1.0),
                lambda: ops.clip_gradients([a, b], 1.0, out=[b, a]), lambda: ops.clip_gradients([a, b], 1.0, out=[c[:64], c[32:96]]),
                lambda: ops.clip_gradients([c[:64]], 1.0, out=[c[1:65]]), lambda: ops.clip_gradients([a], -1.0),
                lambda: ops.clip_gradients([a], float("nan")), lambda: ops.clip_gradients([a], 1.0, eps=-1.0)):
        with pytest.raises(LatticeError):
            bad()
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(before, (a, b, c)))
    ops.clip_gradients([a, a, a[3:9]], 1.0, out=[b, c[:64], c[64:70]])      # inputs may be the same


def test_same_bits_and_graph(_gpu):  # noqa: F811
    from paper_2108_03917_amd import Dense

    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    own = Dense(side)
    g = [rand(i, 1 + 7001 * i, dtype=("f32", "bf16")[i % 2]) for i in range(90)]
    out = [torch.empty_like(x) for x in g]
    n0 = own.clip_gradients(g, 1.0, out=out)
    first = [x.clone() for x in out]
    assert torch.equal(own.clip_gradients(g, 1.0, out=out), n0) and all(torch.equal(a, b) for a, b in zip(first, out))
    with torch.cuda.stream(side):
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            norm = own.clip_gradients(g, 1.0, out=out)
        for i in range(3):
            g[5].copy_(rand(100 + i, 1 + 7001 * 5, dtype="bf16") * (1 + i))
            graph.replay()
            side.synchronize()
            got = [norm.clone()] + [x.clone() for x in out]
            want = [own.clip_gradients(g, 1.0, out=out), *out]
            side.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(got, want)), i
    own.close()
