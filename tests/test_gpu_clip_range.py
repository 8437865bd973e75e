"""Clipping with norms that fp32 does not hold, with factors below its least normal number,
and without a largest norm.

Tolerances as in test_gpu_clip: a factor rounded once to 24 bits and the product once more,
2 x 2^-24, or to bf16 (2^-8) in place of the latter; below the least normal number values
are spaced evenly, by 2^-149 (bf16 2^-133).
"""
import math

import pytest
import torch

from tests.test_gpu_dense import DEV, HALF, T, _gpu, ops, rand  # noqa: F401

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


def check(ops, grads, most, eps=0.0, out=None):  # noqa: F811
    before = [g.clone() for g in grads]
    got = ops.clip_gradients(grads, most, eps, out)
    norm = math.sqrt(sum(g.double().square().sum().item() for g in before))
    if norm < 2.0 ** 127:
        assert abs(got.item() - norm) <= 1.01 * U * norm
    else:
        assert got.item() > 2.0 ** 126          # infinity where fp32 has no such number
    most = torch.tensor(most).double().item()    # as the call takes it
    for a, b in zip(before, grads if out is None else out):
        want = a.double() * min(1.0, most / (norm + eps))
        half, least = (HALF, 2.0 ** -133) if b.dtype == torch.bfloat16 else (U, 2.0 ** -149)
        assert torch.all((b.double() - want).abs() <= (half + 2 * U) * want.abs() + least)


@pytest.mark.parametrize("n", [600, 300000])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_norms_that_fp32_does_not_hold(ops, n, dtype):  # noqa: F811
    """One workgroup's and two passes' way; factors down to 1e-79."""
    for size, most in ((1e37, 1.0), (1e38, 1e-5), (3e38, 1e-3), (1e38, 1e37), (1e38, 1e-38), (1e10, 1e-30), (1e-3, 1e-37)):
        x = (rand(1, n).clamp(-1, 1) * size).to(T[dtype])
        y = (rand(2, 77).clamp(-1, 1) * size).to(T[dtype])
        check(ops, [x.clone(), y.clone()], most)
        check(ops, [x, y], most, out=[torch.empty_like(x), torch.empty_like(y, dtype=T["f32"])])


@pytest.mark.parametrize("n", [600, 300000])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_no_largest_norm(ops, n, dtype):  # noqa: F811
    """The norm alone, and copies, whatever the norm."""
    for value in (1.0, math.inf, -math.inf, math.nan):
        x = rand(1, n, dtype=dtype)
        x[n // 2] = value
        y = rand(2, 100)
        before = x.clone(), y.clone()
        out = [torch.zeros_like(x), torch.zeros_like(y)]
        for norm in (ops.clip_gradients([x, y], math.inf, out=out), ops.clip_gradients([x, y], math.inf)):
            assert torch.isnan(norm) if math.isnan(value) else norm.item() == math.inf if math.isinf(value) else norm.item() > 1
        for got in (out, (x, y)):
            for a, b in zip(got, before):
                assert torch.equal(torch.nan_to_num(a, nan=7.0, posinf=8.0, neginf=9.0),
                                   torch.nan_to_num(b, nan=7.0, posinf=8.0, neginf=9.0))
