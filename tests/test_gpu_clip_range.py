"""Clipping without a largest norm.  What is compared is exact."""
import math

import pytest
import torch

from tests.test_gpu_dense import _gpu, ops, rand  # noqa: F401

pytestmark = pytest.mark.gpu


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
