"""Rotation of as many rows as there may be: more than a launch has workgroups for, one
each.  Tolerances as in test_gpu_rotate."""
import pytest
import torch

from tests.test_gpu_attention import within
from tests.test_gpu_dense import DEV, T, _gpu, ops, rand  # noqa: F401
from tests.test_gpu_rotate import frequencies, rotate_ref

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,rows,C", [("bf16", 1 << 30, 2), ("f32", (1 << 28) + 5, 4), ("bf16", (1 << 27) + 7, 36)])
def test_very_many_rows(ops, dtype, rows, C):  # noqa: F811
    some = rand(1, 1 << 20, 1, C, dtype=dtype)
    q = some.repeat((rows + (1 << 20) - 1) // (1 << 20), 1, 1)[:rows]
    pos = torch.arange(rows, dtype=torch.int32, device=DEV) % 1000
    at = torch.cat([torch.arange(1000, device=DEV), rows - 1 - torch.arange(1000, device=DEV),
                    torch.randint(rows, (20000,), device=DEV, generator=torch.Generator(device=DEV).manual_seed(2))])
    before, f = q[at], frequencies(C // 2)
    assert ops.rotate_heads(q, None, pos, f, out_q=q)[0] is q
    within(q[at], *rotate_ref(before, pos[at][:, None], f, [C // 2], None, True, 1e-6, False), "out")
    whole = q[:1 << 20]
    for i in range(1, rows >> 20):          # rows whose positions are the same, a period of 125 further
        if i % 125 == 0:
            assert torch.equal(q[i << 20:(i + 1) << 20], whole), i
