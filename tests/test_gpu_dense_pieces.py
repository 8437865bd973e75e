"""Dense operators on inputs that are taken in several pieces: of rows, of
classes, and of matrices of a batch.  References and tolerances are those of
test_gpu_dense.py unless a test derives its own."""
import pytest
import torch

from tests.gpu_util import REL_F32
from tests.test_gpu_dense import _gpu, check, check_loss, labels, loss_ref, ops, rand  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_bias_gradient_of_many_pieces_of_rows(ops, dtype):  # noqa: F811
    """More pieces of rows (of 65 536) than are held apart: 66 of them."""
    N, C, K = 65 * 65536 + 777, 4, 129
    x, w, t, bias = rand(1, N, C, dtype=dtype), rand(2, K, C, dtype=dtype) * 0.3, labels(3, N, K), rand(4, K)
    loss, none, none2, gb = ops.linear_cross_entropy(x, w, t, bias, want_grad=True, want_input=False, want_weight=False)
    assert none is None and none2 is None
    ref = loss_ref(x, w, t, bias, True)
    check(loss, *ref["loss"], REL_F32, "loss")
    check(gb, *ref["grad_bias"], REL_F32, "grad_bias")
    assert torch.equal(ops.linear_cross_entropy(x, w, t, bias, want_grad=True)[3], gb)
