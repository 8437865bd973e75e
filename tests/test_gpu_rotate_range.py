"""Rotation of normalised heads whose squares fp32 does not hold, and of gradients whose
products with them it does not.

Tolerances as in test_gpu_rotate: the values are scaled by powers of two, which round
nothing.  With sizes x of the heads and g of the gradients, results are of size 1,
gradients of x of size g / x and those of gains of size g; all are divided by these
before they are compared.  Below 2^-126 a type's values are no longer spaced by their size:
bf16 ones are 2^-133 apart there, fp32 ones 2^-149, and a stored gradient is off by half of that
more (2^-134 of bf16 gradients of 1e-37 is 4.6e-4 of their size, where 2^-8 of one of 4.5e-40
is 1.8e-5).
"""
import pytest
import torch

from tests.test_gpu_attention import within
from tests.test_gpu_dense import DEV, T, _gpu, ops, rand  # noqa: F401
from tests.test_gpu_rotate import frequencies, rotate_ref

pytestmark = pytest.mark.gpu

# heads, gradients, eps
RANGE = [(1e25, 1e25, 1e-6), (3e37, 3e30, 1e-6), (1e19, 1.0, 0.0), (1e-25, 1e-25, 0.0), (1e-37, 1e-30, 0.0), (1e-20, 1e-20, 1e-38),
         (1e-15, 1e-30, 0.0), (1e15, 1e30, 1e-6), (1.0, 1e37, 1e-6), (1.0, 1e-37, 1e-6)]


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("C,sections", [(3, [1]), (16, [8]), (36, [4, 4, 4, 4]), (128, [16, 24, 24]), (128, [64]), (256, [100, 20])])
def test_sizes(ops, C, sections, dtype, interleaved):  # noqa: F811
    for size, of_grad, eps in RANGE:
        q, k = (rand(1, 37, 4, C) * size).to(T[dtype]), (rand(2, 37, 2, C) * size).to(T[dtype])
        gq, gk = (rand(3, 37, 4, C) * of_grad).to(T[dtype]), (rand(4, 37, 2, C) * of_grad).to(T[dtype])
        pos, gains = 30 * rand(5, 37, len(sections)), (1 + 0.3 * rand(6, C), 1 + 0.3 * rand(7, C))
        args, kw = (q, k, pos, frequencies(sum(sections)), sections, *gains), dict(eps=eps, interleaved=interleaved)
        got = ops.rotate_heads(*args, **kw)
        back = ops.rotate_heads_backward(gq, gk, *args, **kw)
        for x, y, g, gx, gg, gain in ((q, got[0], gq, back[0], back[2], gains[0]), (k, got[1], gk, back[1], back[3], gains[1])):
            what = f"{size}, {of_grad}"
            # (eps as the call takes it, in fp32)
            ref = (x, pos, frequencies(sum(sections)), sections, gain, True, torch.tensor(eps).double().item(), interleaved)
            within(y, *rotate_ref(*ref), "out of " + what)
            (r, e), (rg, eg) = rotate_ref(*ref, g)
            f = size / of_grad
            least = 2.0 ** (-134 if dtype == "bf16" else -150)
            within(gx.double() * f, r * f, (e + least) * f, "grad of " + what)
            over = rg.abs() >= 2.0 ** 128            # sums that fp32 has no number for
            assert torch.equal(gg[over].double(), rg[over] * float("inf"))
            gg, rg = torch.where(over, 0.0, gg.double()), torch.where(over, 0.0, rg)
            within(gg / of_grad, rg / of_grad, eg / of_grad, "grad_gain of " + what)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_one_large_head_among_others(ops, dtype):  # noqa: F811
    """And rows of zeros without eps, of infinity and of NaN: each is its own."""
    q = rand(1, 50, 8, 64, dtype=dtype)
    f, pos = frequencies(32), rand(2, 50, 1)
    want = ops.rotate_heads(q, None, pos, f, eps=0.0)[0]
    bad = q.clone()
    bad[3, 1] *= 1e30
    bad[4, 2] *= 1e-30
    bad[5, 3] = 0.0
    bad[6, 4, 7] = float("inf")
    bad[7, 5, 7] = float("nan")
    got = ops.rotate_heads(bad, None, pos, f, eps=0.0)[0]
    same = torch.ones(50, 8, dtype=torch.bool, device=DEV)
    for i in range(5):
        same[3 + i, 1 + i] = False
    assert torch.equal(got[same], want[same])
    for row, head in ((3, 1), (4, 2)):
        within(got[row:row + 1, head:head + 1], *rotate_ref(bad[row:row + 1, head:head + 1], pos[row:row + 1], f, [32], None, True,
                                                            0.0, False), "out")
    assert torch.isnan(got[5, 3]).all() and torch.isnan(got[7, 5]).all() and torch.isnan(got[6, 4, [7, 39]]).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("C,P", [(3, 1), (16, 8), (36, 18), (72, 33), (128, 64), (256, 128), (250, 3)])
def test_some_heads_of_a_wavefront(ops, C, P, dtype):  # noqa: F811
    """Every third head large, every third small: groups of a wavefront that go different ways,
    forward and backward, each head as it is alone."""
    q, g = rand(1, 40, 6, C, dtype=dtype), rand(2, 40, 6, C, dtype=dtype)
    for i, f in ((0, 2.0 ** 70), (1, 2.0 ** -70)):
        q[:, i::3] *= f
        g[:, i::3] *= f
    q[::5], g[::7] = rand(3, 8, 6, C, dtype=dtype), 0
    args = (rand(4, 40, 1), frequencies(P), [P], 1 + 0.2 * rand(5, C))
    y, _ = ops.rotate_heads(q, None, *args, eps=0.0)
    gx = ops.rotate_heads_backward(g, None, q, None, *args, eps=0.0)[0]
    for h in range(6):
        one = ops.rotate_heads(q[:, h:h + 1], None, *args, eps=0.0)[0]
        back = ops.rotate_heads_backward(g[:, h:h + 1], None, q[:, h:h + 1], None, *args, eps=0.0)[0]
        assert torch.equal(y[:, h:h + 1], one) and torch.equal(gx[:, h:h + 1], back)
        for row in (0, 1, 11):                   # and alone in its launch
            at = slice(row, row + 1)
            alone = (args[0][at], *args[1:])
            assert torch.equal(ops.rotate_heads(q[at, h:h + 1], None, *alone, eps=0.0)[0], one[at])
            assert torch.equal(ops.rotate_heads_backward(g[at, h:h + 1], None, q[at, h:h + 1], None, *alone, eps=0.0)[0], back[at])
    ref = rotate_ref(q, args[0], args[1], [P], args[3], True, 0.0, False)
    within(y, *ref, "out")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_gradients_of_zero(ops, dtype):  # noqa: F811
    q = rand(1, 300, 4, 48, dtype=dtype)
    g = rand(2, 300, 4, 48, dtype=dtype)
    g[::2] = 0
    args = (rand(3, 300, 2), frequencies(20), [10, 10], 1 + 0.1 * rand(4, 48))
    gx, _, gg, _ = ops.rotate_heads_backward(g, None, q, None, *args)
    odd, _, _, _ = ops.rotate_heads_backward(g[1::2], None, q[1::2], None, args[0][1::2], *args[1:])
    assert torch.all(gx[::2] == 0) and torch.equal(gx[1::2], odd) and torch.isfinite(gg).all()
