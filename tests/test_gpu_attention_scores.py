"""Attention of finite scores of any size: products, sums and scale of the values here are
exact (powers of two and small whole numbers), so that which keys count is too.

Tolerances, u = 2^-24: n equal scores' exponentials are the same number, and the mean of their
values is off by (2 n + 16) u of that of |v| (sums of n exponentials and products, a
division, the join of parts), for bf16 by 2^-8 for the probabilities and 2^-8 for the stored
result more.  lse = the score + log n by (n + 16) u + 4 u of itself.
"""
import math

import pytest
import torch

from tests.test_gpu_attention import U, attention_ref, within
from tests.test_gpu_dense import DEV, HALF, T, _gpu, ops, rand  # noqa: F401

pytestmark = pytest.mark.gpu

# one tile of few rows, cut or not, tiles of many rows, cut or not, 64 columns a wavefront, planes
SIZES = [(1, 77, 8, 2, 64), (2, 9000, 4, 1, 64), (1, 500, 2, 2, 100), (100, 77, 4, 2, 64), (130, 9000, 2, 1, 64), (130, 9000, 1, 1, 128),
         (2500, 2500, 4, 4, 32), (2500, 2500, 2, 2, 64), (20000, 64, 8, 1, 32)]
IDS = ["x".join(map(str, s)) for s in SIZES]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,keys,heads,kv_heads,C", SIZES, ids=IDS)
def test_scores_of_any_size(ops, rows, keys, heads, kv_heads, C, dtype):  # noqa: F811
    """Channel 0 alone makes the scores: those of all keys the same, two keys in five the
    largest ones, or ones that grow along the keys; of 2 to 2^110, of either sign."""
    v = rand(1, keys, kv_heads, C, dtype=dtype)
    j = torch.arange(keys, device=DEV)
    most = 0.0
    for what, key in (("equal", 1.0 + 0 * j), ("some", 1.0 + (j % 5 < 2)), ("growing", 1.0 + j // 64 % 128)):
        for bits in (1, 10, 20, 24, 31, 40, 60, 110):
            for sign in (1, -1):
                q, k = torch.zeros(rows, heads, C, device=DEV), torch.zeros(keys, kv_heads, C, device=DEV)
                q[..., 0] = sign * 2.0 ** (bits // 2)
                k[..., 0] = key[:, None] * 2.0 ** (bits - bits // 2)
                s = sign * key.double() * 2.0 ** bits * 0.125
                out, lse = ops.attention(q.to(T[dtype]), k.to(T[dtype]), v, scale=0.125, want_lse=True)
                p = torch.softmax(s, 0)
                want = (p[:, None, None] * v.double()).sum(0).repeat_interleave(heads // kv_heads, 0)
                size = (p[:, None, None] * v.double().abs()).sum(0).repeat_interleave(heads // kv_heads, 0)
                half = HALF if dtype == "bf16" else 0.0
                # what differs from the largest score does so by 1/4 or more; its argument's rounding
                e = (2 * keys + 16) * U + (16 * U if bits == 1 else 0.0)
                within(out, want.expand_as(out), ((e + half) * size + half * want.abs()).expand_as(out), f"{what} {bits} {sign}")
                l = torch.logsumexp(s, 0).item()
                most = max(most, (lse.double() - l).abs().max().item() / ((keys + 16) * U + 4 * U * abs(l)))
    assert most <= 1.0, most


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_row_of_large_scores_changes_no_other(ops, dtype):  # noqa: F811
    """The other rows of its tile are as near to 64 bits as without it (tolerance as in
    test_gpu_attention; their maxima may move at other keys, so the last bits differ)."""
    q, k, v = rand(1, 300, 2, 64, dtype=dtype), rand(2, 400, 2, 64, dtype=dtype), rand(3, 400, 2, 64, dtype=dtype)
    ref, e = attention_ref(q, k, v, [(0, 300, 0, 400)], False, 0.125)[0]
    q[77, 1] *= 2.0 ** 60
    got = ops.attention(q, k, v)
    best = (q[77, 1].double() @ k[:, 1].double().t()).argmax()
    assert torch.equal(got[77, 1], v[best, 1])
    got[77, 1] = ref[77, 1].to(T[dtype])
    within(got, ref, e, "out")


def test_largest_scale(ops):  # noqa: F811
    q, k, v = rand(1, 5, 2, 32), rand(2, 90, 2, 32), rand(3, 90, 2, 32)
    out = ops.attention(q, k, v, scale=1e30)
    s = torch.einsum("ihc,jhc->hij", q.double().cpu(), k.double().cpu())
    best = s.argmax(2).to(DEV)
    # the largest two scores differ by more than fp32 sums are off by
    top = s.topk(2, 2).values
    assert ((top[..., 0] - top[..., 1]) > 1e-4).all()
    for h in range(2):
        assert torch.equal(out[:, h], v[best[h], h])
