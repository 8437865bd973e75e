"""Attention of values that are not numbers: a row that sees a score that is none gets
none, however its keys are shared out among wavefronts and parts; a row without keys, or
with scores of -inf alone, gets zeros and an lse of -inf.

No tolerance: what is compared is where NaN lies, and zeros.
"""
import math

import pytest
import torch

from tests.test_gpu_attention import starts_of
from tests.test_gpu_dense import DEV, T, _gpu, ops, rand  # noqa: F401

pytestmark = pytest.mark.gpu

NAN = float("nan")


def all_nan(x):
    return torch.isnan(x).all()


# rows, keys, heads, key heads, channels: one tile of few rows, tiles of many rows, both cut
# into parts, channels that go to LDS straight and through registers, and (fp32) planes
SIZES = [(1, 33, 8, 8, 64), (1, 65, 4, 1, 64), (1, 77, 8, 8, 64), (3, 77, 4, 2, 36), (1, 77, 2, 2, 128), (1, 9000, 8, 2, 64),
         (2, 9000, 4, 1, 100), (100, 77, 4, 2, 64), (130, 9000, 2, 1, 64), (130, 9000, 2, 1, 128), (2500, 2500, 4, 4, 32),
         (2500, 2500, 2, 2, 64)]
IDS = ["x".join(map(str, s)) for s in SIZES]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,keys,heads,kv_heads,C", SIZES, ids=IDS)
def test_a_query(ops, rows, keys, heads, kv_heads, C, dtype):  # noqa: F811
    q, k, v, g = rand(1, rows, heads, C, dtype=dtype), rand(2, keys, kv_heads, C, dtype=dtype), \
        rand(3, keys, kv_heads, C, dtype=dtype), rand(4, rows, heads, C, dtype=dtype)
    q[rows // 2, heads - 1, C // 2] = NAN
    for causal in (False, True):
        out, lse = ops.attention(q, k, v, causal=causal, want_lse=True)
        bad = torch.zeros(rows, heads, dtype=torch.bool, device=DEV)
        bad[rows // 2, heads - 1] = not causal or rows // 2 + keys - rows >= 0
        assert torch.equal(torch.isnan(lse), bad.t())
        assert torch.equal(torch.isnan(out).all(2), bad) and torch.equal(torch.isnan(out).any(2), bad)
        gq, gk, _ = ops.attention_backward(g, q, k, v, out, lse, causal=causal)
        assert torch.equal(torch.isnan(gq).all(2), bad) and torch.isnan(gk).any() == bad.any()


def places(keys):
    """Keys that are NaN: the newest one, the first, and whole blocks of 32 or 64."""
    return {"newest": (keys - 1, keys), "first": (0, 1), "second block": (32, min(64, keys)),
            "blocks": (keys // 2 // 64 * 64, min(keys, keys // 2 // 64 * 64 + 64)), "all": (0, keys)}


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,keys,heads,kv_heads,C", SIZES, ids=IDS)
def test_keys(ops, rows, keys, heads, kv_heads, C, dtype):  # noqa: F811
    q, clean, v = rand(1, rows, heads, C, dtype=dtype), rand(2, keys, kv_heads, C, dtype=dtype), \
        rand(3, keys, kv_heads, C, dtype=dtype)
    group = heads // kv_heads
    for what, (a, b) in places(keys).items():
        k = clean.clone()
        k[a:b, kv_heads - 1, 1] = NAN
        for causal in (False, True):
            out, lse = ops.attention(q, k, v, causal=causal, want_lse=True)
            # rows that see one of them; those that a mask keeps from all may get them too
            sees = torch.arange(rows, device=DEV) + keys - rows >= (a if causal else -keys)
            mine = slice(heads - group, heads)
            assert all_nan(out[sees, mine]) and all_nan(lse[mine][:, sees]), (what, causal)
            rest = slice(0, heads - group)
            none = torch.arange(rows, device=DEV) + keys - rows < (0 if causal else -keys)
            assert torch.isfinite(out[:, rest]).all() and torch.isfinite(lse[rest][:, ~none]).all(), (what, causal)
            assert torch.all(out[none] == 0) and torch.all(lse[:, none] == -math.inf), (what, causal)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_caches_whose_newest_key_is_none(ops, dtype):  # noqa: F811
    """A token of each of 40 sequences, of which every other one's newest key is NaN."""
    cap, C = 70, 64
    lengths = torch.arange(1, 41, dtype=torch.int32, device=DEV) + 29
    q, k, v = rand(1, 40, 4, C, dtype=dtype), rand(2, 40, cap, 2, C, dtype=dtype), rand(3, 40, cap, 2, C, dtype=dtype)
    bad = torch.arange(40, device=DEV) % 2 == 1
    k[bad, lengths[bad].long() - 1] = NAN
    out, lse = ops.attention(q, k.view(-1, 2, C), v.view(-1, 2, C), starts_of(*[1] * 40), starts_of(*[cap] * 40), lengths,
                             causal=True, want_lse=True)
    assert all_nan(out[bad]) and all_nan(lse[:, bad])
    assert torch.isfinite(out[~bad]).all() and torch.isfinite(lse[:, ~bad]).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,keys,heads,kv_heads,C", SIZES, ids=IDS)
def test_a_value(ops, rows, keys, heads, kv_heads, C, dtype):  # noqa: F811
    """A channel of one value: that channel of all rows, no other one, and no lse."""
    q, k, v = rand(1, rows, heads, C, dtype=dtype), rand(2, keys, kv_heads, C, dtype=dtype), \
        rand(3, keys, kv_heads, C, dtype=dtype)
    v[keys // 2, 0, 5] = NAN
    out, lse = ops.attention(q, k, v, want_lse=True)
    bad = torch.zeros_like(out, dtype=torch.bool)
    bad[:, :heads // kv_heads, 5] = True
    assert torch.equal(torch.isnan(out), bad) and torch.isfinite(lse).all()


@pytest.mark.parametrize("C", [32, 64])
def test_planes_of_values_too_large_for_them(ops, C):  # noqa: F811
    """A query of 2^127 and more, where fp32 products go by three bf16."""
    q, k, v = (rand(i, 2500, 4, C) for i in range(3))
    q[7, 2, 3] = 3.4e38
    out, lse = ops.attention(q, k, v, want_lse=True)
    assert all_nan(out[7, 2]) and torch.isnan(lse[2, 7]) and torch.isnan(out).sum() == C


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,keys", [(1, 77), (1, 9000), (130, 200), (130, 9000)])
def test_scores_of_minus_infinity_alone(ops, rows, keys, dtype):  # noqa: F811
    """Zeros; NaN where fp32 products go by three bf16, which hold no infinity."""
    q, k, v = torch.ones(rows, 2, 64, device=DEV).to(T[dtype]), rand(2, keys, 2, 64, dtype=dtype), \
        rand(3, keys, 2, 64, dtype=dtype)
    k[:, 1, 9] = -math.inf
    out, lse = ops.attention(q, k, v, want_lse=True)
    if dtype == "f32" and rows * keys > 1e6:
        assert all_nan(out[:, 1]) and all_nan(lse[1])
    else:
        assert torch.all(out[:, 1] == 0) and torch.all(lse[1] == -math.inf)
    assert torch.isfinite(out[:, 0]).all() and torch.isfinite(lse[0]).all()
