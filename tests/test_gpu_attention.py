"""Attention over packed sequences, forward and backward, against a plain 64-bit
implementation.

Tolerances, fixed from the arithmetic, u = 2^-24 being half a step of fp32.  With
A the largest sum of |scale q_c k_c| of a row, n the longest chain of additions and
C the channels:
  * a score is off by (C + 4) u A, its exponential by that, 3 A u of the argument's
    rounding and 4 u of its own; a probability, with the sum of n of them, by
    twice that and n u:                     e_p = u (2 (C + 8) A + 2 n + 16)
  * out, relative to sum p |v|: e_p and n u; for bf16 the probability's rounding,
    2^-8, and that of the stored result, 2^-8 of itself.
  * lse: u ((C + 8) A + n + 8 + 2 |lse|); probabilities made from it e_p + 2 u |lse|.
  * t = p (g.v - g.out) is off by p times ((e_p + (C + 4) u) (|g|.|v| + |g|.|out|)
    + |g| times what out is off by); for bf16 by 2^-8 of itself more.
  * sums over t and p by n u more, stored bf16 results by 2^-8 of themselves.
"""
import math

import pytest
import torch

from tests.test_gpu_dense import DEV, HALF, T, _gpu, ops, rand  # noqa: F401

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


def within(got, ref, bound, what):
    got, ref = got.double(), ref.double()
    assert got.shape == ref.shape, (what, got.shape, ref.shape)
    assert torch.isfinite(got).all() or not torch.isfinite(ref).all(), f"{what}: not finite"
    err = (got - ref).abs()
    worst = (err / (bound + 1e-30)).max().item() if err.numel() else 0.0
    assert worst <= 1.0, f"{what}: error {worst:.3g} times the tolerance (largest {err.max().item():.3g})"


def attention_ref(q, k, v, sequences, causal, scale, g=None):
    """sequences: (q0, rows, k0, keys) of each.  [(value, tolerance)] of out, lse and,
    given g, grad_q, grad_k, grad_v; rows of no sequence 0 and -inf."""
    half = HALF if q.dtype == torch.bfloat16 else 0.0
    q, k, v = q.double(), k.double(), v.double()
    heads, kv_heads, C = q.shape[1], k.shape[1], q.shape[2]
    zeros = torch.zeros_like
    out, out_e, lse = zeros(q), zeros(q), torch.full((heads, q.shape[0]), -math.inf, device=q.device).double()
    lse_e = zeros(lse)
    gq, gq_e, gk, gk_e, gv, gv_e = zeros(q), zeros(q), zeros(k), zeros(k), zeros(v), zeros(v)
    for q0, n, k0, m in sequences:
        if n == 0 or m == 0:
            continue
        for h in range(heads):
            kh = h // (heads // kv_heads)
            Q, K, V = q[q0:q0 + n, h], k[k0:k0 + m, kh], v[k0:k0 + m, kh]
            s = Q @ K.t() * scale
            A = (Q.abs() @ K.abs().t() * scale).amax(1, keepdim=True)
            if causal:
                i, j = torch.arange(n, device=q.device)[:, None], torch.arange(m, device=q.device)[None]
                s = torch.where(j <= i + m - n, s, -math.inf)
            l = torch.logsumexp(s, 1, keepdim=True)
            p = torch.where(l == -math.inf, 0.0, torch.exp(s - torch.where(l == -math.inf, 0.0, l)))
            o = p @ V
            e_p = U * (2 * (C + 8) * A + 2 * m + 16)
            o_e = (e_p + U * m + half) * (p @ V.abs()) + half * o.abs()
            sl = slice(q0, q0 + n)
            out[sl, h], out_e[sl, h], lse[h, sl] = o, o_e, l[:, 0]
            size = torch.where(l == -math.inf, 0.0, l.abs())
            lse_e[h, sl] = (U * ((C + 8) * A + m + 8 + 2 * size))[:, 0]
            if g is None:
                continue
            G = g[sl, h].double()
            e_p = e_p + 2 * U * size
            gv[k0:k0 + m, kh] += p.t() @ G
            gv_e[k0:k0 + m, kh] += (p * (e_p + U * n * heads + half)).t() @ G.abs()
            dp, delta = G @ V.t(), (G * o).sum(1, keepdim=True)
            t = p * (dp - delta)
            mag = G.abs() @ V.abs().t() + (G.abs() * o.abs()).sum(1, keepdim=True)
            t_e = p * ((e_p + (C + 4) * U) * mag + (G.abs() * o_e).sum(1, keepdim=True)) + half * t.abs()
            gq[sl, h] = t @ K * scale
            gq_e[sl, h] = (t_e + U * m * t.abs()) @ K.abs() * scale
            gk[k0:k0 + m, kh] += t.t() @ Q * scale
            gk_e[k0:k0 + m, kh] += (t_e + U * n * heads * t.abs()).t() @ Q.abs() * scale
    res = [(out, out_e), (lse, lse_e)]
    if g is not None:
        res += [(x, e + half * x.abs()) for x, e in ((gq, gq_e), (gk, gk_e), (gv, gv_e))]
    return res


def starts_of(*lengths, first=0):
    s = [first]
    for n in lengths:
        s.append(s[-1] + n)
    return torch.tensor(s, dtype=torch.int32, device=DEV)


def check_all(ops, q, k, v, sequences, causal, scale=None, g=None, **packing):  # noqa: F811
    ref = attention_ref(q, k, v, sequences, causal, scale or 1 / math.sqrt(q.shape[2]), g)
    out, lse = ops.attention(q, k, v, causal=causal, scale=scale, want_lse=True, **packing)
    within(out, *ref[0], "out")
    none = ref[1][0] == -math.inf
    assert torch.equal(lse == -math.inf, none)
    within(torch.where(none, 0.0, lse), torch.where(none, 0.0, ref[1][0]), ref[1][1], "lse")
    if g is not None:
        got = ops.attention_backward(g, q, k, v, out, lse, causal=causal, scale=scale, **packing)
        for x, (r, e), name in zip(got, ref[2:], ("grad_q", "grad_k", "grad_v")):
            within(x, r, e, name)
    return out, lse


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("C", [1, 7, 20, 32, 36, 64, 72, 100, 128])
def test_one_sequence(ops, C, dtype, causal):  # noqa: F811
    q, k, v, g = rand(1, 131, 2, C, dtype=dtype), rand(2, 131, 1, C, dtype=dtype), rand(3, 131, 1, C, dtype=dtype), \
        rand(4, 131, 2, C, dtype=dtype)
    check_all(ops, q, k, v, [(0, 131, 0, 131)], causal, g=g)


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,keys", [(1, 1), (1, 2), (2, 1), (1, 33), (31, 32), (64, 64), (65, 63), (128, 129), (300, 7),
                                       (3, 700), (257, 511), (1, 3000)])
def test_lengths(ops, rows, keys, dtype, causal):  # noqa: F811
    """Fewer and more keys than rows: causal rows without a key among them."""
    q, k, v, g = rand(1, rows, 4, 64, dtype=dtype), rand(2, keys, 2, 64, dtype=dtype), rand(3, keys, 2, 64, dtype=dtype), \
        rand(4, rows, 4, 64, dtype=dtype)
    check_all(ops, q, k, v, [(0, rows, 0, keys)], causal, g=g)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("heads,kv_heads", [(1, 1), (3, 3), (6, 2), (5, 1), (8, 8), (16, 2), (40, 1), (140, 1), (24, 8)])
def test_head_layouts(ops, heads, kv_heads, dtype):  # noqa: F811
    q, k, v, g = rand(1, 90, heads, 32, dtype=dtype), rand(2, 90, kv_heads, 32, dtype=dtype), \
        rand(3, 90, kv_heads, 32, dtype=dtype), rand(4, 90, heads, 32, dtype=dtype)
    s = starts_of(50, 1, 39)
    check_all(ops, q, k, v, [(0, 50, 0, 50), (50, 1, 50, 1), (51, 39, 51, 39)], True, g=g, q_starts=s)


PACKS = [(1,), (1, 1, 1), (5, 0, 7), (0, 0, 0), (64, 64, 64), (1, 200, 3, 0, 129, 1), (33,) * 9, tuple(range(1, 80)), (300, 2, 256)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,heads,kv_heads,keys", [(2, 65536, 1, 70), (1, 65536, 1, 3000), (3, 4096, 64, 40)])
def test_very_many_heads(ops, rows, heads, kv_heads, keys, dtype):  # noqa: F811
    """The query heads of a key head are as many rows of one head."""
    C, group = 16, heads // kv_heads
    q, g = rand(1, rows, heads, C, dtype=dtype), rand(4, rows, heads, C, dtype=dtype)
    k, v = rand(2, keys, kv_heads, C, dtype=dtype), rand(3, keys, kv_heads, C, dtype=dtype)

    def as_rows(x):
        return x.view(rows, kv_heads, group, -1).transpose(1, 2).reshape(rows * group, kv_heads, -1)

    ref = attention_ref(as_rows(q), k, v, [(0, rows * group, 0, keys)], False, 0.25, as_rows(g))
    out, lse = ops.attention(q, k, v, want_lse=True)
    grads = ops.attention_backward(g, q, k, v, out, lse)
    within(as_rows(out), *ref[0], "out")
    within(as_rows(lse.t().contiguous())[..., 0].t(), *ref[1], "lse")
    for x, (r, e), name in zip((as_rows(grads[0]), *grads[1:]), ref[2:], ("grad_q", "grad_k", "grad_v")):
        within(x, r, e, name)


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("lengths", PACKS, ids=[str(len(p)) + "x" + str(max(p)) for p in PACKS])
def test_packed(ops, lengths, dtype, causal):  # noqa: F811
    n = sum(lengths)
    qkv = rand(1, n, 8, 40, dtype=dtype)
    q, k, v = qkv[:, :4], qkv[:, 4:6], qkv[:, 6:]
    s = starts_of(*lengths)
    at = s.tolist()
    check_all(ops, q, k, v, [(a, m, a, m) for a, m in zip(at, lengths)], causal, g=rand(2, n, 4, 40, dtype=dtype), q_starts=s)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("C", [64, 100, 128])
@pytest.mark.parametrize("new", [1, 2, 5])
def test_against_a_cache(ops, new, C, dtype):  # noqa: F811
    """New rows of each sequence against a cache that each fills in part; the rest
    of it holds NaN."""
    cap, lengths = 700, [700, 0, 1, 33, 64, 65, 699, 3, 512]
    n = len(lengths)
    q = rand(1, n * new, 8, C, dtype=dtype)
    k, v = rand(2, n, cap, 2, C, dtype=dtype), rand(3, n, cap, 2, C, dtype=dtype)
    clean = k.clone(), v.clone()
    for b, m in enumerate(lengths):
        k[b, m:] = float("nan")
        v[b, m:] = float("nan")
    seqs = [(b * new, new, b * cap, m) for b, m in enumerate(lengths)]
    packing = dict(q_starts=starts_of(*[new] * n), kv_starts=starts_of(*[cap] * n),
                   kv_lengths=torch.tensor(lengths, dtype=torch.int32, device=DEV))
    flat = [x.view(n * cap, 2, C) for x in (k, v, *clean)]
    for causal in (True, False):
        g = rand(4, n * new, 8, C, dtype=dtype)
        ref = attention_ref(q, flat[2], flat[3], seqs, causal, 1 / math.sqrt(C), g)
        out, lse = ops.attention(q, flat[0], flat[1], causal=causal, want_lse=True, **packing)
        within(out, *ref[0], "out")
        got = ops.attention_backward(g, q, flat[0], flat[1], out, lse, causal=causal, **packing)
        for x, (r, e), name in zip(got, ref[2:], ("grad_q", "grad_k", "grad_v")):
            within(x, r, e, name)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_far_keys_are_split(ops, dtype):  # noqa: F811
    """Few rows of long sequences: keys shared out among workgroups, and joined."""
    q, k, v = rand(1, 3, 4, 64, dtype=dtype), rand(2, 9000, 1, 64, dtype=dtype), rand(3, 9000, 1, 64, dtype=dtype)
    check_all(ops, q, k, v, [(0, 3, 0, 9000)], True, g=rand(4, 3, 4, 64, dtype=dtype))
    q, g = rand(1, 200, 2, 64, dtype=dtype), rand(4, 200, 2, 64, dtype=dtype)
    check_all(ops, q, k, v, [(0, 100, 0, 8000), (100, 100, 8000, 1000)], False, g=g, q_starts=starts_of(100, 100),
              kv_starts=starts_of(8000, 1000))


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("C,heads,kv_heads,lengths", [(20, 8, 2, (2000, 1, 0, 1400)), (32, 4, 4, (2500,)), (36, 6, 1, (1900, 33)),
                                                      (64, 3, 3, (1, 2100, 64))])
def test_many_rows(ops, C, heads, kv_heads, lengths, dtype, causal):  # noqa: F811
    """Enough of them for fp32 products to go by planes of bf16, of strided heads."""
    n = sum(lengths)
    qkv = rand(1, n, heads + 2 * kv_heads, C, dtype=dtype)
    q, k, v = qkv[:, :heads], qkv[:, heads:heads + kv_heads], qkv[:, heads + kv_heads:]
    s = starts_of(*lengths)
    at = s.tolist()
    check_all(ops, q, k, v, [(a, m, a, m) for a, m in zip(at, lengths)], causal, g=rand(2, n, heads, C, dtype=dtype),
              q_starts=s)


@pytest.mark.parametrize("size", [1e-12, 1e12])
def test_many_rows_of_small_and_large_values(ops, size):  # noqa: F811
    n = 2500
    q, k, v, g = (rand(i, n, 4, 32) for i in range(4))
    check_all(ops, q * size, k / size, v * size, [(0, n, 0, n)], True, g=g / size)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("C", [36, 64])
def test_strides(ops, C, dtype):  # noqa: F811
    """Heads before rows, an odd first element, repeated heads and repeated keys."""
    n = 150
    s = starts_of(100, 50)
    seqs = [(0, 100, 0, 100), (100, 50, 100, 50)]
    q = rand(1, 4, n, C, dtype=dtype).transpose(0, 1)
    k = rand(2, n * 2 * C + 3, dtype=dtype)[3:].view(n, 2, C)
    v = rand(3, n, 1, C + 5, dtype=dtype)[..., 5:].expand(n, 2, C)
    g = rand(4, 1, 4, C, dtype=dtype).expand(n, 4, C)
    out, _ = check_all(ops, q, k, v, seqs, True, g=g, q_starts=s)
    to = torch.full((4, n, C + 1), 7.0, device=DEV, dtype=T[dtype])
    got = ops.attention(q, k, v, s, causal=True, out=to.transpose(0, 1)[..., :C])
    assert torch.equal(got, out) and torch.all(to[..., C] == 7)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("C,far", [(64, "rows"), (36, "rows"), (64, "heads")])
def test_offsets_past_32_bits(ops, C, far, dtype):  # noqa: F811
    """Rows 8 MB apart, or heads 2.1 GB: the last of them lie 6 to 7 GB behind the first."""
    n, e = 900, 4 if dtype == "f32" else 2
    gap = (1 << 23) // e if far == "rows" else (2100 << 20) // e
    heads, kv_heads = 4, 2 if far == "rows" else 4
    buffer = torch.empty(n * gap if far == "rows" else 3 * gap + (1 << 20), device=DEV, dtype=T[dtype])

    def place(i, h):
        at = buffer[i * (gap // 8 if far == "rows" else 1 << 17):]
        x = at.as_strided((n, h, C), (gap, C, 1) if far == "rows" else (C, gap, 1))
        return x.copy_(rand(i, n, h, C, dtype=dtype))

    q, k, v, g = place(1, heads), place(2, kv_heads), place(3, kv_heads), place(4, heads)
    s, seqs = starts_of(n - 50, 50), [(0, n - 50, 0, n - 50), (n - 50, 50, n - 50, 50)]
    out, lse = check_all(ops, q, k, v, seqs, True, g=g, q_starts=s)
    check_all(ops, q[-1:], k, v, [(0, 1, 0, n)], False, g=g[-1:])
    if far == "rows":
        to = place(5, heads)
        assert torch.equal(ops.attention(q, k, v, s, causal=True, out=to), out)
        near = ops.attention_backward(g, q, k, v, out, lse, s, causal=True)
        for a, b in zip(near, ops.attention_backward(g, q, k, v, to, lse, s, causal=True)):
            assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows", [90, 4000])
def test_rows_of_no_sequence(ops, rows, dtype):  # noqa: F811
    """Left alone in a given out, else zeros; whatever they hold reaches no result."""
    n = rows + 60
    q, k, v, g = rand(1, n, 2, 64, dtype=dtype), rand(2, n, 2, 64, dtype=dtype), rand(3, n, 2, 64, dtype=dtype), \
        rand(4, n, 2, 64, dtype=dtype)
    s = starts_of(rows - 40, 40, first=25)
    seqs = [(25, rows - 40, 25, rows - 40), (rows - 15, 40, rows - 15, 40)]
    inside = torch.zeros(n, dtype=torch.bool, device=DEV)
    inside[25:25 + rows] = True
    clean = out, _ = check_all(ops, q, k, v, seqs, False, g=g, q_starts=s)
    assert torch.all(out[~inside] == 0)
    grads = ops.attention_backward(g, q, k, v, *clean, s)
    for x in (q, k, v, g):
        x[~inside] = float("nan")
    to = torch.full_like(q, 5.0)
    again = ops.attention(q, k, v, s, out=to)
    assert torch.equal(again[inside], out[inside]) and torch.all(again[~inside] == 5)
    got = ops.attention_backward(g, q, k, v, *clean, s)
    for a, b in zip(got, grads):
        assert torch.equal(a, b) and torch.all(a[~inside] == 0)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_very_many_sequences(ops, dtype):  # noqa: F811
    """More starts than a wavefront's lanes, and than those squared."""
    lengths = [i % 4 for i in range(5000)]
    n = sum(lengths)
    s = starts_of(*lengths)
    q, k, v, g = (rand(i, n, 1, 8, dtype=dtype) for i in range(4))
    owner = torch.repeat_interleave(torch.arange(5000, device=DEV), torch.tensor(lengths, device=DEV))
    out, lse = ops.attention(q, k, v, s, want_lse=True)
    got = ops.attention_backward(g, q, k, v, out, lse, s)
    Q, K, V, G = (x[:, 0].double() for x in (q, k, v, g))
    z = torch.where(owner[:, None] == owner, Q @ K.t() / math.sqrt(8), -math.inf)
    p = torch.softmax(z, 1)
    t = p * (G @ V.t() - (G * (p @ V)).sum(1, keepdim=True))
    # scores up to 10, two or three keys: 60 u of the sums of |terms|, and the roundings
    half = 3 * HALF if dtype == "bf16" else 0.0
    mag = p * (G.abs() @ V.abs().t() + (G.abs() * (p @ V.abs())).sum(1, keepdim=True))
    rel = 200 * U + half
    within(out[:, 0], p @ V, rel * (p @ V.abs()), "out")
    within(got[0][:, 0], t @ K / math.sqrt(8), rel * (mag @ K.abs()), "grad_q")
    within(got[1][:, 0], t.t() @ Q / math.sqrt(8), rel * (mag.t() @ Q.abs()), "grad_k")
    within(got[2][:, 0], p.t() @ G, rel * (p.t() @ G.abs()), "grad_v")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("keys", [1, 4])
def test_more_tiles_than_a_launch(ops, keys, dtype):  # noqa: F811
    """140000 sequences of 32 heads, a row and 1 or 4 keys each: 4.5 million tiles, more
    than the 2^22 of a launch.  The tolerances of attention_ref, a sequence along an axis."""
    n, heads, C = 140000, 32, 8
    q, k, v, g = rand(1, n, heads, C, dtype=dtype), rand(2, n * keys, heads, C, dtype=dtype), \
        rand(3, n * keys, heads, C, dtype=dtype), rand(4, n, heads, C, dtype=dtype)
    s = torch.arange(n + 1, device=DEV, dtype=torch.int32)
    out, lse = ops.attention(q, k, v, s, s * keys, want_lse=True)
    got = ops.attention_backward(g, q, k, v, out, lse, s, s * keys)
    half, scale = HALF if dtype == "bf16" else 0.0, 1 / math.sqrt(C)
    Q, G = q.double()[:, None], g.double()[:, None]
    K, V = k.double().view(n, keys, heads, C), v.double().view(n, keys, heads, C)
    z = (Q * K).sum(3, keepdim=True) * scale
    A = (Q * K).abs().sum(3, keepdim=True).amax(1, keepdim=True) * scale
    l = torch.logsumexp(z, 1, keepdim=True)
    p = torch.exp(z - l)
    e_p = U * (2 * (C + 8) * A + 2 * keys + 16)
    o = (p * V).sum(1, keepdim=True)
    o_e = ((e_p + U * keys + half) * p * V.abs()).sum(1, keepdim=True) + half * o.abs()
    within(out, o[:, 0], o_e[:, 0], "out")
    within(lse.t(), l[:, 0, :, 0], (U * ((C + 8) * A + keys + 8 + 2 * l.abs()))[:, 0, :, 0], "lse")
    e_p = e_p + 2 * U * l.abs()
    t = p * ((G * V).sum(3, keepdim=True) - (G * o).sum(3, keepdim=True))
    mag = (G * V).abs().sum(3, keepdim=True) + (G * o).abs().sum(3, keepdim=True)
    t_e = p * ((e_p + (C + 4) * U) * mag + (G.abs() * o_e).sum(3, keepdim=True)) + half * t.abs()
    for x, r, e, name in ((got[0], (t * K).sum(1) * scale, ((t_e + U * keys * t.abs()) * K.abs()).sum(1) * scale, "grad_q"),
                          (got[1], (t * Q * scale).flatten(0, 1), ((t_e + U * heads * t.abs()) * Q.abs() * scale).flatten(0, 1),
                           "grad_k"),
                          (got[2], (p * G).flatten(0, 1), (p * (e_p + U * heads + half) * G.abs()).flatten(0, 1), "grad_v")):
        within(x, r, e + half * r.abs(), name)


def test_no_sequences_and_one_with_a_length(ops):  # noqa: F811
    q, k, v, g = (rand(i, 50, 2, 32) for i in range(4))
    none = torch.zeros(1, dtype=torch.int32, device=DEV)
    out, lse = ops.attention(q, k, v, none, want_lse=True)
    assert torch.all(out == 0) and torch.all(lse == -math.inf)
    assert all(torch.all(x == 0) for x in ops.attention_backward(g, q, k, v, out, lse, none))
    for m in (0, 1, 33, 50):
        check_all(ops, q, k, v, [(0, 50, 0, m)], True, g=g, kv_lengths=torch.tensor([m], dtype=torch.int32, device=DEV))
    empty = rand(5, 0, 2, 32)
    out, lse = ops.attention(q, empty, empty, want_lse=True)
    assert torch.all(out == 0)
    got = ops.attention_backward(g, q, empty, empty, out, lse)
    assert torch.all(got[0] == 0) and got[1].shape == got[2].shape == (0, 2, 32)
    out, lse = ops.attention(empty, k, v, want_lse=True)
    assert out.shape == (0, 2, 32) and lse.shape == (2, 0)
    got = ops.attention_backward(empty, empty, k, v, out, lse)
    assert torch.all(got[1] == 0) and torch.all(got[2] == 0)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_large_scores(ops, dtype):  # noqa: F811
    """Scores of thousands, growing along the keys (the running maximum moves), and
    falling ones."""
    C, n = 64, 200
    for sign in (1, -1):
        k = torch.linspace(1, 4, n, device=DEV)[:, None, None].expand(n, 1, C).contiguous() * sign
        q = torch.full((n, 1, C), 16.0, device=DEV)
        q, k = q.to(T[dtype]), k.to(T[dtype])
        v, g = rand(3, n, 1, C, dtype=dtype), rand(4, n, 1, C, dtype=dtype)
        check_all(ops, q, k, v, [(0, n, 0, n)], True, scale=1.0, g=g)


def test_infinite_scores(ops):  # noqa: F811
    """A key that nothing attends to (-inf) and one that scores +inf (NaN, in that row
    alone)."""
    q, k, v = torch.ones(3, 1, 8, device=DEV), torch.ones(4, 1, 8, device=DEV), rand(1, 4, 1, 8)
    q[1, 0, 0] = -1.0
    k[2, 0, 0] = -math.inf
    out = ops.attention(q, k, v)
    assert torch.isfinite(out[0]).all() and torch.isfinite(out[2]).all() and torch.isnan(out[1]).all()
    want = attention_ref(q[:1], torch.cat([k[:2], k[3:]]), torch.cat([v[:2], v[3:]]), [(0, 1, 0, 3)], False, 8 ** -0.5)[0]
    within(out[:1], *want, "out")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_value_that_is_not_finite_stays_in_its_sequence(ops, dtype):  # noqa: F811
    n = 260
    q, k, v, g = (rand(i, n, 2, 64, dtype=dtype) for i in range(4))
    s = starts_of(70, 90, 100)
    out, lse = ops.attention(q, k, v, s, causal=True, want_lse=True)
    grads = ops.attention_backward(g, q, k, v, out, lse, s, causal=True)
    for x in (k, v, q, g):
        bad = x.clone()
        bad[100, 1, 3] = float("nan")
        args = [bad if x is y else y for y in (q, k, v)]
        o, l = ops.attention(*args, s, causal=True, want_lse=True)
        got = (o, *ops.attention_backward(bad if x is g else g, *args, o, l, s, causal=True))
        for a, b in zip(got, (out, *grads)):
            assert torch.equal(a[:70], b[:70]) and torch.equal(a[160:], b[160:])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_same_bits_twice(ops, dtype):  # noqa: F811
    n = 3000
    q, k, v, g = (rand(i, n, h, 64, dtype=dtype) for i, h in enumerate((4, 1, 1, 4)))
    s = starts_of(1000, 3, 1997)

    def both():
        out, lse = ops.attention(q, k, v, s, causal=True, want_lse=True)
        return [out, lse, *ops.attention_backward(g, q, k, v, out, lse, s, causal=True)]

    first = both()
    for _ in range(3):
        assert all(torch.equal(a, b) for a, b in zip(first, both()))


def test_gradients_against_differences(ops):  # noqa: F811
    """The loss sum(out g) moves as its gradients say."""
    n, s = 40, starts_of(25, 15)
    x = [rand(i, n, h, 16) for i, h in enumerate((4, 2, 2))]
    g = rand(9, n, 4, 16)

    def loss(q, k, v):
        return (ops.attention(q, k, v, s, causal=True).double() * g.double()).sum().item()

    out, lse = ops.attention(*x, s, causal=True, want_lse=True)
    grads = ops.attention_backward(g, *x, out, lse, s, causal=True)
    for i in range(3):
        d = rand(20 + i, *x[i].shape)
        h = 1e-2
        step = [y + h * d if j == i else y for j, y in enumerate(x)]
        back = [y - h * d if j == i else y for j, y in enumerate(x)]
        slope = (grads[i].double() * d.double()).sum().item()
        # 4000 outputs off by 1e-6, over 2 h; the third derivative's share 1e-4
        assert abs((loss(*step) - loss(*back)) / (2 * h) - slope) <= 2e-3 * max(1.0, abs(slope))


def test_starts_that_do_not_fit_are_clamped_and_reported(ops):  # noqa: F811
    from paper_2108_03917_amd.lattice import E_RANGE, OK

    q, k, v = (rand(i, 100, 2, 32) for i in range(3))
    assert ops.status() == OK
    for bad in ([0, 50, 200], [-5, 50, 100], [0, 60, 40]):
        s = torch.tensor(bad, dtype=torch.int32, device=DEV)
        out, lse = ops.attention(q, k, v, s, want_lse=True)
        assert ops.status() == E_RANGE, bad
        ops.attention_backward(q, q, k, v, out, lse, s)
        assert ops.status() == E_RANGE, bad
    s = torch.tensor([0, 50, 100], dtype=torch.int32, device=DEV)
    for bad in ([51, 0], [-1, 3]):
        ops.attention(q, k, v, s, kv_lengths=torch.tensor(bad, dtype=torch.int32, device=DEV))
        assert ops.status() == E_RANGE, bad
    ops.attention(q, k, v, s, kv_lengths=torch.tensor([50, 0], dtype=torch.int32, device=DEV))
    assert ops.status() == OK


@pytest.mark.parametrize("sequences", [7, 61, 62, 300])
def test_starts_in_any_order_touch_nothing_else(ops, sequences):  # noqa: F811
    """Random starts and lengths, far outside the rows too: what lies around the
    tensors stays as it is."""
    from paper_2108_03917_amd.lattice import E_RANGE, OK

    n, C, pad = 500, 32, 4096
    g = torch.Generator(device=DEV)
    for seed in range(4):
        g.manual_seed(seed)
        far = 2 ** 31 - 1 if seed % 2 else 2 * n

        def starts():
            return torch.randint(-far, far, (sequences + 1,), generator=g, device=DEV).int()

        room = torch.full((2 * pad + n * 2 * C,), 3.0, device=DEV)
        out = room[pad:-pad].view(n, 2, C)
        q, k, v = (rand(i, n, 2, C) for i in range(3))
        packing = dict(q_starts=starts(), kv_starts=starts(), kv_lengths=starts()[1:])
        ops.attention(q, k, v, causal=bool(seed & 1), out=out, **packing)
        o, lse = ops.attention(q, k, v, causal=bool(seed & 1), want_lse=True, **packing)
        ops.attention_backward(q, q, k, v, o, lse, causal=bool(seed & 1), **packing)
        assert torch.all(room[:pad] == 3) and torch.all(room[-pad:] == 3)
        assert ops.status() == E_RANGE
    s = starts_of(n)
    ops.attention(q, k, v, s)
    assert ops.status() == OK


def test_refusals(ops):  # noqa: F811
    from paper_2108_03917_amd import LatticeError

    q, k, v = rand(1, 10, 4, 16), rand(2, 10, 2, 16), rand(3, 10, 2, 16)
    s = starts_of(4, 6)
    for bad in (lambda: ops.attention(q, k[:, :, :8], v[:, :, :8]), lambda: ops.attention(q, k, v[:5]),
                lambda: ops.attention(q, rand(1, 10, 3, 16), rand(1, 10, 3, 16)),
                lambda: ops.attention(q, k.bfloat16(), v), lambda: ops.attention(q.half(), k.half(), v.half()),
                lambda: ops.attention(q.cpu(), k, v), lambda: ops.attention(q[..., ::2], k[..., ::2], v[..., ::2]),
                lambda: ops.attention(q[0], k, v), lambda: ops.attention(q, k, v, s.long()),
                lambda: ops.attention(q, k, v, s, kv_starts=s[:2]), lambda: ops.attention(q, k, v, kv_starts=s),
                lambda: ops.attention(q, k, v, s, kv_lengths=s), lambda: ops.attention(q, k, v, out=q[:5]),
                lambda: ops.attention_backward(q, q, k, v, q, rand(1, 10, 4))):
        with pytest.raises(ValueError):
            bad()
    wide = rand(1, 10, 1, 129)
    for bad in (lambda: ops.attention(wide, wide, wide), lambda: ops.attention(q, k, v, scale=0.0),
                lambda: ops.attention(q, k, v, scale=-1.0), lambda: ops.attention(q, k, v, scale=float("nan")),
                lambda: ops.attention(q, k, v, out=q), lambda: ops.attention(q, k, v, out=rand(1, 10, 1, 16).expand(10, 4, 16))):
        with pytest.raises(LatticeError):
            bad()


def test_streams_and_graph(_gpu):  # noqa: F811
    """Called under another stream than the handle's, and captured: replays give what
    eager calls give, also after larger calls."""
    from paper_2108_03917_amd import Dense

    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    own = Dense(side)
    n = 600
    q, k, v, g = (rand(i, n, h, 64, dtype="bf16") for i, h in enumerate((8, 2, 2, 8)))
    s = starts_of(350, 250)
    long_k, long_q = rand(7, 6000, 2, 64, dtype="bf16"), rand(8, 2, 8, 64, dtype="bf16")

    def all_of():
        out, lse = own.attention(q, k, v, s, causal=True, want_lse=True)
        return [out, lse, *own.attention_backward(g, q, k, v, out, lse, s, causal=True),
                own.attention(long_q, long_k, long_k)]

    eager = [x.clone() for x in all_of()]          # another stream is current
    with torch.cuda.stream(side):
        graph = torch.cuda.CUDAGraph()
        side.synchronize()
        with torch.cuda.graph(graph, stream=side):
            got = all_of()
        for i in range(4):
            q.copy_(rand(30 + i, n, 8, 64, dtype="bf16"))
            own.attention(long_q, long_k.repeat(1 + i, 1, 1), long_k.repeat(1 + i, 1, 1))
            graph.replay()
            side.synchronize()
            want = all_of()
            side.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(got, want)), i
    assert not torch.equal(eager[0], got[0])
    own.close()
