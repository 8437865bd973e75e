"""Dense operators on inputs that are taken in several pieces: of rows, of
classes, and of matrices of a batch.  References and tolerances are those of
test_gpu_dense.py unless a test derives its own."""
import pytest
import torch

from tests.gpu_util import REL_F32
from tests.test_gpu_dense import _gpu, check, check_loss, check_update, labels, loss_ref, ops, rand, update_ref  # noqa: F401

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


def loss_terms(x, w, target, bias):
    """What bounds the gradients of bf16 operands (mean loss): for grad_x and
    grad_w the value, the fp32 scale (see loss_ref), the sum of |terms| and the
    root of the sum of their squares."""
    ref = loss_ref(x, w, target, bias, True)
    x, w = x.double(), w.double()
    on = (target >= 0) & (target < w.shape[0])
    G = torch.softmax(x @ w.t() + bias.double(), 1)
    G.scatter_add_(1, torch.where(on, target, 0)[:, None], torch.full_like(G[:, :1], -1.0))
    G *= (on / on.sum())[:, None]
    G *= G
    return {"grad_x": (*ref["grad_x"], (G @ (w * w)).sqrt()),
            "grad_w": (*ref["grad_w"], (G.t() @ (x * x)).sqrt())}, ref


def check_gradients(got, terms, bits):
    """Gradients of bf16 operands whose d loss / dz has `bits` significant bits:
    2^-8 of itself for the stored result; fp32 sums; and the intermediate's
    rounding, at most 2^-bits of each term, with signs that the operands' random
    signs make independent: the sum passes 8 times 2^-bits of the terms' root
    of squares once in 1e13 elements (Hoeffding)."""
    for name, g in zip(("grad_x", "grad_w"), got):
        v, scale, _, rss = terms[name]
        bound = 2.0 ** -8 * v.abs() + REL_F32 * scale + 8 * 2.0 ** -bits * rss + 1e-30
        worst = ((g.double() - v).abs() / bound).max().item()
        assert worst <= 1.0, f"{name}: error {worst:.3g} times the tolerance"


@pytest.mark.parametrize("N,C,K", [(7000, 200, 60001), (4700, 192, 65536)])
def test_kept_logits_in_pieces(ops, N, C, K):  # noqa: F811
    """fp32 with at least 192 channels keeps a piece's logits, 2^28 at most: two
    pieces of rows, the last one shorter and no multiple of a tile, and
    several of classes."""
    x, w, t, bias = rand(1, N, C), rand(2, K, C) * 0.1, labels(3, N, K), rand(4, K)
    got = ops.linear_cross_entropy(x, w, t, bias, want_rows=True, want_grad=True)
    check_loss(got, loss_ref(x, w, t, bias, True), "f32")
    again = ops.linear_cross_entropy(x, w, t, bias, want_rows=True, want_grad=True)
    assert all(torch.equal(a, b) for a, b in zip(got, again))


@pytest.mark.parametrize("N,C,K,dtype", [(105536, 100, 1200, "f32"), (105536, 64, 2500, "bf16"),
                                         (105536, 72, 2500, "bf16"), (70000, 48, 200, "bf16")])
def test_loss_in_pieces_of_rows_and_classes(ops, N, C, K, dtype):  # noqa: F811
    """The last piece holds 6 to 38 of a hundred rows: far more of a gradient than
    the tolerance.  Operands as they are (64 bf16 channels) and laid out."""
    x, w, t, bias = rand(1, N, C, dtype=dtype), rand(2, K, C, dtype=dtype) * 0.3, labels(3, N, K), rand(4, K)
    got = ops.linear_cross_entropy(x, w, t, bias, want_rows=True, want_grad=True)
    terms, ref = loss_terms(x, w, t, bias)
    check_loss(got, ref, dtype)
    if dtype == "bf16":
        check_gradients(got[2:4], terms, 8)


@pytest.mark.parametrize("batch,m,n,dtype", [(450, 8, 8192, "f32"), (450, 8192, 8, "bf16"), (133, 130, 4096, "f32"),
                                             (200, 130, 4096, "bf16")])
def test_update_in_chunks_of_a_batch(ops, batch, m, n, dtype):  # noqa: F811
    """More matrices than are taken together (scratch of 2 GiB); the last chunk
    is smaller, down to one matrix, and takes other tiles."""
    g = rand(1, batch, m, n, dtype=dtype)
    got = ops.orthogonalize(g)
    for b0 in range(0, batch, 64):
        check_update(got[b0:b0 + 64], update_ref(g[b0:b0 + 64]), b0)
    # each as alone, up to the parts that its sums are made of
    for b in (0, batch - 1):
        check_update(ops.orthogonalize(g[b]), got[b].double(), b)


FEW = [(5000, 64, 20), (3000, 128, 20), (700, 96, 50), (257, 33, 3), (2000, 128, 100), (900, 256, 40)]


@pytest.mark.parametrize("N,C,K", FEW)
def test_gradients_of_few_classes_in_bf16(ops, N, C, K):  # noqa: F811
    """d loss / dz keeps 16 bits in the products that give the gradients."""
    x, w, t, bias = rand(1, N, C, dtype="bf16"), (rand(2, K, C) * 0.3).bfloat16(), labels(3, N, K), rand(4, K)
    got = ops.linear_cross_entropy(x, w, t, bias, want_rows=True, want_grad=True)
    terms, ref = loss_terms(x, w, t, bias)
    check_loss(got, ref, "bf16")
    check_gradients(got[2:4], terms, 16)


MANY = [(1000, 64, 200), (513, 100, 777), (300, 130, 129), (128, 260, 1000), (2048, 512, 3000), (40, 64, 1000),
        (3000, 260, 100), (105536, 64, 2500), (70000, 48, 200)]


@pytest.mark.parametrize("N,C,K", MANY)
def test_gradients_of_many_classes_in_16_bits(ops, N, C, K):  # noqa: F811
    """A handle that asks for them, on every tile, in one piece and in several;
    what the bits do not enter is the same, bit for bit."""
    from paper_2108_03917_amd import Dense

    x, w, t, bias = rand(1, N, C, dtype="bf16"), (rand(2, K, C) * 0.3).bfloat16(), labels(3, N, K), rand(4, K)
    own = Dense(gradient_bits=16)
    got = own.linear_cross_entropy(x, w, t, bias, want_rows=True, want_grad=True)
    terms, ref = loss_terms(x, w, t, bias)
    check_loss(got, ref, "bf16")
    check_gradients(got[2:4], terms, 16)
    again = own.linear_cross_entropy(x, w, t, bias, want_rows=True, want_grad=True)
    assert all(torch.equal(a, b) for a, b in zip(got, again))
    only = [own.linear_cross_entropy(x, w, t, bias, want_grad=True, want_input=i == 0, want_weight=i == 1,
                                     want_bias=False)[1 + i] for i in range(2)]
    assert torch.equal(only[0], got[2]) and torch.equal(only[1], got[3])
    eight = ops.linear_cross_entropy(x, w, t, bias, want_rows=True, want_grad=True)
    assert torch.equal(eight[0], got[0]) and torch.equal(eight[1], got[1])
    check(got[4], eight[4].double(), ref["grad_bias"][1], REL_F32, "grad_bias")
    torch.cuda.synchronize()
    own.close()


def test_gradient_bits_that_are_neither(ops):  # noqa: F811
    from paper_2108_03917_amd import Dense

    for bits in (0, 7, 24):
        with pytest.raises(ValueError):
            Dense(gradient_bits=bits)


@pytest.mark.parametrize("batch,m,n", [(1, 1531, 700), (2, 1255, 1504), (1, 2000, 2048)])
def test_update_is_as_accurate_as_fp32_products(ops, batch, m, n):  # noqa: F811
    """The same steps in plain fp32 products are no nearer to 64 bits."""
    g = rand(1, batch, m, n) + rand(2, batch, m, 40) @ rand(3, batch, 40, n)
    ref = update_ref(g)
    a, b, c = 3.4445, -4.7750, 2.0315
    x = g.mT.contiguous() if m > n else g
    x = x / (x.square().sum((-2, -1), keepdim=True).sqrt() + 1e-7)
    for _ in range(5):
        s = torch.matmul(x, x.mT.contiguous())
        x = a * x + torch.matmul(b * s + c * torch.matmul(s, s), x)
    plain = ((x.mT if m > n else x).double() - ref).norm()
    assert (ops.orthogonalize(g).double() - ref).norm() <= plain
