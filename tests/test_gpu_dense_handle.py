"""The handle of the dense operators: graphs and scratch, empty inputs."""
import pytest
import torch

from tests.test_gpu_dense import DEV, _gpu, labels, ops, rand  # noqa: F401

pytestmark = pytest.mark.gpu


def test_graph_replays_after_larger_calls(_gpu):  # noqa: F811
    """What a graph uses stays when later calls need more scratch, those in the
    capture itself among them."""
    from paper_2108_03917_amd import Dense

    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        own = Dense(s)
        x, w, t, b = rand(1, 300, 64), rand(2, 500, 64), labels(3, 300, 500), rand(4, 500)
        large, tl = rand(5, 5000, 64), labels(6, 5000, 500)
        g, wide = rand(7, 200, 250), rand(8, 600, 1000)

        def all_of():
            y, mean, rstd = own.layer_norm(x, want_stats=True)
            r = [*own.layer_norm_backward(x, x, mean, rstd)]
            r += own.linear_cross_entropy(x, w, t, b, want_rows=True, want_grad=True)
            return r + [own.orthogonalize(g)]

        all_of()
        s.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            out = all_of()
            out += own.linear_cross_entropy(large[:1500], w, tl[:1500], b, want_grad=True)
            out += all_of()
        for i in range(4):
            x.copy_(rand(10 + i, 300, 64))
            g.copy_(rand(20 + i, 200, 250))
            # more scratch each time but the last
            n = min(2000 + 1500 * i, 5000)
            own.linear_cross_entropy(large[:n], w, tl[:n], b, want_grad=True)
            own.orthogonalize(wide)
            graph.replay()
            s.synchronize()
            eager = all_of()
            eager += own.linear_cross_entropy(large[:1500], w, tl[:1500], b, want_grad=True)
            eager += all_of()
            s.synchronize()
            assert all(torch.equal(a, c) for a, c in zip(out, eager)), i
        own.close()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("C", [32, 9000, 17000])
def test_layer_norm_without_rows(ops, C, dtype):  # noqa: F811
    x = rand(1, 0, C, dtype=dtype)
    y, mean, rstd = ops.layer_norm(x, want_stats=True)
    assert y.shape == (0, C) and mean.shape == rstd.shape == (0,)
    gx, gg, gb = ops.layer_norm_backward(x, x, mean, rstd)
    assert gx.shape == (0, C) and gx.dtype == x.dtype
    assert gg.shape == gb.shape == (C,) and torch.all(gg == 0) and torch.all(gb == 0)
    gx, gg, gb = ops.layer_norm_backward(x, x, mean, rstd, want_params=False)
    assert gx.shape == (0, C) and gg is None and gb is None
    gx, gg, gb = ops.layer_norm_backward(x, x, mean, rstd, want_input=False)
    assert gx is None and torch.all(gg == 0) and torch.all(gb == 0)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("m,n", [(30, 64), (64, 3000), (150, 170)])
@pytest.mark.parametrize("steps", [0, 1, 5])
def test_update_of_zeros_without_eps(ops, m, n, steps, dtype):  # noqa: F811
    """Zeros stay zeros where nothing is added to their norm; a NaN stays one."""
    g = rand(1, 3, m, n, dtype=dtype)
    g[1] = 0
    g[2, 1, 2] = float("nan")
    got = ops.orthogonalize(g, steps=steps, eps=0.0)
    assert torch.all(got[1] == 0) and torch.isfinite(got[0]).all() and torch.isnan(got[2]).any()
    assert torch.equal(got[0], ops.orthogonalize(g[0], steps=steps, eps=0.0))
