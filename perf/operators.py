"""The dense operators of a training step around the lattice: what is measured.

Three kinds of call, each from one row to the largest size a user has:

  norm     layer normalisation of the channels of each row, and with train=True
           the gradients of the rows, the gain and the shift
  loss     the linear classifier with its softmax cross entropy, from features to
           the mean loss (and each row's loss), and with train=True the gradients
           of the features, the weights and the bias; rows without a label count
           for nothing
  update   the orthogonalised form of a gradient matrix (or of a batch of them) by
           five Newton-Schulz steps, which a training program subtracts from its
           weights

``run`` computes them in elementary operations in 32 bits where ``own`` is false,
and calls the library where it is true.
"""
import math

import torch

own = False

DEV = "cuda" if torch.cuda.is_available() else "cpu"
EPS = 1e-5                                # of the normalisation
IGNORE = -100                             # the label of a row that has none
NS = (3.4445, -4.7750, 2.0315)            # coefficients of a Newton-Schulz step
NS_STEPS, NS_EPS = 5, 1e-7


def _norm(name, rows, channels, dtype, train):
    return {"name": name, "op": "norm", "rows": rows, "channels": channels, "dtype": dtype, "train": train}


def _loss(name, rows, channels, classes, dtype, train):
    return {"name": name, "op": "loss", "rows": rows, "channels": channels, "classes": classes, "dtype": dtype,
            "train": train}


def _update(name, batch, m, n, dtype):
    return {"name": name, "op": "update", "batch": batch, "m": m, "n": n, "dtype": dtype}


def listed():
    return [
        # one row at inference: the smallest call, all latency
        _norm("norm_one_row", 1, 1024, "bf16", False),
        # a LiDAR scan's points, a width that is no power of two, both directions
        _norm("norm_scan_ragged", 82411, 100, "f32", True),
        # wide rows of a large batch, both directions: all bandwidth
        _norm("norm_wide", 16384, 4096, "bf16", True),
        # a training step's loss on one part-segmentation object
        _loss("loss_object", 2613, 64, 50, "f32", True),
        # the same on the points of the largest indoor room
        _loss("loss_room", 537211, 64, 20, "f32", True),
        # a LiDAR scan, wider features stored in 16 bits
        _loss("loss_scan", 103889, 128, 20, "bf16", True),
        # a few rows scored against a large vocabulary: the weights are read once
        _loss("loss_vocab_few", 64, 1024, 32768, "bf16", False),
        # a training step over a large vocabulary: the largest call
        _loss("loss_vocab_train", 8192, 1024, 65536, "bf16", True),
        # the weights of one 64 -> 64 convolution over nine taps
        _update("update_conv", 1, 64, 576, "f32"),
        # the 128 -> 128 convolutions of a deep network, all in one call
        _update("update_layers", 12, 128, 1152, "f32"),
        # a tall matrix of odd size
        _update("update_tall_ragged", 1, 1531, 700, "f32"),
        # the weights of a wide layer
        _update("update_wide", 1, 2048, 8192, "bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """A case of the same ranges, sizes spread over their logarithm."""
    op = rng.choice(["norm", "loss", "loss", "update"])
    dtype = rng.choice(["bf16", "f32"])
    if op == "norm":
        channels = _log(rng, 16, 8192)
        rows = min(_log(rng, 1, 540000), 16384 * 4096 // channels)
        case = _norm("", rows, channels, dtype, rng.random() < 0.7)
    elif op == "loss" and rng.random() < 0.5:       # the labels of a segmentation
        case = _loss("", _log(rng, 100, 537211), rng.choice([16, 32, 48, 64, 64, 96, 100, 128, 256]),
                     _log(rng, 2, 128), dtype, rng.random() < 0.75)
    elif op == "loss":                              # a vocabulary
        channels, classes = _log(rng, 64, 2048), _log(rng, 1000, 65536)
        most = (2.0e11 if dtype == "f32" else 5.0e11) / (channels * classes)
        case = _loss("", max(1, int(min(_log(rng, 1, 8192), most))), channels, classes, dtype, rng.random() < 0.6)
    else:
        m, n = sorted((_log(rng, 8, 2048), _log(rng, 64, 8192)))
        most = (6.0e9 if dtype == "f32" else 3.0e10) / (m * m * n)
        if most < 1:                                # no dearer than the largest listed one
            n = max(m, int(n * most))
        batch = max(1, min(_log(rng, 1, 16), int(most)))
        if rng.random() < 0.3:
            m, n = n, m
        case = _update("", batch, m, n, dtype)
    del case["name"]
    return case


# -- inputs ------------------------------------------------------------------

def _type(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))

    def normal(*shape):
        return torch.randn(*shape, generator=g, device=DEV)

    t = _type(case)
    if case["op"] == "norm":
        r, c = case["rows"], case["channels"]
        s = {"x": (normal(r, c) * (0.5 + torch.rand(r, 1, generator=g, device=DEV)) + 0.3 * normal(1, c)).to(t),
             "gamma": 1 + 0.2 * normal(c), "beta": 0.1 * normal(c)}
        if case["train"]:
            s["grad"] = normal(r, c).to(t)
    elif case["op"] == "loss":
        r, c, k = case["rows"], case["channels"], case["classes"]
        # frequent and rare classes, and one row in twenty without a label
        target = (torch.rand(r, generator=g, device=DEV) ** 2 * k).long().clamp_(max=k - 1)
        target[torch.rand(r, generator=g, device=DEV) < 0.05] = IGNORE
        s = {"x": normal(r, c).to(t), "w": (normal(k, c) * (2 / math.sqrt(c))).to(t), "bias": 0.5 * normal(k),
             "target": target}
    else:
        b, m, n = case["batch"], case["m"], case["n"]
        # a gradient's spectrum: a part of low rank, and noise
        rank = max(1, min(m, n) // 4)
        low = torch.matmul(normal(b, m, rank), normal(b, rank, n)) / math.sqrt(rank)
        s = {"g": ((low + 0.25 * normal(b, m, n)) * 1e-3).to(t)}
        if b == 1:
            s["g"] = s["g"][0]
    s["case"] = case
    return s


# -- one pass ----------------------------------------------------------------

_kept = []


def _dense():
    """The library's handle that a program keeps for its life."""
    if not _kept:
        from paper_2108_03917_amd import Dense

        _kept.append(Dense())
    return _kept[0]


def run(state):
    case = state["case"]
    if own:
        ops = _dense()
        if case["op"] == "norm":
            if not case["train"]:
                return ops.layer_norm(state["x"], state["gamma"], state["beta"], eps=EPS)
            y, mean, rstd = ops.layer_norm(state["x"], state["gamma"], state["beta"], eps=EPS, want_stats=True)
            return [y, *ops.layer_norm_backward(state["grad"], state["x"], mean, rstd, state["gamma"])]
        if case["op"] == "loss":
            args = (state["x"], state["w"], state["target"], state["bias"])
            if case["train"]:
                return ops.linear_cross_entropy(*args, ignore_index=IGNORE, want_grad=True)
            return ops.linear_cross_entropy(*args, ignore_index=IGNORE, want_rows=True)
        return ops.orthogonalize(state["g"], steps=NS_STEPS, coefficients=NS, eps=NS_EPS)
    return {"norm": _plain_norm, "loss": _plain_loss, "update": _plain_update}[case["op"]](state, case)


def _plain_norm(state, case):
    x, gamma, beta = state["x"].float(), state["gamma"], state["beta"]
    mean = x.mean(1, keepdim=True)
    d = x - mean
    rstd = torch.rsqrt((d * d).mean(1, keepdim=True) + EPS)
    xh = d * rstd
    y = (xh * gamma + beta).to(state["x"].dtype)
    if not case["train"]:
        return y
    g = state["grad"].float()
    gg = g * gamma
    gx = rstd * (gg - gg.mean(1, keepdim=True) - xh * (gg * xh).mean(1, keepdim=True))
    return [y, gx.to(state["x"].dtype), (g * xh).sum(0), g.sum(0)]


def _plain_loss(state, case):
    x, w, target = state["x"].float(), state["w"].float(), state["target"]
    valid = target != IGNORE
    count = valid.sum().clamp(min=1)
    safe = torch.where(valid, target, 0)[:, None]
    z = torch.matmul(x, w.t()) + state["bias"]
    top = z.amax(1, keepdim=True)
    e = torch.exp(z - top)
    total = e.sum(1, keepdim=True)
    rows = torch.where(valid, (top + torch.log(total) - z.gather(1, safe))[:, 0], 0.0)
    loss = rows.sum() / count
    if not case["train"]:
        return [loss, rows]
    share = torch.where(valid, 1.0 / count, 0.0)[:, None]
    p = e * (share / total)
    p.scatter_add_(1, safe, -share)
    return [loss, torch.matmul(p, w).to(state["x"].dtype), torch.matmul(p.t(), x).to(state["w"].dtype), p.sum(0)]


def _plain_update(state, case):
    a, b, c = NS
    x = state["g"].float()
    tall = case["m"] > case["n"]
    if tall:
        x = x.mT.contiguous()
    x = x / (torch.sqrt((x * x).sum((-2, -1), keepdim=True)) + NS_EPS)
    for _ in range(NS_STEPS):
        s = torch.matmul(x, x.mT.contiguous())
        x = a * x + torch.matmul(b * s + c * torch.matmul(s, s), x)
    if tall:
        x = x.mT
    return x.to(state["g"].dtype).contiguous()


# -- 64 bits -----------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "norm":
        x = s["x"].double()
        var, mu = torch.var_mean(x, dim=1, correction=0, keepdim=True)
        sd = (var + EPS).sqrt()
        h = (x - mu) / sd
        gain = s["gamma"].double()
        y = torch.addcmul(s["beta"].double(), h, gain)
        if not case["train"]:
            return y
        g = s["grad"].double()
        # the Jacobian of the normalisation is a projection: off the mean and off h
        v = g * gain
        v = v - v.mean(1, keepdim=True)
        v = v - h * (v * h).sum(1, keepdim=True) / x.shape[1]
        return [y, v / sd, (g * h).sum(0), g.sum(0)]
    if case["op"] == "loss":
        x, w, t = s["x"].double(), s["w"].double(), s["target"]
        has = t.ne(IGNORE).nonzero()[:, 0]          # the rows with a label, alone
        labels = t[has]
        z = torch.addmm(s["bias"].double(), x[has], w.t())
        lse = torch.logsumexp(z, dim=1)
        each = lse - z[torch.arange(has.numel(), device=z.device), labels]
        n = max(1, has.numel())
        if not case["train"]:
            rows = torch.zeros(x.shape[0], dtype=torch.float64, device=x.device)
            rows[has] = each
            return [each.sum() / n, rows]
        p = (z - lse[:, None]).exp_()
        del z
        p[torch.arange(has.numel(), device=p.device), labels] -= 1
        p /= n
        gx = torch.zeros_like(x)
        gx[has] = p @ w
        return [each.sum() / n, gx, p.t() @ x[has], p.sum(0)]
    g = s["g"].double().reshape(case["batch"], case["m"], case["n"])
    a, b, c = NS
    out = []
    for one in g:
        u = one if case["m"] <= case["n"] else one.t()
        u = u / (torch.linalg.norm(u) + NS_EPS)
        eye = torch.eye(u.shape[0], dtype=torch.float64, device=u.device)
        for _ in range(NS_STEPS):
            s2 = u @ u.t()
            u = (a * eye + s2 @ (b * eye + c * s2)) @ u
        out.append(u if case["m"] <= case["n"] else u.t())
    out = torch.stack(out)
    return out[0] if case["batch"] == 1 else out


# -- what a pass cannot do without -------------------------------------------

def work(case):
    e = 4 if case["dtype"] == "f32" else 2
    if case["op"] == "norm":
        r, c = case["rows"], case["channels"]
        n = r * c
        if not case["train"]:
            return {"bytes": 2 * e * n + 8 * c, "flops": 8 * n}
        # rows and their gradients in, normalised rows and gradients out
        return {"bytes": 4 * e * n + 16 * c, "flops": 22 * n}
    if case["op"] == "loss":
        r, c, k = case["rows"], case["channels"], case["classes"]
        reads = e * (r * c + k * c) + 8 * r + 4 * k
        if not case["train"]:
            return {"bytes": reads + 4 * r, "flops": 2 * r * c * k}
        # the logits, and the two products that the gradients are
        return {"bytes": reads + e * (r * c + k * c) + 4 * k, "flops": 6 * r * c * k}
    b, m, n = case["batch"], min(case["m"], case["n"]), max(case["m"], case["n"])
    # a step: the symmetric x x', the symmetric square of it, and its product with x
    step = m * (m + 1) * n + m * m * (m + 1) + 2 * m * m * n
    return {"bytes": 2 * e * b * m * n, "flops": NS_STEPS * b * step}
