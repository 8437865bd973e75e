"""Attention between the points or tokens of a sequence, and what stands around it
in a training step: what is measured.

Three kinds of call, each from the smallest to the largest size a user has:

  attend   softmax attention over packed sequences of different lengths, with
           grouped heads: "packed", each row a query, a key and a value, and with
           train=True the gradients of all three; or "cached", a few new rows of
           each sequence against a cache of which each sequence fills a part
  rotate   the norm of each head's query and key with a gain for each channel, and
           the rotation by the row's position along one axis or several, in one
           call for both; with train=True the gradients of queries, keys and gains
  clip     the norm over all gradients of a model, and the gradients scaled down
           to a largest norm

``run`` computes them in elementary operations in 32 bits where ``own`` is false,
and calls the library where it is true.
"""
import math

import torch

own = False

DEV = "cuda" if torch.cuda.is_available() else "cpu"
EPS = 1e-6                                # of the norms of heads and of all gradients


def _packed(name, sequences, tokens, heads, kv_heads, dim, dtype, causal, train):
    return {"name": name, "op": "attend", "form": "packed", "sequences": sequences, "tokens": tokens, "heads": heads,
            "kv_heads": kv_heads, "dim": dim, "dtype": dtype, "causal": causal, "train": train}


def _cached(name, sequences, new, capacity, heads, kv_heads, dim, dtype):
    return {"name": name, "op": "attend", "form": "cached", "sequences": sequences, "new": new, "capacity": capacity,
            "heads": heads, "kv_heads": kv_heads, "dim": dim, "dtype": dtype, "causal": True, "train": False}


def _rotate(name, tokens, heads, kv_heads, dim, axes, dtype, train):
    return {"name": name, "op": "rotate", "tokens": tokens, "heads": heads, "kv_heads": kv_heads, "dim": dim,
            "axes": axes, "dtype": dtype, "train": train}


def _clip(name, tensors, values, dtype):
    return {"name": name, "op": "clip", "tensors": tensors, "values": values, "dtype": dtype}


def listed():
    return [
        # one new token of one short sequence: the smallest call, all latency
        _cached("attend_one_token", 1, 1, 77, 8, 8, 64, "bf16"),
        # the next token of many sequences, each with its part of a cache: the
        # caches are read once
        _cached("attend_tokens_cached", 48, 1, 8192, 32, 8, 128, "bf16"),
        # all points of each object of a batch of part-segmentation objects, a
        # training step in 32 bits; no order among points
        _packed("attend_objects_train", 16, 16 * 2613, 4, 4, 32, "f32", False, True),
        # heads of a width that is no power of two, sequences from one row on
        _packed("attend_ragged_odd_train", 7, 1501, 6, 2, 36, "bf16", True, True),
        # one long sequence in order, a forward pass
        _packed("attend_long", 1, 16384, 16, 4, 128, "bf16", True, False),
        # a training step on a batch of sequences of different lengths: the largest
        _packed("attend_packed_train", 12, 16384, 16, 4, 128, "bf16", True, True),
        # one new token of one sequence
        _rotate("rotate_one_token", 1, 32, 8, 128, 1, "bf16", False),
        # the points of a LiDAR scan, by their coordinates, a training step
        _rotate("rotate_scan_train", 82411, 4, 4, 36, 3, "f32", True),
        # a training step's rows of wide heads, by place and time
        _rotate("rotate_wide_train", 16384, 32, 8, 128, 4, "bf16", True),
        # the gradients of a small lattice network
        _clip("clip_small", 6, 42000, "f32"),
        # those of a deep network with layers of many sizes
        _clip("clip_layers", 60, 30_000_001, "f32"),
        # those of a large network
        _clip("clip_large", 48, 400_000_000, "bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """A case of the same ranges, sizes spread over their logarithm."""
    op = rng.choice(["attend", "attend", "attend", "rotate", "clip"])
    dtype = rng.choice(["bf16", "f32"])
    dim = rng.choice([16, 20, 24, 32, 36, 40, 48, 64, 64, 72, 80, 96, 100, 128, 128])
    kv_heads = rng.choice([1, 2, 3, 4, 5, 8])
    heads = kv_heads * rng.choice([1, 1, 2, 3, 4, 8])
    if op == "attend" and rng.random() < 0.4:
        sequences, new, capacity = _log(rng, 1, 64), rng.choice([1, 1, 1, 2, 3, 5]), _log(rng, 16, 16384)
        most = 2.0e8 / (kv_heads * dim)             # values of all keys
        sequences = max(1, min(sequences, int(most / capacity)))
        capacity = max(16, min(capacity, int(most / sequences)))
        case = _cached("", sequences, new, capacity, heads, kv_heads, dim, dtype)
    elif op == "attend":
        train = rng.random() < 0.6
        sequences, tokens = _log(rng, 1, 64), _log(rng, 64, 32768)
        tokens = max(tokens, sequences)
        # the plain form holds the scores of all pairs of a sequence several times
        most = 6.0e8 if train else 2.1e9
        each = most / (heads * sequences * (6 if sequences > 1 else 1))
        tokens = max(sequences, min(tokens, int(sequences * math.sqrt(each))))
        case = _packed("", sequences, tokens, heads, kv_heads, dim, dtype, rng.random() < 0.5, train)
    elif op == "rotate":
        tokens = min(_log(rng, 1, 130000), 16384 * 40 * 128 // ((heads + kv_heads) * dim))
        case = _rotate("", tokens, heads, kv_heads, dim, rng.choice([1, 2, 3, 4]), dtype, rng.random() < 0.7)
    else:
        tensors = _log(rng, 1, 60)
        case = _clip("", tensors, max(tensors, _log(rng, 300, 200_000_000)), dtype)
    del case["name"]
    return case


def _parts(n, total, least):
    """n whole numbers that add up to total, of many sizes, the first the least of
    them where there are several."""
    weight = [0.1 + (0.6180339887 * (i + 1) % 1.0) ** 2 for i in range(n)]
    if n > 2:
        weight[0] = 0.0
    got = [least + int((total - n * least) * w / sum(weight)) for w in weight]
    got[n // 2] += total - sum(got)
    return got


def _lengths(case):
    """Keys of each sequence."""
    n = case["sequences"]
    if case["form"] == "packed":
        return _parts(n, case["tokens"], 1)
    cap = case["capacity"]
    got = [cap - int(0.8 * cap * (0.6180339887 * i % 1.0)) for i in range(n)]
    if n > 4:
        got[1], got[2] = min(cap, case["new"]), 0     # a first token, and an empty place
    return got


def _sections(case):
    """Pairs of channels that turn with each axis; a few turn with none."""
    pairs, axes = case["dim"] // 2, case["axes"]
    if axes == 1:
        return [pairs]
    return [pairs // axes] * axes


# -- inputs ------------------------------------------------------------------

def _type(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))

    def normal(*shape):
        return torch.randn(*shape, generator=g, device=DEV)

    t = _type(case)
    h, kh, d = case.get("heads"), case.get("kv_heads"), case.get("dim")
    s = {"case": case}
    if case["op"] == "attend":
        lengths = _lengths(case)
        n = len(lengths)
        ends = torch.tensor(lengths).cumsum(0)
        if case["form"] == "packed":
            rows = keys = case["tokens"]
            # one projection gives queries, keys and values, next to each other
            qkv = normal(rows, h + 2 * kh, d).to(t)
            s["q"], s["k"], s["v"] = qkv[:, :h], qkv[:, h:h + kh], qkv[:, h + kh:]
            s["starts"] = torch.cat([torch.zeros(1, dtype=torch.long), ends]).to(torch.int32).to(DEV)
        else:
            rows, keys = n * case["new"], n * case["capacity"]
            s["q"], s["k"], s["v"] = normal(rows, h, d).to(t), normal(keys, kh, d).to(t), normal(keys, kh, d).to(t)
            s["q_starts"] = torch.arange(n + 1, dtype=torch.int32, device=DEV) * case["new"]
            s["kv_starts"] = torch.arange(n + 1, dtype=torch.int32, device=DEV) * case["capacity"]
            s["lengths"] = torch.tensor(lengths, dtype=torch.int32).to(DEV)
        if case["train"]:
            s["grad"] = normal(rows, h, d).to(t)
    elif case["op"] == "rotate":
        n, pairs = case["tokens"], sum(_sections(case))
        qk = (normal(n, h + kh, d) * (0.5 + torch.rand(n, 1, 1, generator=g, device=DEV))).to(t)
        s["q"], s["k"] = qk[:, :h], qk[:, h:]
        if case["axes"] == 1:                      # places of tokens in a long text
            s["pos"] = torch.randint(0, 100000, (n, 1), generator=g, device=DEV).to(torch.float32)
        else:                                      # metres, and the scan's number
            s["pos"] = 40 * normal(n, case["axes"])
        per = _sections(case)[0]
        turn = torch.arange(pairs, device=DEV) % per
        s["freq"] = (10000.0 ** (-turn.double() / per)).float()
        s["gain_q"], s["gain_k"] = 1 + 0.2 * normal(d), 1 + 0.2 * normal(d)
        if case["train"]:
            s["grad_q"], s["grad_k"] = normal(n, h, d).to(t), normal(n, kh, d).to(t)
    else:
        sizes = _parts(case["tensors"], case["values"], 1)
        s["grads"] = [(normal(v) * 10.0 ** (-3 + i % 3)).to(t) for i, v in enumerate(sizes)]
        s["out"] = [torch.empty_like(v) for v in s["grads"]]
        # about a third of their norm
        s["most"] = 0.3 * math.sqrt(sum(v * 100.0 ** (-3 + i % 3) for i, v in enumerate(sizes)))
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
        if case["op"] == "attend":
            q, k, v = state["q"], state["k"], state["v"]
            if case["form"] == "cached":
                return ops.attention(q, k, v, state["q_starts"], state["kv_starts"], state["lengths"], causal=True)
            if not case["train"]:
                return ops.attention(q, k, v, state["starts"], causal=case["causal"])
            out, lse = ops.attention(q, k, v, state["starts"], causal=case["causal"], want_lse=True)
            return [out, *ops.attention_backward(state["grad"], q, k, v, out, lse, state["starts"],
                                                 causal=case["causal"])]
        if case["op"] == "rotate":
            args = (state["q"], state["k"], state["pos"], state["freq"], _sections(case), state["gain_q"],
                    state["gain_k"])
            out = [*ops.rotate_heads(*args, eps=EPS)]
            if case["train"]:
                out += ops.rotate_heads_backward(state["grad_q"], state["grad_k"], *args, eps=EPS)
            return out
        norm = ops.clip_gradients(state["grads"], state["most"], eps=EPS, out=state["out"])
        return [norm, *state["out"]]
    return {"attend": _plain_attend, "rotate": _plain_rotate, "clip": _plain_clip}[case["op"]](state, case)


def _plain_attend(state, case):
    """Sequences side by side, padded to the longest."""
    h, kh, d = case["heads"], case["kv_heads"], case["dim"]
    group = h // kh
    n, lengths = case["sequences"], _lengths(case)
    q, k, v = state["q"].float(), state["k"].float(), state["v"].float()
    if case["form"] == "packed":
        q_start = k_start = state["starts"][:-1].long()
        q_len = k_len = state["starts"][1:].long() - q_start
        lq = lk = max(lengths)
    else:
        q_start, k_start = state["q_starts"][:-1].long(), state["kv_starts"][:-1].long()
        q_len, k_len = state["q_starts"][1:].long() - q_start, state["lengths"].long()
        lq, lk = case["new"], max(lengths)
    i, j = torch.arange(lq, device=DEV), torch.arange(lk, device=DEV)

    def side_by_side(x, start, length, at):         # [rows, heads, d] to [n, heads, longest, d]
        has = at < length[:, None]
        y = x[torch.where(has, start[:, None] + at, 0)]
        return torch.where(has[:, :, None, None], y, 0.0).transpose(1, 2).contiguous()

    def rows_of(x, start, rows):                    # and back
        r = torch.arange(rows, device=DEV)
        b = (r[:, None] >= start[None, 1:]).sum(1)
        return x[b, :, r - start[b]]

    qs = side_by_side(q, q_start, q_len, i).view(n, kh, group * lq, d)
    ks, vs = side_by_side(k, k_start, k_len, j), side_by_side(v, k_start, k_len, j)
    seen = j < k_len[:, None, None]
    if case["causal"]:
        seen = seen & (j <= i[:, None] + (k_len - q_len)[:, None, None])
    seen = seen[:, None, None]
    scale = 1 / math.sqrt(d)
    p = torch.matmul(qs, ks.mT.contiguous()).view(n, kh, group, lq, lk).mul_(scale)
    p.masked_fill_(~seen, -math.inf)
    top = p.amax(-1, keepdim=True)
    p.sub_(torch.where(top == -math.inf, 0.0, top)).exp_()
    p.div_(p.sum(-1, keepdim=True).clamp_(min=1e-30))
    p = p.view(n, kh, group * lq, lk)
    o = torch.matmul(p, vs)
    rows = q.shape[0]
    out = rows_of(o.view(n, h, lq, d), q_start, rows).to(state["q"].dtype)
    if not case["train"]:
        return out
    go = side_by_side(state["grad"].float(), q_start, q_len, i).view(n, kh, group * lq, d)
    gv = torch.matmul(p.mT.contiguous(), go)
    gs = torch.matmul(go, vs.mT.contiguous())
    gs.sub_((go * o).sum(-1, keepdim=True)).mul_(p).mul_(scale)
    del p
    gq = torch.matmul(gs, ks)
    gk = torch.matmul(gs.mT.contiguous(), qs)
    t = state["q"].dtype
    return [out, rows_of(gq.view(n, h, lq, d), q_start, rows).to(t), rows_of(gk, k_start, k.shape[0]).to(t),
            rows_of(gv, k_start, k.shape[0]).to(t)]


def _angles(state, case):
    """Of each row and pair of channels, [rows, 1, pairs], in 64 bits: a far
    position's angle has too many turns for 32."""
    per = _sections(case)[0]
    turn = torch.arange(state["freq"].shape[0], device=DEV)
    a = state["pos"].double()[:, turn // per] * state["freq"].double()
    return torch.cos(a).float()[:, None], torch.sin(a).float()[:, None]


def _plain_rotate(state, case):
    cos, sin = _angles(state, case)
    half = cos.shape[-1]

    def turned(x, s):                               # channels c and c + half are a pair, the others stay
        a, b = x[..., :half], x[..., half:2 * half]
        return torch.cat([a * cos - b * s, b * cos + a * s, x[..., 2 * half:]], -1)

    xq, xk = state["q"].float(), state["k"].float()
    rq = torch.rsqrt((xq * xq).mean(-1, keepdim=True) + EPS)
    rk = torch.rsqrt((xk * xk).mean(-1, keepdim=True) + EPS)
    out = [turned(xq * rq * state["gain_q"], sin).to(state["q"].dtype),
           turned(xk * rk * state["gain_k"], sin).to(state["k"].dtype)]
    if not case["train"]:
        return out

    def gradients(g, x, r, gain):
        u = turned(g.float(), -sin)
        n = x * r
        w = u * gain
        return (r * (w - n * (w * n).mean(-1, keepdim=True))).to(g.dtype), (u * n).sum((0, 1))

    gq, ggq = gradients(state["grad_q"], xq, rq, state["gain_q"])
    gk, ggk = gradients(state["grad_k"], xk, rk, state["gain_k"])
    return out + [gq, gk, ggq, ggk]


def _plain_clip(state, case):
    squares = torch.stack([(g.float() * g.float()).sum() for g in state["grads"]])
    norm = torch.sqrt(squares.sum())
    factor = torch.clamp(state["most"] / (norm + EPS), max=1.0)
    return [norm] + [(g.float() * factor).to(g.dtype) for g in state["grads"]]


# -- 64 bits -----------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    wide = dict(dtype=torch.float64, device=DEV)

    def attend():
        """One sequence, one head and a piece of its queries at a time."""
        h, kh, d = case["heads"], case["kv_heads"], case["dim"]
        out, gq = torch.zeros(s["q"].shape, **wide), torch.zeros(s["q"].shape, **wide)
        gk, gv = torch.zeros(s["k"].shape, **wide), torch.zeros(s["k"].shape, **wide)
        at = 0
        for b, keys in enumerate(_lengths(case)):
            if case["form"] == "packed":
                q0, k0, queries = at, at, keys
                at += keys
            else:
                q0, k0, queries = b * case["new"], b * case["capacity"], case["new"]
            if keys == 0:
                continue
            for head in range(h):
                mine = head * kh // h
                k, v = s["k"][k0:k0 + keys, mine].double(), s["v"][k0:k0 + keys, mine].double()
                for first in range(0, queries, 8192):
                    rows = slice(q0 + first, q0 + min(queries, first + 8192))
                    q = s["q"][rows, head].double()
                    z = (q @ k.t()) / math.sqrt(d)
                    last = torch.full((z.shape[0],), keys - 1, device=DEV)
                    if case["causal"]:
                        last = torch.arange(first, first + z.shape[0], device=DEV) + keys - queries
                    z = z.masked_fill(torch.arange(keys, device=DEV)[None] > last[:, None], -math.inf)
                    p = torch.where((last < 0)[:, None], 0.0, torch.softmax(z, dim=1))
                    out[rows, head] = p @ v
                    if case["train"]:
                        g = s["grad"][rows, head].double()
                        gv[k0:k0 + keys, mine] += p.t() @ g
                        dp = g @ v.t()
                        # the Jacobian of the softmax takes off the mean under p
                        ds = p * (dp - (p * dp).sum(1, keepdim=True)) / math.sqrt(d)
                        gq[rows, head] = ds @ k
                        gk[k0:k0 + keys, mine] += ds.t() @ q
        return [out, gq, gk, gv] if case["train"] else out

    def rotate():
        per = _sections(case)[0]
        pairs = s["freq"].shape[0]
        angle = torch.stack([s["pos"][:, p // per].double() * s["freq"][p].double() for p in range(pairs)], 1)[:, None]
        phase = torch.polar(torch.ones_like(angle), angle)

        def turn(x, phase):                         # pairs as complex numbers
            z = torch.complex(x[..., :pairs].contiguous(), x[..., pairs:2 * pairs].contiguous()) * phase
            return torch.cat([z.real, z.imag, x[..., 2 * pairs:]], -1)

        out, gx, gg = [], [], []
        for name in ("q", "k"):
            x, gain = s[name].double(), s["gain_" + name].double()
            size = (x.square().mean(-1, keepdim=True) + EPS).sqrt()
            unit = x / size
            out.append(turn(unit * gain, phase))
            if case["train"]:
                u = turn(s["grad_" + name].double(), phase.conj())
                w = u * gain
                gx.append((w - unit * (w * unit).mean(-1, keepdim=True)) / size)
                gg.append((u * unit).sum((0, 1)))
        return out + gx + gg

    def clip():
        norm = math.sqrt(sum(float(g.double().square().sum()) for g in s["grads"]))
        factor = min(1.0, s["most"] / (norm + EPS))
        return [torch.tensor(norm, dtype=torch.float64)] + [g.double() * factor for g in s["grads"]]

    return {"attend": attend, "rotate": rotate, "clip": clip}[case["op"]]()


# -- what a pass cannot do without -------------------------------------------

def work(case):
    e = 4 if case["dtype"] == "f32" else 2
    if case["op"] == "attend":
        h, kh, d = case["heads"], case["kv_heads"], case["dim"]
        lengths = _lengths(case)
        if case["form"] == "packed":
            pairs = sum(n * (n + 1) // 2 if case["causal"] else n * n for n in lengths)
            rows = keys = case["tokens"]
        else:
            new = case["new"]
            pairs = sum(max(0, n - new + i + 1) for n in lengths for i in range(new))
            rows, keys = len(lengths) * new, sum(lengths)
        q, kv = e * rows * h * d, e * keys * kh * d
        if not case["train"]:
            return {"bytes": 2 * q + 2 * kv, "flops": 4 * d * h * pairs}
        # and the scores again, two products for d loss / d scores and the values'
        # gradient, two for those of queries and keys
        return {"bytes": 4 * q + 4 * kv, "flops": 14 * d * h * pairs}
    if case["op"] == "rotate":
        n = case["tokens"] * (case["heads"] + case["kv_heads"]) * case["dim"]
        rest = 4 * case["tokens"] * case["axes"] + 8 * case["dim"]
        if not case["train"]:
            return {"bytes": 2 * e * n + rest, "flops": 7 * n}
        return {"bytes": 4 * e * n + 2 * rest, "flops": 20 * n}
    return {"bytes": 2 * e * case["values"] + 4, "flops": 3 * case["values"]}
