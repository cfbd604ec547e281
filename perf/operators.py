"""Workloads of the 8-bit layer products and of the orthogonalised update.

Three kinds of pass:

* ``serve``: a linear layer whose weights were quantised once, ``y = x W^T (+ bias)``, for one token up to a long prompt;
* ``train``: the same layer in training: quantise the weights, forward, gradients of inputs, weights and bias;
* ``orth``:  momentum and Newton-Schulz orthogonalisation of the update of one matrix or of several of one shape.

``own`` chooses between the plain form (elementary torch operations in 32 bits) and this package's calls.
"""
import math

import torch

own = False

NS_COEF = (3.4445, -4.7750, 2.0315)
NS_EPS = 1e-7
MOMENTUM = 0.95
_DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}


# ---- cases ----------------------------------------------------------------------------------------------

def _serve(name, tokens, k, n, dtype="bf16", bias=False):
    return {"name": name, "kind": "serve", "tokens": tokens, "k": k, "n": n, "dtype": dtype, "bias": bias}


def _train(name, tokens, k, n, dtype="bf16", bias=False):
    return {"name": name, "kind": "train", "tokens": tokens, "k": k, "n": n, "dtype": dtype, "bias": bias}


def _orth(name, batch, rows, cols, dtype="fp32", nesterov=True):
    return {"name": name, "kind": "orth", "batch": batch, "rows": rows, "cols": cols, "dtype": dtype, "nesterov": nesterov}


def listed():
    return [
        # one token of one sequence through a square projection: latency
        _serve("token_2k", 1, 2048, 2048),
        # a decoding batch through a wide projection: the weights' bytes are all of it
        _serve("batch16_4k_16k", 16, 4096, 16384, bias=True),
        # a short prompt, no size a multiple of a tile
        _serve("prompt_odd", 333, 1000, 2500, dtype="fp32", bias=True),
        # a long prompt through a large layer
        _serve("prompt_8k", 8192, 8192, 8192),
        # a small layer in training, with bias
        _train("train_small", 512, 768, 768, bias=True),
        # an odd one in 32 bits (tokens of a ragged batch)
        _train("train_odd", 1999, 1153, 514, dtype="fp32", bias=True),
        # a layer of ordinary size in training
        _train("train_4k", 4096, 4096, 4096),
        # the four 64-channel 3x3 convolutions of ResNet-18, flattened to matrices: launches and latency
        _orth("conv64_x4", 4, 64, 576),
        # its three 512-channel ones
        _orth("conv512_x3", 3, 512, 4608),
        # its 1000-way last layer: taller than wide, odd
        _orth("head_1000x512", 1, 1000, 512, nesterov=False),
        # twelve square projections of a small transformer, gradients in bf16
        _orth("square768_x12", 12, 768, 768, dtype="bf16"),
        # one large square projection
        _orth("square4k", 1, 4096, 4096),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _ragged(rng, v):
    """v as it is, or moved off the multiples of eight."""
    return v if rng.random() < 0.4 else max(1, v // 8 * 8) if rng.random() < 0.5 else max(1, v // 8 * 8 + rng.choice((-3, -1, 1, 3)))


def draw(rng):
    kind = rng.choice(("serve", "serve", "train", "orth", "orth"))
    while True:
        if kind == "serve":
            tokens = _log_int(rng, 1, 32) if rng.random() < 0.5 else _log_int(rng, 16, 8192)
            c = {"kind": kind, "tokens": tokens, "k": _ragged(rng, _log_int(rng, 256, 8192)), "n": _ragged(rng, _log_int(rng, 256, 16384)),
                 "dtype": rng.choice(("bf16", "bf16", "fp16", "fp32")), "bias": rng.random() < 0.4}
        elif kind == "train":
            c = {"kind": kind, "tokens": _log_int(rng, 64, 8192), "k": _ragged(rng, _log_int(rng, 128, 6000)),
                 "n": _ragged(rng, _log_int(rng, 128, 6000)), "dtype": rng.choice(("bf16", "bf16", "fp32")), "bias": rng.random() < 0.4}
        else:
            batch = rng.choice((1, 1, 1, 2, 3, 6, 12))
            rows = _ragged(rng, _log_int(rng, 32, 4096))
            cols = _ragged(rng, max(16, min(8192, int(rows * math.exp(rng.uniform(math.log(0.25), math.log(4)))))))
            c = {"kind": kind, "batch": batch, "rows": rows, "cols": cols, "dtype": rng.choice(("fp32", "fp32", "bf16")),
                 "nesterov": rng.random() < 0.8}
        most = work({"kind": "serve", "tokens": 8192, "k": 8192, "n": 8192, "dtype": "bf16", "bias": False})
        top = work({"kind": "orth", "batch": 1, "rows": 4096, "cols": 4096, "dtype": "fp32", "nesterov": True})
        w = work(c)
        if w["flops"] <= (top if kind == "orth" else most)["flops"] and w["bytes"] <= most["bytes"]:
            return c


# ---- inputs ---------------------------------------------------------------------------------------------

def _activations(gen, tokens, k, dtype):
    """Normal entries, a few channels thirty times as large (as hidden states have them), tokens of unlike size."""
    x = torch.randn(tokens, k, device="cuda", generator=gen)
    channel = 1 + 29 * (torch.rand(k, device="cuda", generator=gen) < 0.005).float()
    token = torch.exp(0.5 * torch.randn(tokens, 1, device="cuda", generator=gen))
    return (x * channel * token).to(dtype)


def _int8_weights(w):
    """Weights as a program of this form loads them: whole numbers, rows on 16-byte boundaries, and a scale for each
    output channel."""
    s = w.abs().amax(1) * torch.tensor(1 / 127, dtype=torch.float32, device=w.device)
    q = torch.zeros(w.shape[0], (w.shape[1] + 15) // 16 * 16, dtype=torch.int8, device=w.device)
    q[:, :w.shape[1]] = torch.round(w * torch.reciprocal(s)[:, None]).to(torch.int8)
    return q[:, :w.shape[1]], s


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed) * 7919 + 13)
    dt = _DTYPES[case["dtype"]]
    st = {"case": case}
    if case["kind"] == "orth":
        b, m, n = case["batch"], case["rows"], case["cols"]
        r = max(1, min(m, n) // 16)       # gradients of a layer: a few strong directions and noise, decades between layers

        def grads():
            low = torch.randn(b, m, r, device="cuda", generator=gen) @ torch.randn(b, r, n, device="cuda", generator=gen)
            return low / math.sqrt(r) + torch.randn(b, m, n, device="cuda", generator=gen)
        sigma = 10 ** (-4 + 3 * torch.rand(b, 1, 1, device="cuda", generator=gen))
        st["g"] = (sigma * grads()).to(dt)
        st["momentum"] = (4 * sigma * grads()).contiguous()
        return st
    tokens, k, n = case["tokens"], case["k"], case["n"]
    st["x"] = _activations(gen, tokens, k, dt)
    w = torch.randn(n, k, device="cuda", generator=gen) / math.sqrt(k)
    w *= torch.exp(0.3 * torch.randn(n, 1, device="cuda", generator=gen))
    st["bias"] = 0.1 * torch.randn(n, device="cuda", generator=gen) if case["bias"] else None
    if case["kind"] == "serve":
        st["wq"], st["ws"] = _int8_weights(w)
    else:
        st["w"] = w
        # gradients of outputs: heavy tails, small
        t = torch.randn(tokens, n, device="cuda", generator=gen)
        st["dy"] = (1e-3 * t * torch.exp(torch.randn(tokens, 1, device="cuda", generator=gen))).to(dt)
    return st


# ---- plain forms ----------------------------------------------------------------------------------------

def _quantize(x, dim):
    """Whole numbers and scales along `dim`: the largest magnitude becomes 127; a line of zeros stays one."""
    s = x.abs().amax(dim, keepdim=True) * torch.tensor(1 / 127, dtype=torch.float32, device=x.device)
    return torch.round(x * torch.where(s < 2.0 ** -126, 0.0, torch.reciprocal(s))), s


def _plain_product(qa, sa, qb, sb):
    """sa (qa qb^T) sb for row scales sa, sb."""
    return (qa @ qb.T) * sa.reshape(-1, 1) * sb.reshape(1, -1)


def _plain_serve(st):
    x = st["x"]
    q, s = _quantize(x.float(), 1)
    y = _plain_product(q, s, st["wq"].float(), st["ws"])
    if st["bias"] is not None:
        y = y + st["bias"]
    return {"y": y.to(x.dtype)}


def _plain_train(st):
    x, w, dy = st["x"].float(), st["w"], st["dy"].float()
    y = _plain_product(*_quantize(x, 1), *_quantize(w, 1))
    out = {}
    if st["bias"] is not None:
        y = y + st["bias"]
        out["db"] = dy.sum(0)
    wc, ws = _quantize(w, 0)
    out["dx"] = _plain_product(*_quantize(dy, 1), wc.T, ws).to(st["x"].dtype)
    dc, ds = _quantize(dy, 0)
    xc, xs = _quantize(x, 0)
    out["dw"] = _plain_product(dc.T, ds, xc.T, xs)
    out["y"] = y.to(st["x"].dtype)
    return out


def _plain_ns_step(x):
    a = x @ x.transpose(1, 2)
    return NS_COEF[0] * x + (NS_COEF[1] * a + NS_COEF[2] * (a @ a)) @ x


def _plain_orth(st):
    g, buf = st["g"].float(), st["momentum"]
    buf.mul_(MOMENTUM).add_(g)
    u = g + MOMENTUM * buf if st["case"]["nesterov"] else buf
    tall = u.shape[1] > u.shape[2]
    x = u.transpose(1, 2) if tall else u
    x = x / ((x * x).sum((1, 2), keepdim=True).sqrt() + NS_EPS)
    x = _plain_ns_step(_plain_ns_step(_plain_ns_step(_plain_ns_step(_plain_ns_step(x)))))
    return {"momentum": buf, "update": (x.transpose(1, 2) if tall else x).contiguous().to(torch.bfloat16)}


# ---- the package's calls --------------------------------------------------------------------------------

_plans = {}      # what a program keeps: one plan for each shape of matrix


def _own_orth(st):
    from paper_1905_05957_b200 import OrthUpdate
    c = st["case"]
    key = (c["batch"], c["rows"], c["cols"], c["nesterov"])
    if key not in _plans:
        _plans.clear()
        _plans[key] = OrthUpdate(c["rows"], c["cols"], batch=c["batch"], momentum=MOMENTUM, nesterov=c["nesterov"],
                                 coef=NS_COEF, steps=5, eps=NS_EPS)
    return {"momentum": st["momentum"], "update": _plans[key].update(st["g"], st["momentum"], out_dtype=torch.bfloat16)}


def _own_serve(st):
    from paper_1905_05957_b200 import Int8Matrix, int8_linear
    return {"y": int8_linear(st["x"], Int8Matrix(st["wq"], st["ws"]), st["bias"])}


def _own_train(st):
    from paper_1905_05957_b200 import Int8Linear
    layer = Int8Linear(st["w"], st["bias"])
    y = layer.forward(st["x"], training=True)
    dx, dw, db = layer.backward(st["dy"])
    out = {"y": y, "dx": dx, "dw": dw}
    if db is not None:
        out["db"] = db
    return out


def run(state):
    kind = state["case"]["kind"]
    if own:
        return {"serve": _own_serve, "train": _own_train, "orth": _own_orth}[kind](state)
    return {"serve": _plain_serve, "train": _plain_train, "orth": _plain_orth}[kind](state)


# ---- what a pass cannot do without ----------------------------------------------------------------------

def work(case):
    size = {"fp32": 4, "bf16": 2, "fp16": 2}[case["dtype"]]
    if case["kind"] == "orth":
        b, m, n = case["batch"], min(case["rows"], case["cols"]), max(case["rows"], case["cols"])
        # gradient and momentum in, momentum and update out; the two symmetric products at half
        return {"bytes": b * m * n * (size + 4 + 4 + 2), "flops": 5 * b * (m * m * n + m * m * m + 2 * m * m * n)}
    t, k, n = case["tokens"], case["k"], case["n"]
    extra = 4 * n if case["bias"] else 0
    if case["kind"] == "serve":
        return {"bytes": size * t * k + n * k + 4 * n + size * t * n + extra, "flops": 2 * t * k * n}
    # x, w, dy in; y, dx, dw (and the bias's gradient) out
    return {"bytes": size * t * k + 4 * n * k + size * t * n + size * t * n + size * t * k + 4 * n * k + 2 * extra,
            "flops": 6 * t * k * n}


# ---- the definitions in 64 bits -------------------------------------------------------------------------

def _codes64(v, axis):
    """The whole numbers nearest to v / s along `axis`, and s: the scales are numbers of 32 bits by definition."""
    top = v.abs().max(axis, keepdim=True).values.to(torch.float32)
    s = (top * torch.tensor(1 / 127, dtype=torch.float32, device=v.device)).to(torch.float64)
    return torch.round(v / s), s


def exact(case, seed):
    st = prepare(case, seed)
    f8 = torch.float64
    if case["kind"] == "orth":
        g = st["g"].to(f8)
        buf = MOMENTUM * st["momentum"].to(f8) + g
        u = MOMENTUM * buf + g if case["nesterov"] else buf
        flip = case["rows"] > case["cols"]
        z = torch.stack([(v.T if flip else v) / (torch.linalg.matrix_norm(v) + NS_EPS) for v in u])
        p, q, r = NS_COEF
        for _ in range(5):
            gram = torch.bmm(z, z.mT)
            z = p * z + q * torch.bmm(gram, z) + r * torch.bmm(gram, torch.bmm(gram, z))
        return {"momentum": buf, "update": z.mT if flip else z}
    x = st["x"].to(f8)
    bias = 0 if st["bias"] is None else st["bias"].to(f8)
    xq, xs = _codes64(x, 1)
    if case["kind"] == "serve":
        return {"y": torch.mm(xq, st["wq"].to(f8).T) * xs * st["ws"].to(f8) + bias}
    w, dy = st["w"].to(f8), st["dy"].to(f8)
    wq, ws = _codes64(w, 1)
    out = {"y": torch.mm(xq * xs, (wq * ws).T) + bias}
    if case["bias"]:
        out["db"] = dy.sum(0)
    gq, gs = _codes64(dy, 1)
    vq, vs = _codes64(w, 0)
    out["dx"] = torch.mm(gq * gs, vq * vs)
    hq, hs = _codes64(dy, 0)
    zq, zs = _codes64(x, 0)
    out["dw"] = torch.mm((hq * hs).T, zq * zs)
    return out
