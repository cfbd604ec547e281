"""Workloads of the 16-bit layer with its epilogue, of the norms around a residual connection, and of dropout.

Four kinds of pass:

* ``serve``:   a linear layer in 16-bit floats, ``y = act(x W^T + b) + r``, for one token up to a long prompt;
* ``train``:   the same layer in training: forward, gradients of inputs, weights and bias;
* ``norm``:    what stands between two blocks of a network, ``h = a x + D(g * post(y))`` and ``n = pre(h)`` (post and pre RMS or layer norms, g a
  gate, D dropout), forward alone or with all gradients;
* ``dropout``: dropout of activations and of their gradients, the mask drawn again instead of kept.

``own`` chooses between the plain form (elementary torch operations in 32 bits) and this package's calls.
"""
import math

import torch

own = False

NORM_EPS = 1e-5
_DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
_SIZES = {"fp32": 4, "bf16": 2, "fp16": 2}


# ---- cases ----------------------------------------------------------------------------------------------

def _linear(name, kind, tokens, k, n, dtype="bf16", act="none", bias=False, residual=False):
    return {"name": name, "kind": kind, "tokens": tokens, "k": k, "n": n, "dtype": dtype, "act": act, "bias": bias, "residual": residual}


def _norm(name, rows, cols, norm="rms", dtype="bf16", stream="", post=True, pre=True, groups=0, p=0.0, train=False):
    return {"name": name, "kind": "norm", "rows": rows, "cols": cols, "norm": norm, "dtype": dtype, "stream": stream or dtype, "post": post,
            "pre": pre, "groups": groups, "p": p, "train": train}


def _dropout(name, rows, cols, dtype="bf16", p=0.1):
    return {"name": name, "kind": "dropout", "rows": rows, "cols": cols, "dtype": dtype, "p": p}


def listed():
    return [
        # one token of one sequence through a widening projection: latency
        _linear("token_2k_8k", "serve", 1, 2048, 8192, act="gelu", bias=True),
        # a decoding batch through a wide projection: the weights' bytes are all of it
        _linear("batch16_4k_16k", "serve", 16, 4096, 16384, act="silu"),
        # a short prompt, no size a multiple of a tile, added to the residual stream
        _linear("prompt_333", "serve", 333, 1000, 2500, dtype="fp16", bias=True, residual=True),
        # a long prompt through a large layer, added to the residual stream
        _linear("prompt_8k", "serve", 8192, 8192, 8192, bias=True, residual=True),
        # an odd layer in training (tokens of a ragged batch)
        _linear("layer_odd", "train", 1999, 1153, 514, dtype="fp16", act="gelu_tanh", bias=True),
        # a layer of ordinary size in training
        _linear("layer_4k", "train", 4096, 4096, 4096, act="gelu", bias=True),
        # one token between two blocks: latency
        _norm("norm_token", 1, 4096),
        # a ragged prompt, odd width, floats, layer norms
        _norm("norm_777x1153", 777, 1153, norm="layer", dtype="fp32"),
        # training of a small network: layer norm before a block only, dropout on what it adds
        _norm("norm_train_768", 4096, 768, norm="layer", post=False, p=0.1, train=True),
        # training of a large one: eight sequences with a gate each, residual stream in 32 bits
        _norm("norm_train_4k", 16384, 4096, stream="fp32", groups=8, p=0.05, train=True),
        # dropout of a small layer's activations
        _dropout("drop_512x768", 512, 768),
        # of a large one's
        _dropout("drop_16k_8k", 16384, 8192, p=0.2),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _ragged(rng, v):
    """v as it is, or moved off the multiples of eight."""
    return v if rng.random() < 0.4 else max(1, v // 8 * 8) if rng.random() < 0.5 else max(1, v // 8 * 8 + rng.choice((-3, -1, 1, 3)))


def draw(rng):
    kind = rng.choice(("serve", "serve", "train", "norm", "norm", "dropout"))
    top = {c["name"]: work(c) for c in listed()}
    while True:
        if kind in ("serve", "train"):
            tokens = _log_int(rng, 64, 8192) if kind == "train" else _log_int(rng, 1, 32) if rng.random() < 0.5 else _log_int(rng, 16, 8192)
            c = {"kind": kind, "tokens": tokens, "k": _ragged(rng, _log_int(rng, 256, 8192)), "n": _ragged(rng, _log_int(rng, 256, 16384)),
                 "dtype": rng.choice(("bf16", "bf16", "fp16")), "act": rng.choice(("none", "relu", "gelu", "gelu_tanh", "silu")),
                 "bias": rng.random() < 0.5, "residual": rng.random() < 0.4}
            most = top["prompt_8k"]
        elif kind == "norm":
            dtype = rng.choice(("bf16", "bf16", "fp16", "fp32"))
            groups = rng.choice((0, 0, 1, 4, 16))
            rows = _log_int(rng, 1, 32768)
            c = {"kind": kind, "rows": max(1, rows // groups) * groups if groups else rows, "cols": _ragged(rng, _log_int(rng, 64, 8192)),
                 "norm": rng.choice(("rms", "layer")), "dtype": dtype, "stream": rng.choice((dtype, dtype, "fp32")), "post": rng.random() < 0.6,
                 "pre": rng.random() < 0.8, "groups": groups, "p": rng.choice((0.0, 0.0, 0.1, 0.5)), "train": rng.random() < 0.6}
            most = top["norm_train_4k"]
        else:
            c = {"kind": kind, "rows": _log_int(rng, 64, 32768), "cols": _ragged(rng, _log_int(rng, 64, 16384)),
                 "dtype": rng.choice(("bf16", "fp16", "fp32")), "p": rng.choice((0.1, 0.2, 0.5))}
            most = top["drop_16k_8k"]
        w = work(c)
        if w["flops"] <= most["flops"] and w["bytes"] <= most["bytes"]:
            return c


# ---- inputs ---------------------------------------------------------------------------------------------

def _activations(gen, tokens, k, dtype):
    """Normal entries, a few channels ten times as large (as hidden states have them), tokens of unlike size."""
    x = torch.randn(tokens, k, device="cuda", generator=gen)
    channel = 1 + 9 * (torch.rand(k, device="cuda", generator=gen) < 0.005).float()
    token = torch.exp(0.5 * torch.randn(tokens, 1, device="cuda", generator=gen))
    return (x * channel * token).to(dtype)


def _gradients(gen, tokens, n, dtype):
    """Small, with heavy tails from token to token."""
    t = torch.randn(tokens, n, device="cuda", generator=gen)
    return (1e-2 * t * torch.exp(torch.randn(tokens, 1, device="cuda", generator=gen))).to(dtype)


def _rows16(w):
    """The weights as a program that serves them keeps them: rows on 16-byte boundaries."""
    buf = torch.zeros(w.shape[0], (w.shape[1] + 7) // 8 * 8, dtype=w.dtype, device=w.device)
    buf[:, :w.shape[1]] = w
    return buf[:, :w.shape[1]]


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed) * 7919 + 13)
    dt = _DTYPES[case["dtype"]]
    st = {"case": case}
    if case["kind"] in ("serve", "train"):
        tokens, k, n = case["tokens"], case["k"], case["n"]
        st["x"] = _activations(gen, tokens, k, dt)
        w = torch.randn(n, k, device="cuda", generator=gen) / math.sqrt(k)
        w = (w * torch.exp(0.3 * torch.randn(n, 1, device="cuda", generator=gen))).to(dt)
        st["w"] = _rows16(w) if case["kind"] == "serve" else w
        st["bias"] = 0.1 * torch.randn(n, device="cuda", generator=gen) if case["bias"] else None
        st["residual"] = _activations(gen, tokens, n, dt) if case["residual"] else None
        if case["kind"] == "train":
            st["dy"] = _gradients(gen, tokens, n, dt)
        return st
    rows, cols = case["rows"], case["cols"]
    st["draws"] = (int(seed) * 1000003 + 17, 3, int(seed) % 1000)      # seed, layer, step: what the random bits are a function of
    if case["kind"] == "dropout":
        st["x"], st["dy"] = _activations(gen, rows, cols, dt), _gradients(gen, rows, cols, dt)
        return st
    ds = _DTYPES[case["stream"]]
    st["y"] = _activations(gen, rows, cols, dt)
    st["x"] = _activations(gen, rows, cols, ds)
    if case["norm"] == "layer":      # layer norms take a mean away
        st["x"] += 0.5
        st["y"] += 0.25

    def weight():
        return 1 + 0.2 * torch.randn(cols, device="cuda", generator=gen)
    layer = case["norm"] == "layer"
    st["post_weight"] = weight() if case["post"] else None
    st["post_bias"] = 0.1 * torch.randn(cols, device="cuda", generator=gen) if case["post"] and layer else None
    st["pre_weight"] = weight() if case["pre"] else None
    st["pre_bias"] = 0.1 * torch.randn(cols, device="cuda", generator=gen) if case["pre"] and layer else None
    st["gate"] = 0.5 * torch.randn(case["groups"], cols, device="cuda", generator=gen) if case["groups"] else None
    if case["train"]:
        st["dh"] = _gradients(gen, rows, cols, ds)
        st["dn"] = _gradients(gen, rows, cols, dt) if case["pre"] else None
    return st


RESIDUAL_SCALE = 0.9


# ---- plain forms ----------------------------------------------------------------------------------------

def _act(z, name):
    if name == "relu":
        return torch.where(z > 0, z, 0.0)
    if name == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    if name == "gelu_tanh":
        return 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z * z * z)))
    if name == "silu":
        return z / (1 + torch.exp(-z))
    return z


def _act_slope(z, name):
    if name == "relu":
        return (z > 0).float()
    if name == "gelu":
        return 0.5 * (1 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) * (1 / math.sqrt(2 * math.pi))
    if name == "gelu_tanh":
        t = torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z * z * z))
        return 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * math.sqrt(2 / math.pi) * (1 + 3 * 0.044715 * z * z)
    if name == "silu":
        s = 1 / (1 + torch.exp(-z))
        return s * (1 + z * (1 - s))
    return torch.ones_like(z)


def _plain_linear(st):
    c, dt = st["case"], st["x"].dtype
    x, w = st["x"].float(), st["w"].float()
    z = x @ w.T
    if st["bias"] is not None:
        z = z + st["bias"]
    y = _act(z, c["act"])
    if st["residual"] is not None:
        y = y + st["residual"].float()
    out = {"y": y.to(dt)}
    if c["kind"] == "train":
        dz = st["dy"].float() * _act_slope(z, c["act"])
        out["dx"], out["dw"] = (dz @ w).to(dt), (dz.T @ x).to(dt)
        if st["bias"] is not None:
            out["db"] = dz.sum(0).to(dt)
    return out


def _philox(c0, c1, c2, c3, k0, k1):
    """Philox4x32-10 on int64 tensors that hold 32-bit words; products wrap around, which their low 64 bits survive."""
    low = 0xFFFFFFFF
    p, q = c0 * 0xD2511F53, c2 * 0xCD9E8D57
    c0, c1, c2, c3 = (q >> 32 & low) ^ c1 ^ k0, q & low, (p >> 32 & low) ^ c3 ^ k1, p & low
    return c0, c1, c2, c3, (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low


def _drop_threshold(p):
    """Dropout's probability in 65536ths: an entry is dropped where its 16 random bits are below it."""
    return int(math.floor(p * 65536 + 0.5))


def _kept(rows, cols, p, draws, device):
    """The mask: entry c of row r takes half c mod 8 (the low half of word 0 first) of Philox4x32-10 of counter (c / 8, r, layer, step), with the
    seed's two words as the key, the high one xored with 0x44524F50."""
    seed, layer, step = draws
    groups = (cols + 7) // 8
    zero = torch.zeros(rows, groups, dtype=torch.int64, device=device)
    s = (zero + torch.arange(groups, device=device), zero + torch.arange(rows, device=device)[:, None], zero + layer, zero + step,
         seed & 0xFFFFFFFF, seed >> 32 & 0xFFFFFFFF ^ 0x44524F50)
    s = _philox(*_philox(*_philox(*_philox(*_philox(*s)))))
    s = _philox(*_philox(*_philox(*_philox(*_philox(*s)))))
    w = torch.stack(s[:4], 2)
    half = torch.stack((w & 0xFFFF, w >> 16), 3).reshape(rows, 8 * groups)
    return half[:, :cols] >= _drop_threshold(p)


def _plain_dropout(st):
    c, x, dy = st["case"], st["x"], st["dy"]
    kept = _kept(c["rows"], c["cols"], c["p"], st["draws"], x.device)
    scale = 65536 / (65536 - _drop_threshold(c["p"]))
    return {"y": torch.where(kept, x.float() * scale, 0.0).to(x.dtype), "dx": torch.where(kept, dy.float() * scale, 0.0).to(x.dtype)}


def _plain_normed(v, kind):
    """The normalised rows and the reciprocal of their size."""
    if kind == "layer":
        v = v - v.mean(1, keepdim=True)
    r = 1 / torch.sqrt((v * v).mean(1, keepdim=True) + NORM_EPS)
    return v * r, r


def _plain_norm_back(t, hat, r, kind):
    """The gradient of the rows from that of the normalised ones."""
    d = t - hat * (t * hat).mean(1, keepdim=True)
    if kind == "layer":
        d = d - t.mean(1, keepdim=True)
    return r * d


def _by_group(g, rows):
    """The gate of every row: rows are as many equal runs as there are gates."""
    return g.repeat_interleave(rows // g.shape[0], 0)


def _plain_norm(st):
    c = st["case"]
    rows, kind = c["rows"], c["norm"]
    dt, ds = st["y"].dtype, st["x"].dtype
    y, x = st["y"].float(), st["x"].float()
    u = y
    if c["post"]:
        hat1, r1 = _plain_normed(y, kind)
        u = hat1 * st["post_weight"]
        if st["post_bias"] is not None:
            u = u + st["post_bias"]
    v = u
    if c["groups"]:
        gate = _by_group(st["gate"], rows)
        u = u * gate
    if c["p"]:
        kept = _kept(rows, c["cols"], c["p"], st["draws"], y.device)
        scale = 65536 / (65536 - _drop_threshold(c["p"]))
        u = torch.where(kept, u * scale, 0.0)
    h = RESIDUAL_SCALE * x + u
    out = {"h": h.to(ds)}
    if c["pre"]:
        hat2, r2 = _plain_normed(h, kind)
        n = hat2 * st["pre_weight"]
        if st["pre_bias"] is not None:
            n = n + st["pre_bias"]
        out["n"] = n.to(dt)
    if not c["train"]:
        return out
    d = st["dh"].float()
    if c["pre"]:
        dn = st["dn"].float()
        out["pre_weight"] = (dn * hat2).sum(0)
        if st["pre_bias"] is not None:
            out["pre_bias"] = dn.sum(0)
        d = d + _plain_norm_back(dn * st["pre_weight"], hat2, r2, kind)
    out["dx"] = (RESIDUAL_SCALE * d).to(ds)
    if c["p"]:
        d = torch.where(kept, d * scale, 0.0)
    if c["groups"]:
        out["gate"] = (d * v).reshape(c["groups"], rows // c["groups"], -1).sum(1)
        d = d * gate
    if c["post"]:
        out["post_weight"] = (d * hat1).sum(0)
        if st["post_bias"] is not None:
            out["post_bias"] = d.sum(0)
        d = _plain_norm_back(d * st["post_weight"], hat1, r1, kind)
    out["dy"] = d.to(dt)
    return out


# ---- the package's calls --------------------------------------------------------------------------------

def _own_linear(st):
    from paper_1905_05957_b200 import Linear16, linear16
    c = st["case"]
    if c["kind"] == "serve":
        return {"y": linear16(st["x"], st["w"], st["bias"], activation=c["act"], residual=st["residual"])}
    layer = Linear16(st["w"], st["bias"], activation=c["act"])
    out = {"y": layer.forward(st["x"], residual=st["residual"], training=True)}
    out["dx"], out["dw"], db = layer.backward(st["dy"])
    if db is not None:
        out["db"] = db
    return out


def _own_dropout(st):
    from paper_1905_05957_b200 import dropout
    seed, layer, step = st["draws"]
    p = st["case"]["p"]
    return {"y": dropout(st["x"], p, seed, step=step, layer=layer), "dx": dropout(st["dy"], p, seed, step=step, layer=layer)}


def _own_norm(st):
    from paper_1905_05957_b200 import ResidualNorm
    c = st["case"]
    seed, layer, step = st["draws"]
    op = ResidualNorm(c["norm"], post_weight=st["post_weight"], post_bias=st["post_bias"], gate=st["gate"], pre_weight=st["pre_weight"],
                      pre_bias=st["pre_bias"], residual_scale=RESIDUAL_SCALE, eps=NORM_EPS, p=c["p"], seed=seed, layer=layer)
    h, n = op.forward(st["y"], st["x"], step=step, training=c["train"])
    out = {"h": h}
    if n is not None:
        out["n"] = n
    if c["train"]:
        out["dy"], out["dx"], grads = op.backward(st["dh"], st["dn"])
        out.update(grads)
    return out


def run(state):
    kind = state["case"]["kind"]
    if own:
        return {"serve": _own_linear, "train": _own_linear, "norm": _own_norm, "dropout": _own_dropout}[kind](state)
    return {"serve": _plain_linear, "train": _plain_linear, "norm": _plain_norm, "dropout": _plain_dropout}[kind](state)


# ---- what a pass cannot do without ----------------------------------------------------------------------

def work(case):
    size = _SIZES[case["dtype"]]
    if case["kind"] in ("serve", "train"):
        t, k, n = case["tokens"], case["k"], case["n"]
        # x, weights, bias and residual in, y out
        once = size * (t * k + n * k + t * n) + (4 * n if case["bias"] else 0) + (size * t * n if case["residual"] else 0)
        if case["kind"] == "serve":
            return {"bytes": once, "flops": 2 * t * k * n}
        # and the gradient of y in, those of x, the weights and the bias out
        return {"bytes": once + size * (t * n + t * k + n * k) + (size * n if case["bias"] else 0), "flops": 6 * t * k * n}
    entries = case["rows"] * case["cols"]
    if case["kind"] == "dropout":
        return {"bytes": 4 * size * entries, "flops": 2 * entries}
    stream = _SIZES[case["stream"]]
    vectors = 4 * case["cols"] * (case["groups"] + (1 + (case["norm"] == "layer")) * (case["post"] + case["pre"]))
    # x and y in, h and n out; the gradients of h and n in, those of x and y out
    one = size * (1 + case["pre"]) + 2 * stream
    return {"bytes": entries * one * (2 if case["train"] else 1) + vectors * (2 if case["train"] else 1), "flops": entries * (40 if case["train"] else 14)}


# ---- the definitions in 64 bits -------------------------------------------------------------------------

def _bits64(rows, cols, draws):
    """The same random halves from a generator of its own: 32 x 32-bit products by 16-bit limbs, counters as one flat list."""
    seed, layer, step = draws
    groups = -(-cols // 8)
    at = torch.arange(rows * groups, device="cuda")
    ctr = [at % groups, at // groups, torch.full_like(at, layer), torch.full_like(at, step)]
    key = [seed % 2 ** 32, (seed // 2 ** 32) % 2 ** 32 ^ 0x44524F50]

    def wide(a, m):
        ml, mh = m % 65536, m // 65536
        al, ah = a % 65536, a // 65536
        low = al * ml
        mid = ah * ml + low // 65536
        mid2 = al * mh + mid % 65536
        return ah * mh + mid // 65536 + mid2 // 65536, (mid2 % 65536) * 65536 + low % 65536
    for _ in range(10):
        h0, l0 = wide(ctr[0], 0xD2511F53)
        h1, l1 = wide(ctr[2], 0xCD9E8D57)
        ctr = [h1 ^ ctr[1] ^ key[0], l1, h0 ^ ctr[3] ^ key[1], l0]
        key = [(key[0] + 0x9E3779B9) % 2 ** 32, (key[1] + 0xBB67AE85) % 2 ** 32]
    halves = torch.empty(rows * groups, 8, dtype=torch.int32, device="cuda")
    for i, word in enumerate(ctr):
        halves[:, 2 * i], halves[:, 2 * i + 1] = word % 65536, word // 65536
    return halves.view(rows, groups * 8)[:, :cols]


def _dropped64(v, p, draws):
    below = round(p * 65536)
    return v * (_bits64(*v.shape, draws) >= below).to(v.dtype) / (1 - below / 65536)


def _exact_linear(st):
    c, f8 = st["case"], torch.float64
    x, w = st["x"].to(f8).requires_grad_(), st["w"].to(f8).requires_grad_()
    b = torch.zeros(c["n"], dtype=f8, device="cuda") if st["bias"] is None else st["bias"].to(f8)
    b.requires_grad_()
    z = torch.addmm(b, x, w.mT)
    y = {"none": lambda v: v, "relu": torch.relu, "gelu": torch.nn.functional.gelu, "silu": torch.nn.functional.silu,
         "gelu_tanh": lambda v: torch.nn.functional.gelu(v, approximate="tanh")}[c["act"]](z)
    if st["residual"] is not None:
        y = y + st["residual"].to(f8)
    out = {"y": y.detach()}
    if c["kind"] == "train":
        out["dx"], out["dw"], db = torch.autograd.grad(y, (x, w, b), st["dy"].to(f8))
        if c["bias"]:
            out["db"] = db
    return out


def _exact_norm(st):
    c, f8 = st["case"], torch.float64
    leaf = {k: st[k].to(f8).requires_grad_() for k in ("y", "x", "post_weight", "post_bias", "pre_weight", "pre_bias", "gate") if st[k] is not None}

    def norm(v, which):
        if c["norm"] == "layer":
            return torch.nn.functional.layer_norm(v, v.shape[1:], leaf[which + "_weight"], leaf[which + "_bias"], NORM_EPS)
        return v * torch.rsqrt(v.square().mean(1, True) + NORM_EPS) * leaf[which + "_weight"]
    u = norm(leaf["y"], "post") if c["post"] else leaf["y"]
    if c["groups"]:
        u = (u.view(c["groups"], -1, c["cols"]) * leaf["gate"][:, None]).view(u.shape)
    if c["p"]:
        u = _dropped64(u, c["p"], st["draws"])
    h = RESIDUAL_SCALE * leaf["x"] + u
    out, ends, given = {"h": h.detach()}, [h], [st.get("dh")]
    if c["pre"]:
        n = norm(h, "pre")
        out["n"] = n.detach()
        ends.append(n)
        given.append(st.get("dn"))
    if c["train"]:
        grads = torch.autograd.grad(ends, list(leaf.values()), [g.to(f8) for g in given])
        out.update({{"x": "dx", "y": "dy"}.get(k, k): g for k, g in zip(leaf, grads)})
    return out


def exact(case, seed):
    st = prepare(case, seed)
    if case["kind"] == "dropout":
        return {"y": _dropped64(st["x"].double(), case["p"], st["draws"]), "dx": _dropped64(st["dy"].double(), case["p"], st["draws"])}
    with torch.enable_grad():
        return _exact_norm(st) if case["kind"] == "norm" else _exact_linear(st)
