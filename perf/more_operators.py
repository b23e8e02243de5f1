"""The 8-bit layer products and the mixture-of-experts layer that the
performance work measures.

A case is one call on p ranks:

  quantize     s_i = max |x_i| / 127, q = x / s rounded to whole numbers
  linear_int8  y = act(sx_i sw_j (x w^T)_ij + bias_j) + residual
  gated_int8   h = act(sx sg (x wg^T) + bg) * (sx su (x wu^T) + bu)
  moe          the `top` experts of every token by their logits, their weights
               by softmax or sigmoid, and
               y = sum of weight wd_e (act(wg_e x) * (wu_e x)) + residual

`shared`: all ranks read the same x; `pad`: rows of x and of the result lie
this many elements further apart than packed.  moe: `experts` are split over
the ranks, every rank sums those of its own; `masked`: a quarter of the logits
are -inf, and of every eighth token all; `given`: the choice is an input.
"""

import math

import torch

own = False

_TORCH = {"bfloat16": torch.bfloat16, "float16": torch.float16,
          "float32": torch.float32, "int8": torch.int8}
_SIZE = {"bfloat16": 2, "float16": 2, "float32": 4, "int8": 1}


def _quantize(name, p, rows, cols, dtype="bfloat16", pad=0):
    c = {"op": "quantize", "p": p, "rows": rows, "cols": cols, "dtype": dtype,
         "pad": pad}
    return {"name": name, **c} if name else c


def _product(name, op, p, rows, n_in, n_out, out="bfloat16", act="none",
             bias=False, residual=False, shared=False, pad=0):
    c = {"op": op, "p": p, "rows": rows, "n_in": n_in, "n_out": n_out,
         "out": out, "act": act, "bias": bias, "residual": residual,
         "shared": shared, "pad": pad}
    return {"name": name, **c} if name else c


def _moe(name, p, tokens, n_in, hidden, experts, top, dtype="bfloat16",
         weights=None, out=None, act="silu", route="softmax", normalize=True,
         residual=False, masked=False, given=False, pad=0):
    c = {"op": "moe", "p": p, "tokens": tokens, "n_in": n_in,
         "hidden": hidden, "experts": experts, "top": top, "dtype": dtype,
         "weights": weights or dtype, "out": out or dtype, "act": act,
         "route": route, "normalize": normalize, "residual": residual,
         "masked": masked, "given": given, "pad": pad}
    return {"name": name, **c} if name else c


def listed():
    return [
        # one token's activations before an 8-bit product: latency
        _quantize("quantize_1row", 1, 1, 4096),
        # a long prompt's activations, or a layer's weights once, one scale a
        # channel: a stream through memory
        _quantize("quantize_8192rows", 1, 8192, 4096),
        # one token through a projection with bias and residual: one read of
        # the weights, half of what 16 bits read
        _product("int8_1row", "linear_int8", 1, 1, 4096, 4096, bias=True,
                 residual=True),
        # ragged: odd contraction, packed, so every row starts at another
        # alignment; 7 ranks and a row count of the paper's Table 2
        _product("int8_ragged_p7", "linear_int8", 7, 875, 1001, 1000,
                 "float16", act="gelu", bias=True),
        # a long prompt's wide projection
        _product("int8_8192rows", "linear_int8", 1, 8192, 4096, 16384,
                 act="gelu_tanh", bias=True),
        # a serving batch through the gated projections of a layer split over
        # 8 ranks
        _product("gated_int8_16rows_p8", "gated_int8", 8, 16, 4096, 2048,
                 act="silu", shared=True),
        # a prompt through the same layer
        _product("gated_int8_4096rows_p8", "gated_int8", 8, 4096, 4096, 2048,
                 act="silu", shared=True),
        # one token through 8 of 64 experts: a serving step's latency
        _moe("moe_1token", 1, 1, 2048, 1024, 64, 8, residual=True),
        # a small batch, experts split over 8 ranks, 32-bit partial sums for
        # the reduction; masked experts and padded tokens
        _moe("moe_16tokens_p8", 8, 16, 2048, 1024, 64, 8, out="float32",
             route="sigmoid", masked=True),
        # a batch through a few wide experts with 8-bit weights: all of them
        # are read
        _moe("moe_64tokens_int8", 1, 64, 4096, 8192, 8, 2, weights="int8"),
        # ragged: odd widths off 16 bytes, an odd number of experts
        _moe("moe_ragged", 1, 33, 1001, 501, 20, 3, "float16", act="gelu",
             normalize=False),
        # a larger batch with the choice made elsewhere
        _moe("moe_100tokens_given", 1, 100, 2048, 1024, 64, 4, given=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def draw(rng):
    while True:
        op = rng.choice(["quantize", "linear_int8", "linear_int8",
                         "gated_int8", "moe", "moe", "moe"])
        p = rng.choice([1, 1, 2, 4, 7, 8, 8, 36])
        pad = rng.choice([0, 0, 0, 64, 5])
        if op == "quantize":
            c = _quantize(None, p, _log_int(rng, 1, 8192),
                          _log_int(rng, 64, 16384),
                          rng.choice(["bfloat16", "float16", "float32"]), pad)
        elif op == "moe":
            p = rng.choice([1, 1, 1, 2, 4, 8])
            n_in, hidden = _log_int(rng, 256, 8192), _log_int(rng, 128, 8192)
            if rng.random() < 0.7:
                n_in, hidden = -(-n_in // 64) * 64, -(-hidden // 64) * 64
            experts = p * rng.choice([1, 2, 4, 5, 8, 16, 32])
            dtype = rng.choice(["bfloat16", "bfloat16", "bfloat16", "float16",
                                "float32"])
            c = _moe(None, p, _log_int(rng, 1, 128), n_in, hidden, experts,
                     rng.randint(1, min(8, experts)), dtype,
                     "int8" if dtype != "float32" and rng.random() < 0.4
                     else dtype, rng.choice([dtype, dtype, "float32"]),
                     rng.choice(["silu", "gelu", "gelu_tanh", "relu"]),
                     rng.choice(["softmax", "sigmoid"]), rng.random() < 0.7,
                     rng.random() < 0.3,
                     experts >= 4 and rng.random() < 0.3,
                     rng.random() < 0.2, pad)
        else:
            n_in, n_out = _log_int(rng, 64, 16384), _log_int(rng, 64, 16384)
            if rng.random() < 0.6:
                n_in, n_out = -(-n_in // 64) * 64, -(-n_out // 64) * 64
            gate = op == "gated_int8"
            act = rng.choice(["silu", "gelu", "gelu_tanh", "relu"])
            if not gate and rng.random() < 0.4:
                act = "none"
            c = _product(None, op, p, _log_int(rng, 1, 8192), n_in, n_out,
                         rng.choice(["bfloat16", "bfloat16", "float16",
                                     "float32"]), act, rng.random() < 0.5,
                         not gate and rng.random() < 0.3, rng.random() < 0.5,
                         pad)
        # no dearer than the largest listed calls
        w = work(c)
        if w["flops"] <= 1.0e12 and w["bytes"] <= (
                8e8 if op == "moe" else 3e8):
            return c


# ------------------------------------------------------------------ inputs

def _normal(g, *shape, scale=1.0, far=0, dtype=torch.float32):
    t = torch.randn(*shape[:-1], shape[-1] + far, generator=g, device="cuda",
                    dtype=torch.float32)
    return t.mul_(scale).to(dtype)[..., :shape[-1]]


def _codes(g, *shape, far=0):
    """N(0, 1) values as a quantisation leaves them, a step of 1 / 32."""
    t = torch.randn(*shape[:-1], shape[-1] + far, generator=g, device="cuda",
                    dtype=torch.float32)
    return t.mul_(32).round_().clamp_(-127, 127).to(
        torch.int8)[..., :shape[-1]]


def _scales(g, *shape, scale=1.0):
    t = torch.rand(*shape, generator=g, device="cuda", dtype=torch.float32)
    return (t + 0.5) * (scale / 32)


def _inputs(c, seed):
    """Activations and residuals N(0, 1), weights N(0, 1) / sqrt(their
    contraction), logits N(0, 1) * 2."""
    g = torch.Generator("cuda").manual_seed(seed)
    s = {"case": c}
    p, pad = c["p"], c["pad"]
    if c["op"] == "quantize":
        s["x"] = _normal(g, p, c["rows"], c["cols"], far=pad,
                         dtype=_TORCH[c["dtype"]])
        # rows of different sizes
        s["x"] *= torch.exp(_normal(g, p, c["rows"], 1)).to(s["x"].dtype)
        return s
    out = _TORCH[c["out"]]
    if c["op"] != "moe":
        rows, n_in, n_out = c["rows"], c["n_in"], c["n_out"]
        n = 1 if c["shared"] else p
        s["x"], s["sx"] = _codes(g, n, rows, n_in, far=pad), \
            _scales(g, n, rows)
        for k in ("gu" if c["op"] == "gated_int8" else "z"):
            s["w" + k] = _codes(g, p, n_out, n_in)
            s["s" + k] = _scales(g, p, n_out, scale=n_in ** -0.5)
            s["b" + k] = _normal(g, p, n_out, scale=0.5, dtype=out) \
                if c["bias"] else None
        if c["residual"]:
            s["r"] = _normal(g, p, rows, n_out, dtype=out)
        return s
    tokens, n_in, hidden, experts = (c[k] for k in ("tokens", "n_in",
                                                    "hidden", "experts"))
    dt, codes = _TORCH[c["dtype"]], c["weights"] == "int8"
    s["x"] = _normal(g, tokens, n_in, far=pad, dtype=dt)
    for k, shape in (("g", (hidden, n_in)), ("u", (hidden, n_in)),
                     ("d", (n_in, hidden))):
        if codes:
            s["w" + k] = _codes(g, experts, *shape)
            s["s" + k] = _scales(g, experts, shape[0], scale=shape[1] ** -0.5)
        else:
            s["w" + k] = _normal(g, experts, *shape, scale=shape[1] ** -0.5,
                                 dtype=dt)
    logits = _normal(g, tokens, experts, scale=2.0)
    if c["masked"]:
        hide = torch.rand(tokens, experts, generator=g, device="cuda") < 0.25
        hide[7::8] = True
        logits = logits.masked_fill(hide, -math.inf)
    if c["given"]:
        w, s["index"] = _choice(c, logits)
        s["weight"] = w.float()
    else:
        s["logits"] = logits
    if c["residual"]:
        s["r"] = _normal(g, p, tokens, n_in, dtype=out)
    return s


def _handle(s):
    """What a program keeps beside its tensors: result buffers, the arrays of
    addresses, the options and the workspace."""
    from paper_2109_12626_amd import dpar

    c = s["case"]
    p, pad = c["p"], c["pad"]

    def made(*shape, dtype, far=0):
        t = torch.empty(*shape[:-1], shape[-1] + far, dtype=dtype,
                        device="cuda")
        return t[..., :shape[-1]]

    def ranks(t):
        if t is None:
            return None
        if t.shape[0] != p or t.dim() < 2:
            return dpar.pointers([t.data_ptr()] * p)
        return dpar.rows(t)

    r = s["result"] = {}
    if c["op"] == "quantize":
        rows, cols = c["rows"], c["cols"]
        r["q"] = made(p, rows, cols, dtype=torch.int8, far=pad)
        r["scale"] = made(p, rows, dtype=torch.float32)
        opt = dpar.quantize_options(rows, cols, c["dtype"], ldx=cols + pad,
                                    ldq=cols + pad)
        s["call"] = dpar.dpar_quantize
        s["args"] = [ranks(s["x"]), ranks(r["q"]), ranks(r["scale"]), p, opt]
        return
    out = _TORCH[c["out"]]
    if c["op"] != "moe":
        rows, n_in, n_out = c["rows"], c["n_in"], c["n_out"]
        gate = c["op"] == "gated_int8"
        r["y"] = made(p, rows, n_out, dtype=out, far=pad)
        opt = dpar.product_options(rows, n_in, n_out, "int8", c["out"],
                                   c["act"], ldx=n_in + pad, ldy=n_out + pad)
        n = dpar.dpar_product_workspace("gated" if gate else "linear", p, opt)
        args = [s["x"], s["sx"]]
        args += [s["wg"], s["sg"], s["wu"], s["su"], s["bg"], s["bu"]] \
            if gate else [s["wz"], s["sz"], s["bz"], s.get("r")]
        s["call"] = getattr(dpar, "dpar_" + c["op"])
        args = [ranks(t) for t in args + [r["y"]]]
    else:
        tokens, n_in, top = c["tokens"], c["n_in"], c["top"]
        r["y"] = made(p, tokens, n_in, dtype=out, far=pad)
        if not c["given"]:
            r["index"] = made(tokens, top, dtype=torch.int32)
            r["weight"] = made(tokens, top, dtype=torch.float32)
        opt = dpar.moe_options(tokens, n_in, c["hidden"], c["experts"] // p,
                               top, c["dtype"], c["weights"], c["out"],
                               c["act"], c["route"], c["normalize"],
                               ldx=n_in + pad, ldy=n_in + pad)
        n = dpar.dpar_moe_workspace(p, opt)

        def every(t):
            return None if t is None else dpar.pointers([t.data_ptr()] * p)

        def split(k):
            t = s.get(k)
            return None if t is None else dpar.rows(
                t.view(p, -1, *t.shape[1:]))

        def first(k):        # the ranks choose alike: the first one's choice
            if c["given"]:
                return every(s[k])
            return dpar.pointers([r[k].data_ptr()] + [0] * (p - 1))

        s["call"] = dpar.dpar_moe
        args = [every(s["x"]), every(s.get("logits"))] \
            + [split(k) for k in ("wg", "wu", "wd", "sg", "su", "sd")] \
            + [ranks(s.get("r")), ranks(r["y"]), first("index"),
               first("weight")]
    ws = torch.empty(n, dtype=torch.uint8, device="cuda") if n else None
    s["args"] = args + [p, opt, ws, n]


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:
        _handle(s)
    return s


# -------------------------------------------------------------- plain forms

def _act(z, act):
    if act == "relu":
        return torch.clamp_min(z, 0)
    if act == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    if act == "gelu_tanh":
        t = torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z * z * z))
        return 0.5 * z * (1 + t)
    if act == "silu":
        return z * torch.sigmoid(z)
    return z


def _choice(c, logits):
    """Weights (fp32) and numbers of the chosen experts, -1 for none."""
    top = c["top"]
    order = torch.sort(logits, dim=1, descending=True, stable=True)
    best, index = order.values[:, :top], order.indices[:, :top]
    if c["route"] == "softmax":
        # (a token without experts has no largest logit)
        far = best[:, :1].clamp_min(-1e30)
        w = torch.exp(best - far)
        total = w if c["normalize"] else torch.exp(logits - far)
        w = w / total.sum(1, keepdim=True)
    else:
        w = torch.sigmoid(best)
        if c["normalize"]:
            w = w / w.sum(1, keepdim=True)
    none = best == -math.inf
    return w.masked_fill(none, 0.0), index.masked_fill(none, -1).int()


def _plain_moe(s):
    c = s["case"]
    p, tokens, top, experts = (c[k] for k in ("p", "tokens", "top",
                                              "experts"))
    weight, index = (s["weight"], s["index"]) if c["given"] \
        else _choice(c, s["logits"])
    x = s["x"].float()
    at = index.clamp_min(0).long()

    def matrix(k, pick):
        w = s["w" + k]
        w = (w if pick is None else w[pick]).float()
        if c["weights"] == "int8":
            sc = s["s" + k]
            w = w * (sc if pick is None else sc[pick])[..., None]
        return w.transpose(1, 2)

    # each chosen expert's matrices, or all experts' where those are fewer
    pick = at.reshape(-1) if tokens * top < experts else None
    rows = x.repeat_interleave(top, 0)[:, None] if pick is not None else x
    g = torch.matmul(rows, matrix("g", pick))
    u = torch.matmul(rows, matrix("u", pick))
    o = torch.matmul(_act(g, c["act"]) * u, matrix("d", pick))
    if pick is not None:
        o = o.view(tokens, top, -1)
    else:
        o = o.transpose(0, 1).gather(
            1, at[..., None].expand(-1, -1, o.shape[-1]))
    o = o * weight[..., None]
    rank = index.div(experts // p, rounding_mode="floor")
    mine = rank[None] == torch.arange(p, device=rank.device)[:, None, None]
    y = (o * mine[..., None]).sum(2)
    if c["residual"]:
        y = y + s["r"].float()
    r = {"y": y.to(_TORCH[c["out"]])}
    if not c["given"]:
        r["index"], r["weight"] = index, weight
    return r


def run(s):
    if own:
        s["call"](*s["args"], torch.cuda.current_stream())
        return s["result"]
    c = s["case"]
    if c["op"] == "moe":
        return _plain_moe(s)
    if c["op"] == "quantize":
        x = s["x"].float()
        scale = (x.abs().amax(-1).double() / 127).float()
        # in 64 bits: quotients next to a half
        q = torch.round(x.double() / scale.double()[..., None])
        return {"q": q.clamp(-127, 127).to(torch.int8), "scale": scale}
    x, out = s["x"].float(), _TORCH[c["out"]]

    def product(k):
        z = torch.matmul(x, s["w" + k].float().transpose(1, 2))
        z = z * s["sx"][..., None] * s["s" + k][:, None]
        return z + s["b" + k].float()[:, None] if c["bias"] else z

    if c["op"] == "gated_int8":
        y = _act(product("g"), c["act"]) * product("u")
    else:
        y = _act(product("z"), c["act"])
        if c["residual"]:
            y = y + s["r"].float()
    return {"y": y.to(out)}


# ------------------------------------------------------------------- exact

def _value(z, act):
    if act == "none":
        return z
    if act == "relu":
        return torch.where(z > 0, z, 0.0)
    if act == "gelu":
        return z * 0.5 * torch.special.erfc(-z / math.sqrt(2))
    k = 1.0 if act == "silu" else 2 * math.sqrt(2 / math.pi)
    a = z if act == "silu" else z + 0.044715 * z ** 3
    return z / (1 + torch.exp(-k * a))


def _exact_moe(s):
    """Expert after expert, with the tokens that chose it."""
    c = s["case"]
    p, tokens, top, experts = (c[k] for k in ("p", "tokens", "top",
                                              "experts"))
    if c["given"]:
        index, weight = s["index"], s["weight"].double()
    else:
        l = s["logits"].double().cpu()
        index = torch.full((tokens, top), -1, dtype=torch.int32)
        weight = torch.zeros(tokens, top, dtype=torch.float64)
        for t in range(tokens):
            v = l[t].tolist()
            best = sorted((e for e in range(experts) if v[e] > -math.inf),
                          key=lambda e: (-v[e], e))[:top]
            if not best:
                continue
            if c["route"] == "softmax":
                a = [math.exp(v[e] - v[best[0]]) for e in best]
                total = sum(a) if c["normalize"] else sum(
                    math.exp(z - v[best[0]]) for z in v)
            else:
                a = [1 / (1 + math.exp(-v[e])) for e in best]
                total = sum(a) if c["normalize"] else 1.0
            index[t, :len(best)] = torch.tensor(best, dtype=torch.int32)
            weight[t, :len(best)] = torch.tensor(
                [z / total for z in a], dtype=torch.float64)
        index, weight = index.cuda(), weight.cuda()
    x = s["x"].double()
    y = s["r"].double() if c["residual"] else torch.zeros(
        p, tokens, c["n_in"], dtype=torch.float64, device="cuda")

    def matrix(k, e):
        w = s["w" + k][e].double()
        if c["weights"] == "int8":
            w = w * s["s" + k][e].double()[:, None]
        return w.t()

    for e in range(experts):
        t, slot = torch.nonzero(index == e, as_tuple=True)
        if not len(t):
            continue
        h = _value(torch.mm(x[t], matrix("g", e)), c["act"]) \
            * torch.mm(x[t], matrix("u", e))
        y[e * p // experts].index_add_(
            0, t, torch.mm(h, matrix("d", e)) * weight[t, slot][:, None])
    return {"y": y} if c["given"] else {"y": y, "index": index,
                                        "weight": weight}


def exact(case, seed):
    s = _inputs(case, seed)
    if case["op"] == "moe":
        return _exact_moe(s)
    if case["op"] == "quantize":
        x = s["x"].double()
        scale = (x.abs().max(-1).values / 127).float()
        step = scale.double()[..., None]
        # the nearest whole number, halves to the even one
        low = torch.floor(x / step)
        far = x / step - low
        up = (far > 0.5) | ((far == 0.5) & (low.remainder(2) == 1))
        return {"q": (low + up).clamp(-127, 127).to(torch.int8),
                "scale": scale}
    parts = []
    for i in range(case["p"]):
        j = 0 if case["shared"] else i
        x = s["x"][j].double() * s["sx"][j].double()[:, None]

        def affine(k):
            w = s["w" + k][i].double() * s["s" + k][i].double()[:, None]
            z = torch.mm(x, w.t())
            return z + s["b" + k][i].double() if case["bias"] else z

        if case["op"] == "gated_int8":
            y = _value(affine("g"), case["act"]) * affine("u")
        else:
            y = _value(affine("z"), case["act"])
            if case["residual"]:
                y = y + s["r"][i].double()
        parts.append(y)
    return {"y": torch.stack(parts)}


def work(case):
    p = case["p"]
    if case["op"] == "quantize":
        n = p * case["rows"] * case["cols"]
        return {"bytes": n * (_SIZE[case["dtype"]] + 1.0)
                + 4.0 * p * case["rows"], "flops": 3.0 * n}
    eo = _SIZE[case["out"]]
    if case["op"] == "moe":
        tokens, n_in, hidden, experts, top = (
            case[k] for k in ("tokens", "n_in", "hidden", "experts", "top"))
        # tokens that choose, logits they choose among
        real = tokens - (tokens // 8 if case["masked"] else 0)
        # experts that some token chooses, on the average
        met = experts * (1 - (1 - top / experts) ** real)
        ew, e = _SIZE[case["weights"]], _SIZE[case["dtype"]]
        weights = met * 3.0 * hidden * n_in * ew
        if case["weights"] == "int8":
            weights += met * 4.0 * (2 * hidden + n_in)
        choice = tokens * top * 8.0 + (0 if case["given"]
                                       else tokens * experts * 4.0)
        rows = tokens * n_in * (e + p * eo * (2 if case["residual"] else 1))
        return {"bytes": weights + choice + rows,
                "flops": 6.0 * real * top * hidden * n_in}
    rows, n_in, n_out = case["rows"], case["n_in"], case["n_out"]
    n = 2 if case["op"] == "gated_int8" else 1
    read = (1 if case["shared"] else p) * rows * (n_in + 4.0) \
        + p * n * n_out * (n_in + 4.0)
    read += p * n * n_out * eo if case["bias"] else 0
    read += p * rows * n_out * eo if case["residual"] else 0
    return {"bytes": read + p * rows * n_out * eo,
            "flops": 2.0 * p * n * rows * n_in * n_out}
