"""The layer products that the performance work measures: the calls that make
the rows which reduction-to-all sums when a layer is split over p ranks.

A case is one call on p ranks, each with `rows` rows of `n_in` values and
weights of `n_out` x `n_in`:

  linear           y = act(x w^T + bias) + residual
  linear_backward  dz = dy act'(z); dx = dz w, dw = dz^T x, dbias = sum dz
  gated            h = act(x wg^T + bg) * (x wu^T + bu)
  gated_backward   dg = dh u act'(g), du = dh act(g); dx = dg wg + du wu,
                   dwg = dg^T x, dwu = du^T x, dbg = sum dg, dbu = sum du

`shared`: all ranks read the same x (weights split by columns); `pad`: rows of
x and of the result lie this many elements further apart than packed.
"""

import math

import torch

own = False

_TORCH = {"bfloat16": torch.bfloat16, "float16": torch.float16,
          "float32": torch.float32}
_SIZE = {"bfloat16": 2, "float16": 2, "float32": 4}


def _case(name, op, p, rows, n_in, n_out, dtype="bfloat16", out=None,
          act="none", bias=False, residual=False, save=False, shared=False,
          pad=0):
    c = {"op": op, "p": p, "rows": rows, "n_in": n_in, "n_out": n_out,
         "dtype": dtype, "out": out or dtype, "act": act, "bias": bias,
         "residual": residual, "save": save, "shared": shared, "pad": pad}
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # one token through a projection with bias and residual: the smallest
        # call of a serving step, latency and one read of the weights
        _case("linear_1row", "linear", 1, 1, 4096, 4096, bias=True,
              residual=True),
        # 16 tokens through the second projection of a layer split over 8
        # ranks: fp32 partial sums, the rows of a reduction with m = 2^16
        _case("linear_16rows_p8", "linear", 8, 16, 2048, 4096,
              out="float32"),
        # ragged: odd contraction, packed, so every row starts at another
        # alignment; 7 ranks and a row count of the paper's Table 2
        _case("linear_ragged_p7", "linear", 7, 875, 1001, 1000, "float16",
              act="gelu", bias=True),
        # 32-bit layers: 256 tokens on 8 ranks, rows of 2^20 for the reduction
        _case("linear_f32_p8", "linear", 8, 256, 1024, 4096, "float32",
              bias=True),
        # a training step's or a long prompt's wide projection, one rank; the
        # value before the activation is kept for the backward pass
        _case("linear_8192rows", "linear", 1, 8192, 4096, 16384,
              act="gelu_tanh", bias=True, save=True),
        # training: all gradients of a square layer (2^24 values, the size of
        # the data-parallel reduction)
        _case("linear_bwd_4096rows", "linear_backward", 1, 4096, 4096, 4096,
              act="gelu", bias=True),
        # training of small 32-bit layers on 4 ranks with odd widths
        _case("linear_bwd_f32_ragged", "linear_backward", 4, 875, 500, 999,
              "float32", act="relu", bias=True),
        # one token through the gated projections of a layer split over 8
        # ranks: one read of all weights
        _case("gated_1row_p8", "gated", 8, 1, 4096, 2048, act="silu",
              shared=True),
        # a serving batch between the single token and the prompt
        _case("gated_48rows", "gated", 1, 48, 4096, 8192, "float16",
              act="silu"),
        # a prompt or training step, forward, 8 ranks, both projections kept
        _case("gated_4096rows_p8", "gated", 8, 4096, 4096, 2048, act="silu",
              save=True, shared=True),
        # the same layer's backward pass on half the rows
        _case("gated_bwd_2048rows_p8", "gated_backward", 8, 2048, 4096, 2048,
              act="silu", shared=True),
        # ragged training: odd widths, a row count just past a tile
        _case("gated_bwd_ragged", "gated_backward", 2, 129, 1000, 1363,
              "float16", act="gelu", bias=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def draw(rng):
    while True:
        op = rng.choice(["linear", "linear", "linear_backward", "gated",
                         "gated_backward"])
        dtype = rng.choice(["bfloat16", "bfloat16", "bfloat16", "float16",
                            "float32"])
        p = rng.choice([1, 1, 2, 4, 7, 8, 8, 36])
        rows = _log_int(rng, 1, 8192)
        n_in, n_out = _log_int(rng, 64, 16384), _log_int(rng, 64, 16384)
        if rng.random() < 0.6:       # widths of layers; else any, odd too
            n_in, n_out = -(-n_in // 64) * 64, -(-n_out // 64) * 64
        if 3072 in (rows, n_in, n_out):     # no layer here is that wide
            continue
        back, gate = op.endswith("backward"), op.startswith("gated")
        act = rng.choice(["silu", "gelu", "gelu_tanh", "relu"])
        if not gate and rng.random() < 0.4:
            act = "none"
        c = _case(None, op, p, rows, n_in, n_out, dtype, act=act,
                  out="float32" if op == "linear" and rng.random() < 0.3
                  else dtype, bias=rng.random() < 0.5,
                  residual=op == "linear" and rng.random() < 0.3,
                  save=not back and act != "none" and rng.random() < 0.4,
                  shared=rng.random() < 0.5,
                  pad=rng.choice([0, 0, 0, 64, 5]))
        w = work(c)
        # no dearer than the largest listed call, at the slower rate of 32
        # bits too
        most = 5e10 if dtype == "float32" else 1.0e12
        if w["flops"] <= most and w["bytes"] <= 3.5e8:
            return c


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


def _act_grad(z, act):
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "gelu":
        return 0.5 * (1 + torch.erf(z * math.sqrt(0.5))) \
            + z * torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)
    if act == "gelu_tanh":
        c = math.sqrt(2 / math.pi)
        t = torch.tanh(c * (z + 0.044715 * z * z * z))
        return 0.5 * (1 + t) \
            + 0.5 * z * (1 - t * t) * c * (1 + 3 * 0.044715 * z * z)
    if act == "silu":
        s = torch.sigmoid(z)
        return s * (1 + z * (1 - s))
    return torch.ones_like(z)


def _inputs(case, seed):
    """The call's inputs: activations and gradients N(0, 1), weights N(0, 1) /
    sqrt(n_in), and for a backward pass the kept values of its forward one."""
    g = torch.Generator("cuda").manual_seed(seed)
    dt = _TORCH[case["dtype"]]
    p, rows, n_in, n_out = (case[k] for k in ("p", "rows", "n_in", "n_out"))
    pad = case["pad"]

    def normal(*shape, scale=1.0, far=0):
        t = torch.randn(*shape[:-1], shape[-1] + far, generator=g,
                        device="cuda", dtype=torch.float32)
        return (t * scale).to(dt)[..., :shape[-1]]

    s = {"case": case}
    s["x"] = normal(1 if case["shared"] else p, rows, n_in, far=pad)
    gate, back = case["op"].startswith("gated"), \
        case["op"].endswith("backward")
    for k in (("g", "u") if gate else ("z",)):
        s["w" + k] = normal(p, n_out, n_in, scale=n_in ** -0.5)
        s["b" + k] = normal(p, n_out, scale=0.5) if case["bias"] else None
        if back:
            z = torch.matmul(s["x"].float(),
                             s["w" + k].float().transpose(1, 2))
            if case["bias"]:
                z += s["b" + k].float()[:, None]
            s[k] = z.to(dt)
    if back:
        s["dy"] = normal(p, rows, n_out, far=pad)
    if case["residual"]:
        g.manual_seed(seed + 1)
        r = torch.randn(p, rows, n_out, generator=g, device="cuda")
        s["r"] = r.to(_TORCH[case["out"]])
    return s


def _handle(s):
    """What a program keeps beside its tensors: result buffers, the arrays of
    row addresses, the options and the workspace."""
    from paper_2109_12626_amd import dpar

    c = s["case"]
    dt, out = _TORCH[c["dtype"]], _TORCH[c["out"]]
    p, rows, n_in, n_out, pad = (c[k] for k in ("p", "rows", "n_in", "n_out",
                                                "pad"))

    def made(*shape, dtype=out, far=0):
        t = torch.empty(*shape[:-1], shape[-1] + far, dtype=dtype,
                        device="cuda")
        return t[..., :shape[-1]]

    def ranks(t):
        if t is None:
            return None
        if t.shape[0] != p:         # one x for all ranks
            return dpar.pointers([t.data_ptr()] * p)
        return dpar.rows(t)

    gate, back = c["op"].startswith("gated"), c["op"].endswith("backward")
    kept = ("g", "u") if gate else ("z",)
    opt = dpar.product_options(rows, n_in, n_out, c["dtype"], c["out"],
                               c["act"], ldx=n_in + pad, ldy=n_out + pad)
    bytes_ = dpar.dpar_product_workspace(c["op"], p, opt)
    ws = torch.empty(bytes_, dtype=torch.uint8, device="cuda") \
        if bytes_ else None
    r = {}
    args = []
    if back:
        args = [s["dy"], s["x"]] + [s["w" + k] for k in kept] \
            + [s[k] for k in kept]
        r["dx"] = made(p, rows, n_in)
        for k in kept:
            r["dw" + k] = made(p, n_out, n_in)
        for k in kept:
            r["db" + k] = made(p, n_out) if c["bias"] else None
        args += list(r.values())
        args += [made(p, rows, n_out, dtype=dt)
                 if gate or c["act"] != "none" else None for k in kept]
    else:
        args = [s["x"]] + [s["w" + k] for k in kept] \
            + [s["b" + k] for k in kept]
        if not gate:
            args.append(s.get("r"))
        r["y"] = made(p, rows, n_out, far=pad)
        for k in kept:
            r[k] = made(p, rows, n_out, dtype=dt) if c["save"] else None
        args += list(r.values())
    s["keep"] = args
    s["call"] = getattr(dpar, "dpar_" + c["op"])
    s["args"] = [ranks(t) for t in args] + [p, opt, ws, bytes_]
    s["result"] = {k: v for k, v in r.items() if v is not None}


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:
        _handle(s)
    return s


def run(s):
    if own:
        s["call"](*s["args"], torch.cuda.current_stream())
        return s["result"]
    c = s["case"]
    dt, out, act = _TORCH[c["dtype"]], _TORCH[c["out"]], c["act"]
    x = s["x"].float()

    def product(k):
        z = torch.matmul(x, s["w" + k].float().transpose(1, 2))
        return z + s["b" + k].float()[:, None] if c["bias"] else z

    if c["op"] == "linear":
        z = product("z")
        y = _act(z, act)
        if c["residual"]:
            y = y + s["r"].float()
        r = {"y": y.to(out)}
        if c["save"]:
            r["z"] = z.to(dt)
        return r
    if c["op"] == "gated":
        g, u = product("g"), product("u")
        r = {"y": (_act(g, act) * u).to(out)}
        if c["save"]:
            r["g"], r["u"] = g.to(dt), u.to(dt)
        return r
    dy = s["dy"].float()
    if c["op"] == "linear_backward":
        dz = dy * _act_grad(s["z"].float(), act)
        r = {"dx": torch.matmul(dz, s["wz"].float()).to(out),
             "dwz": torch.matmul(dz.transpose(1, 2), x).to(out)}
        if c["bias"]:
            r["dbz"] = dz.sum(1).to(out)
        return r
    g = s["g"].float()
    dg, du = dy * s["u"].float() * _act_grad(g, act), dy * _act(g, act)
    r = {"dx": (torch.matmul(dg, s["wg"].float())
                + torch.matmul(du, s["wu"].float())).to(out),
         "dwg": torch.matmul(dg.transpose(1, 2), x).to(out),
         "dwu": torch.matmul(du.transpose(1, 2), x).to(out)}
    if c["bias"]:
        r["dbg"], r["dbu"] = dg.sum(1).to(out), du.sum(1).to(out)
    return r


def exact(case, seed):
    """The definition in 64 bits, one rank after the other."""
    s = _inputs(case, seed)
    act = case["act"]
    phi = lambda z: 0.5 * torch.special.erfc(-z / math.sqrt(2))  # noqa: E731

    def value_and_slope(z):
        if act == "none":
            return z, torch.ones_like(z)
        if act == "relu":
            return torch.where(z > 0, z, 0.0), torch.where(z > 0, 1.0, 0.0)
        if act == "gelu":
            return z * phi(z), phi(z) + z * torch.exp(-z * z / 2) \
                / math.sqrt(2 * math.pi)
        if act == "silu":
            e = 1 / (1 + torch.exp(-z))
            return z * e, e + z * e * (1 - e)
        # 0.5 (1 + tanh a) = 1 / (1 + exp(-2 a))
        k = 2 * math.sqrt(2 / math.pi)
        e = 1 / (1 + torch.exp(-k * (z + 0.044715 * z ** 3)))
        return z * e, e + z * e * (1 - e) * k * (1 + 0.134145 * z ** 2)

    parts = []
    for i in range(case["p"]):
        x = s["x"][0 if case["shared"] else i].double()
        d = {k: s[k][i].double() for k in
             ("wz", "wg", "wu", "bz", "bg", "bu", "z", "g", "u", "dy", "r")
             if s.get(k) is not None}

        def affine(k):
            return torch.mm(x, d["w" + k].t()) + d.get("b" + k, 0.0)

        o = {}
        if case["op"] == "linear":
            z = affine("z")
            o["y"] = value_and_slope(z)[0] + d.get("r", 0.0)
            if case["save"]:
                o["z"] = z
        elif case["op"] == "gated":
            g, u = affine("g"), affine("u")
            o["y"] = value_and_slope(g)[0] * u
            if case["save"]:
                o["g"], o["u"] = g, u
        else:
            if case["op"] == "linear_backward":
                back = {"z": d["dy"] * value_and_slope(d["z"])[1]}
            else:
                a, da = value_and_slope(d["g"])
                back = {"g": d["dy"] * d["u"] * da, "u": d["dy"] * a}
            o["dx"] = sum(torch.mm(t, d["w" + k]) for k, t in back.items())
            for k, t in back.items():
                o["dw" + k] = torch.mm(t.t(), x)
                if case["bias"]:
                    o["db" + k] = t.sum(0)
        parts.append(o)
    return {k: torch.stack([o[k] for o in parts]) for k in parts[0]}


def work(case):
    p, rows, n_in, n_out = (case[k] for k in ("p", "rows", "n_in", "n_out"))
    e, eo = _SIZE[case["dtype"]], _SIZE[case["out"]]
    gate, back = case["op"].startswith("gated"), \
        case["op"].endswith("backward")
    n = 2 if gate else 1             # projections
    x, w, y = rows * n_in, n * n_out * n_in, rows * n_out
    bias = n * p * n_out if case["bias"] else 0
    read = (1 if case["shared"] else p) * x * e + p * w * e
    if back:
        z = n * y if gate or case["act"] != "none" else 0
        read += p * (y + z) * e
        return {"bytes": read + p * (x + w) * eo + bias * eo,
                "flops": 4.0 * p * n * rows * n_in * n_out}
    read += bias * e + (p * y * eo if case["residual"] else 0)
    kept = n * p * y * e if case["save"] else 0
    return {"bytes": read + p * y * eo + kept,
            "flops": 2.0 * p * n * rows * n_in * n_out}
