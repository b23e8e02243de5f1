"""The layer products in 64 bits, with what the entry points' roundings may
change: every function returns (value, slack) pairs, slack being the bound on
the difference of a result that sums in 32 bits in any order, rounds what the
header says is rounded and stores in a type of unit roundoff u.

A sum of n products in 32 bits differs from the exact one by at most
(n + 3) 2^-24 times the sum of the products' absolute values (each product and
addition rounded once, bias and residual included).  An activation or slope in
32 bits is taken to be 2^-20 (1 + |z|) off at most: its polynomials, the
exponential and the reciprocal are a few 2^-24 off each.
"""

import math

import numpy as np

U = {"float32": 2.0 ** -24, "bfloat16": 2.0 ** -8, "float16": 2.0 ** -11}
TINY = {"float32": 2.0 ** -126, "bfloat16": 2.0 ** -126,
        "float16": 2.0 ** -24}
_E = 2.0 ** -24
_ACT = 2.0 ** -20
_erf = np.vectorize(math.erf, otypes=[np.float64])


def act(z, name):
    """act(z), act'(z)."""
    with np.errstate(over="ignore", invalid="ignore"):
        if name == "none":
            return z, np.ones_like(z)
        if name == "relu":
            return np.maximum(z, 0.0), np.where(z > 0, 1.0, 0.0)
        if name == "gelu":
            c = 0.5 * (1 + _erf(z / math.sqrt(2)))
            d = np.exp(-z * z / 2) / math.sqrt(2 * math.pi)
            return z * c, c + z * d
        if name == "silu":
            s = 1 / (1 + np.exp(-z))
            return z * s, s * (1 + z * (1 - s))
        a = math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)
        t = np.tanh(a)
        da = math.sqrt(2 / math.pi) * (1 + 3 * 0.044715 * z * z)
        return 0.5 * z * (1 + t), 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * da


def _stored(v, slack, dtype):
    return v, slack + U[dtype] * (np.abs(v) + slack) + TINY[dtype]


def _product(a, b, a_slack=0.0):
    """a b for a [m, n], b [n, k]; a_slack: bound on each |error of a|."""
    size = np.abs(a) @ np.abs(b)
    return a @ b, (a.shape[1] + 3) * _E * size + \
        (a_slack @ np.abs(b) if np.ndim(a_slack) else 0.0)


def linear(x, w, bias, residual, act_name, dtype, out):
    z, e = _product(x, w.T)
    if bias is not None:
        z = z + bias
        e = e + _E * (np.abs(z) + np.abs(bias))
    y, d = act(z, act_name)
    ey = e * 1.13 + (0 if act_name == "none" else _ACT * (1 + np.abs(z)))
    if residual is not None:
        y = y + residual
        ey = ey + _E * np.abs(y)
    return {"y": _stored(y, ey, out), "z": _stored(z, e, dtype)}


def _slope(dy, z, act_name, dtype):
    """dy act'(z), rounded to dtype unless there is no activation."""
    v, d = act(z, act_name)
    dz = dy * d
    if act_name == "none":
        return dz, np.zeros_like(dz)
    return _stored(dz, _ACT * np.abs(dy), dtype)


def _grads(pairs, x, ws, out, dtype):
    dx, ex = 0.0, 0.0
    r = {}
    for (name, dz, e), w in zip(pairs, ws):
        v, s = _product(dz, w, e)
        dx, ex = dx + v, ex + s + _E * (np.abs(v) + s)
        v, s = _product(dz.T, x, e.T)
        r["dw" + name] = _stored(v, s, out)
        r["db" + name] = _stored(dz.sum(0), (dz.shape[0] + 3) * _E *
                                 np.abs(dz).sum(0) + e.sum(0), out)
    r["dx"] = _stored(dx, ex, out)
    return r


def linear_backward(dy, x, w, z, act_name, dtype, out):
    dz, e = _slope(dy, z, act_name, dtype)
    return _grads([("z", dz, e)], x, [w], out, dtype)


def gated(x, wg, wu, bg, bu, act_name, dtype, out):
    g, u = (linear(x, w, b, None, "none", dtype, dtype)["z"] for w, b in
            ((wg, bg), (wu, bu)))
    # (their bounds before they are stored)
    eg, eu = ((e - U[dtype] * np.abs(v) - TINY[dtype]) / (1 + U[dtype])
              for v, e in (g, u))
    a, _ = act(g[0], act_name)
    ea = eg * 1.13 + _ACT * (1 + np.abs(g[0]))
    h = a * u[0]
    eh = ea * np.abs(u[0]) + np.abs(a) * eu + ea * eu + _E * np.abs(h)
    return {"h": _stored(h, eh, out), "g": g, "u": u}


def gated_backward(dh, x, wg, wu, g, u, act_name, dtype, out):
    a, d = act(g, act_name)
    err = _ACT * (1 + np.abs(g)) * np.abs(dh)
    dg = _stored(dh * u * d, err * np.abs(u), dtype)
    du = _stored(dh * a, err, dtype)
    return _grads([("g", *dg), ("u", *du)], x, [wg, wu], out, dtype)


# ------------------------------------------------------------------- 8 bits

def quantize(x):
    """(q, scale) of rows x (float64 of what is stored in 32 bits or fewer):
    exact, the scale rounded to 32 bits."""
    most = np.abs(x).max(axis=1, initial=0.0)
    with np.errstate(invalid="ignore", divide="ignore"):
        scale = (most / 127).astype(np.float32)
        scale[~np.isfinite(most)] = np.nan
        q = np.rint(x / scale.astype(np.float64)[:, None])
    q[~(scale > 0)] = 0
    return np.clip(q, -127, 127), scale


def _scaled(x, sx, w, sw):
    """sx sw (x w^T): the sum is exact; its conversion and the two products are
    rounded once each."""
    z = (x @ w.T) * sx[:, None] * sw[None]
    return z, 3.1 * _E * np.abs(z)


def linear_int8(x, sx, w, sw, bias, residual, act_name, out):
    z, e = _scaled(x, sx, w, sw)
    if bias is not None:
        z = z + bias
        e = e + _E * (np.abs(z) + np.abs(bias))
    y, _ = act(z, act_name)
    ey = e * 1.13 + (0 if act_name == "none" else _ACT * (1 + np.abs(z)))
    if residual is not None:
        y = y + residual
        ey = ey + _E * np.abs(y)
    return _stored(y, ey, out)


def gated_int8(x, sx, wg, sg, wu, su, bg, bu, act_name, out):
    def affine(w, s, b):
        z, e = _scaled(x, sx, w, s)
        return (z, e) if b is None else \
            (z + b, e + _E * (np.abs(z + b) + np.abs(b)))

    (g, eg), (u, eu) = affine(wg, sg, bg), affine(wu, su, bu)
    a, _ = act(g, act_name)
    ea = eg * 1.13 + _ACT * (1 + np.abs(g))
    h = a * u
    return _stored(h, ea * np.abs(u) + np.abs(a) * eu + ea * eu
                   + _E * np.abs(h), out)


# ------------------------------------------------------- mixture of experts

def choice(logits, top, route, normalize, scale=1.0):
    """(index, weight) [tokens, top] of logits in 64 bits."""
    tokens, experts = logits.shape
    index = np.full((tokens, top), -1, dtype=np.int32)
    weight = np.zeros((tokens, top))
    with np.errstate(all="ignore"):
        for t in range(tokens):
            v = logits[t]
            best = sorted((e for e in range(experts) if v[e] != -np.inf),
                          key=lambda e: (not np.isnan(v[e]), -v[e], e))[:top]
            if not best:
                continue
            if route == "softmax":
                a = np.exp(v[best] - v[best[0]])
                w = a / (a if normalize else np.exp(v - v[best[0]])).sum()
            else:
                w = 1 / (1 + np.exp(-v[best]))
                if normalize and w.sum() != 0:
                    w = w / w.sum()
            index[t, :len(best)] = best
            weight[t, :len(best)] = w * scale
    return index, weight


def moe(x, index, weight, wg, wu, wd, scales, residual, act_name, dtype, out,
        first=0, chosen=True):
    """y of the rank that holds experts first .. (wg [experts, hidden, in]);
    scales: of 8-bit weights, (sg, su, sd) or None; chosen: the weights are the
    library's own, a few 2^-24 off."""
    tokens, top = index.shape
    hidden, n_in = wg.shape[1:]
    parts = 6                     # products per hidden value at most
    y, ey = np.zeros((tokens, n_in)), np.zeros((tokens, n_in))
    size = np.zeros((tokens, n_in))
    for e in range(len(wg)):
        t, s = np.nonzero(index == first + e)
        if not len(t):
            continue

        def affine(w, sc):
            z, err = _product(x[t], w[e].T)
            return (z, err) if sc is None else \
                (z * sc[e], (err + _E * np.abs(z)) * np.abs(sc[e]))

        sg, su, sd = scales or (None,) * 3
        (g, eg), (u, eu) = affine(wg, sg), affine(wu, su)
        a, _ = act(g, act_name)
        ea = eg * 1.13 + _ACT * (1 + np.abs(g))
        h = a * u
        eh = ea * np.abs(u) + np.abs(a) * eu + ea * eu + _E * np.abs(h)
        # (held whole, its last part as far as bfloat16 goes)
        eh = eh + TINY["bfloat16"]
        o = h @ wd[e].T
        big = (np.abs(h) + eh) @ np.abs(wd[e].T)
        eo = (parts * hidden + 3) * _E * big + eh @ np.abs(wd[e].T)
        if sd is not None:
            o, big, eo = (v * np.abs(sd[e]) if v is not o else v * sd[e]
                          for v in (o, big, eo))
        w = weight[t, s][:, None]
        np.add.at(y, t, w * o)
        np.add.at(size, t, np.abs(w) * big)
        np.add.at(ey, t, np.abs(w) * (eo + (_ACT if chosen else 0)
                                      * (np.abs(o) + eo)))
    # each expert's part in up to 8 pieces, times two factors
    ey += (9 * top + 8) * _E * size
    if residual is not None:
        y = y + residual
        ey = ey + _E * np.abs(y)
    return _stored(y, ey, out)
