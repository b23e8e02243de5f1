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
