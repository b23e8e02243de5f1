"""Activations and their slopes where results are stored in 32 bits, value by
value: x runs through a 1 x 1 identity, so that the product adds no error, and
each result is within what its operations may lose.

With u = 2^-24 (a product or sum in 32 bits is off by u of it; expf by 3 units
in the last place, 6 u, a division by 5 u, erfcf by 16 units, 32 u: the bounds
that OpenCL sets for them):
  silu       z / (1 + e): 6 u + u + 5 u + u, bound 16 u |y|
  gelu       an argument 2 u off changes erfc(x) by 2 u (2 x^2 + 1) of it,
             z^2 = 2 x^2; with erfc and three products (2 z^2 + 37) u |y|
  gelu_tanh  the argument a of 1 / (1 + exp(-a)) is 7 u off, which changes it
             by 7 |a| u of it; with the rest of silu's steps (7 |a| + 16) u |y|
Slopes are sums of two terms, each a few steps more: the same bounds with 40,
40 and 40 for 16, 37 and 16, of the terms' absolute values.
"""

import math

import numpy as np
import pytest
import torch

from tests._gpu import lib, need_gpu

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
TINY = 2.0 ** -125
_erfc = np.vectorize(math.erfc, otypes=[np.float64])


def exact(act, z):
    """act(z) and its bound, act'(z) and its bound."""
    if act == "gelu":
        c = 0.5 * _erfc(-z / math.sqrt(2))
        d = z * np.exp(-z * z / 2) / math.sqrt(2 * math.pi)
        return (z * c, (2 * z * z + 37) * U * np.abs(z * c), c + d,
                (2 * z * z + 40) * U * (np.abs(c) + np.abs(d)))
    k = 2 * math.sqrt(2 / math.pi)
    a, da = (z, 1.0) if act == "silu" else \
        (k * (z + 0.044715 * z ** 3), k * (1 + 3 * 0.044715 * z * z))
    s = 1 / (1 + np.exp(-a))
    d = z * s / (1 + np.exp(a)) * da
    more = 0 if act == "silu" else 7 * np.abs(a)
    return (z * s, (more + 16) * U * np.abs(z * s), s + d,
            (more + 40) * U * (np.abs(s) + np.abs(d)))


@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh"])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("cols", [1, 8])
def test_activations_in_32_bits(act, dtype, cols):
    """At rows of the few-rows kernel, tiles and split tiles; 32-bit slopes
    alone and in sums of one row."""
    need_gpu()
    d = lib()
    t = getattr(torch, dtype)
    far = {"silu": 60.0, "gelu": 10.0, "gelu_tanh": 5.0}[act]
    z = torch.linspace(-far, far, 4001, device="cuda").to(t)
    z = torch.cat([z, z / 64]).float()
    z = z[z.abs() > 2.0 ** -20].to(t)
    v = z.double().cpu().numpy()
    y, ey, s, es = exact(act, v)
    one = torch.ones(1, 1, device="cuda", dtype=t)

    def check(got, want, bound):
        g = got.double().cpu().numpy()
        bad = np.abs(g - want) > bound + TINY
        assert not bad.any(), (int(bad.sum()), v[bad][0], g[bad][0],
                               want[bad][0], bound[bad][0])

    n = z.numel()
    # a column of x each value, weights of ones in the first of `cols` places
    w = torch.zeros(cols, cols, device="cuda", dtype=t)
    w[0, 0] = 1
    x = torch.zeros(n, cols, device="cuda", dtype=t)
    x[:, 0] = z
    got = d.linear(x, w, act=act, out_dtype=torch.float32)
    check(got[:, 0], y, ey)
    for i in range(0, n, 1000):                    # few rows
        got = d.linear(x[i:i + 16], w, act=act, out_dtype=torch.float32)
        check(got[:, 0], y[i:i + 16], ey[i:i + 16])
        v2 = d.gated(x[i:i + 16], w, w, bu=one.expand(1, cols)[0].contiguous(),
                     act=act, out_dtype=torch.float32)
        m = v[i:i + 16] + 1
        check(v2[:, 0], y[i:i + 16] * m,
              (ey[i:i + 16] + 2 * U * np.abs(y[i:i + 16])) * np.abs(m))
    # slopes: every value a column of one row, dbias its sum
    ones = torch.ones(1, n, device="cuda", dtype=t)
    wide = torch.zeros(n, 8, device="cuda", dtype=t)
    _, _, db = d.linear_backward(ones, ones[:, :8].contiguous(), wide,
                                 z[None], act=act, out_dtype=torch.float32,
                                 bias=True)
    check(db, s, es)
    if dtype == "float32":
        dx, _ = d.linear_backward(ones.t().contiguous(),
                                  ones.t().contiguous(), one, z[:, None],
                                  act=act)
        check(dx[:, 0], s, es)
