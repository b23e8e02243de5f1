"""Gradients of the layer products where the tests of whole results do not look:
columns beside one that is not finite, at every kernel that sums weights'
gradients; bias gradients against sums of unrounded values; the gradients
before the activation themselves."""

import numpy as np
import pytest
import torch

from oracle import products as ref
from tests._gpu import _Env, lib, need_gpu
from tests.test_gpu_products import Ranks, close

pytestmark = pytest.mark.gpu

TORCH = {"float32": torch.float32, "bfloat16": torch.bfloat16,
         "float16": torch.float16}


def normal(gen, *shape, dtype, far=0, scale=1.0):
    """Rows `far` values apart."""
    t = torch.randn(*shape[:-1], shape[-1] + far, generator=gen,
                    device="cuda") * scale
    return t.to(TORCH[dtype])[..., :shape[-1]]


# call, ranks, rows, in, out, type, distance between rows; the kernel of dw
WEIGHT_KERNELS = [
    ("gated_backward", 1, 2778, 720, 656, "bfloat16", 0,
     "operands=aligned kernel=128x128 splits="),
    ("gated_backward", 8, 47, 80, 1544, "float16", 0,
     "operands=aligned kernel=128x128 splits=1"),
    ("gated_backward", 1, 5174, 552, 920, "bfloat16", 0,
     "operands=aligned kernel=256x128 splits="),
    ("gated_backward", 4, 42, 72, 4512, "bfloat16", 0,
     "operands=aligned kernel=256x128 splits=1"),
    ("gated_backward", 1, 3813, 1640, 1432, "bfloat16", 0,
     "operands=aligned kernel=256x256 splits="),
    ("gated_backward", 4, 44, 272, 2856, "float16", 0,
     "operands=aligned kernel=256x256 splits=1"),
    ("gated_backward", 1, 2125, 144, 208, "bfloat16", 0,
     "operands=aligned kernel=64x64 splits="),
    ("gated_backward", 4, 44, 8, 2056, "float16", 0,
     "operands=aligned kernel=64x64 splits=1"),
    ("linear_backward", 1, 902, 8, 216, "bfloat16", 0,
     "operands=aligned kernel=64x64x4 splits="),
    ("linear_backward", 1, 43, 8, 216, "float16", 0,
     "operands=aligned kernel=64x64x4 splits=1"),
    ("gated_backward", 1, 5695, 396, 616, "float16", 0,
     "operands=copied kernel=128x128 splits="),
    ("gated_backward", 1, 402, 651, 2616, "bfloat16", 0,
     "operands=copied kernel=128x128 splits=1"),
    ("gated_backward", 1, 3767, 267, 1792, "bfloat16", 0,
     "operands=copied kernel=256x128 splits="),
    ("gated_backward", 1, 411, 3616, 521, "float16", 0,
     "operands=copied kernel=256x128 splits=1"),
    ("gated_backward", 1, 4272, 1731, 1193, "float16", 5,
     "operands=copied kernel=256x256 splits="),
    ("gated_backward", 1, 209, 2316, 1759, "float16", 5,
     "operands=copied kernel=256x256 splits=1"),
    ("gated_backward", 1, 2204, 155, 1360, "float16", 0,
     "operands=copied kernel=64x64 splits="),
    ("gated_backward", 1, 513, 657, 1168, "bfloat16", 0,
     "operands=copied kernel=64x64 splits=1"),
    ("linear_backward", 1, 405, 5, 205, "bfloat16", 0,
     "operands=copied kernel=64x64x4 splits=1"),
    ("gated_backward", 1, 2285, 695, 340, "float16", 0,
     "operands=unaligned kernel=128x128 splits="),
    ("gated_backward", 1, 44, 264, 4961, "bfloat16", 0,
     "operands=unaligned kernel=128x128 splits=1"),
    ("linear_backward", 1, 455, 7, 203, "float16", 0,
     "operands=unaligned kernel=64x64 splits="),
    ("linear_backward", 1, 42, 1, 200, "bfloat16", 0,
     "operands=unaligned kernel=64x64 splits=1"),
    ("linear_backward", 1, 4802, 992, 2608, "float32", 0,
     "operands=aligned kernel=128x128 splits="),
    ("gated_backward", 4, 46, 208, 3648, "float32", 0,
     "operands=aligned kernel=128x128 splits=1"),
    ("gated_backward", 1, 482, 8, 1376, "float32", 0,
     "operands=aligned kernel=64x64 splits="),
    ("gated_backward", 16, 41, 8, 544, "float32", 0,
     "operands=aligned kernel=64x64 splits=1"),
    ("gated_backward", 1, 299, 8, 216, "float32", 0,
     "operands=aligned kernel=64x64x4 splits="),
    ("gated_backward", 1, 42, 8, 208, "float32", 0,
     "operands=aligned kernel=64x64x4 splits=1"),
    ("gated_backward", 1, 3700, 1741, 1454, "float32", 0,
     "operands=copied kernel=128x128 splits="),
    ("gated_backward", 1, 439, 2166, 2671, "float32", 0,
     "operands=copied kernel=128x128 splits=1"),
    ("gated_backward", 1, 2568, 290, 900, "float32", 0,
     "operands=copied kernel=64x64 splits="),
    ("gated_backward", 1, 776, 1110, 500, "float32", 0,
     "operands=copied kernel=64x64 splits=1"),
    ("linear_backward", 1, 5293, 6, 256, "float32", 0,
     "operands=copied kernel=64x64x4 splits="),
    ("gated_backward", 1, 382, 887, 332, "float32", 0,
     "operands=copied kernel=64x64x4 splits=1"),
    ("gated_backward", 2, 3201, 846, 359, "float32", 0,
     "operands=unaligned kernel=128x128 splits="),
    ("gated_backward", 16, 41, 75, 1842, "float32", 5,
     "operands=unaligned kernel=128x128 splits=1"),
    ("linear_backward", 1, 232, 3, 215, "float32", 0,
     "operands=unaligned kernel=64x64 splits="),
    ("gated_backward", 1, 40, 1, 213, "float32", 0,
     "operands=unaligned kernel=64x64 splits=1"),
]


@pytest.mark.parametrize("op,p,rows,n_in,n_out,dtype,far,plan",
                         WEIGHT_KERNELS)
def test_columns_that_are_not_finite_stay_alone(op, p, rows, n_in, n_out,
                                                dtype, far, plan, capfd):
    """An infinity and a NaN in two columns of dy: the other columns' bias
    gradients, the other rows of dw and the other rows of dx are what they are
    with finite values there, bit for bit."""
    need_gpu()
    if torch.cuda.get_device_properties(0).multi_processor_count != 256:
        pytest.skip("the rules count CUs")
    d = lib()
    g = torch.Generator("cuda").manual_seed(31)
    x = normal(g, p, rows, n_in, dtype=dtype, far=far)
    w = normal(g, p, n_out, n_in, dtype=dtype, far=far, scale=n_in ** -0.5)
    dy = normal(g, p, rows, n_out, dtype=dtype, far=far)
    kept = normal(g, p, rows, n_out, dtype=dtype)

    def run():
        if op == "linear_backward":
            return d.linear_backward(dy, x, w, kept, act="silu", bias=True)
        return d.gated_backward(dy, x, w, w, kept, kept, bias=True)

    capfd.readouterr()
    with _Env("DPAR_LOG", 1):
        want = [t.clone() for t in run()]
    log = [ln for ln in capfd.readouterr().err.splitlines()
           if "product=dw" in ln]
    assert len(log) == 1 and plan in log[0] and \
        (plan[-1] == "1") == log[0].endswith("splits=1"), log
    at = {5: float("inf"), n_out - 9: float("nan")}      # columns
    for c, v in at.items():
        dy[:, rows // 2, c] = v
    got = run()
    rows_left = [i for i in range(rows) if i != rows // 2]
    cols_left = [j for j in range(n_out) if j not in at]
    assert torch.equal(got[0][:, rows_left], want[0][:, rows_left])
    for a, b in zip(got[1:], want[1:]):
        assert torch.isfinite(b).all()
        assert torch.equal(a[:, cols_left], b[:, cols_left])
        for c in at:
            assert not torch.isfinite(a[:, c]).any()


def np64(t):
    return t.double().cpu().numpy()


# rows, out: one part, several, columns of less than a piece and of several
# strips, rows off 16 bytes, more ranks than one launch takes
@pytest.mark.parametrize("p,rows,n_out", [
    (1, 1, 1), (2, 5, 72), (1, 63, 64), (3, 65, 131), (1, 700, 40),
    (1, 2048, 200), (2, 4099, 129), (50, 1030, 24), (1, 8192, 1024)])
@pytest.mark.parametrize("act", ["none", "relu", "silu"])
@pytest.mark.parametrize("dtype", ["bfloat16", "float16", "float32"])
def test_bias_gradients_sum_unrounded_values(p, rows, n_out, act, dtype):
    """In 32 bits they are n products and additions off, each of 2^-24, and
    what the activation's slope is; rounding each value to 16 bits first would
    leave 2^-9 or 2^-12 of it.  With and without a workspace."""
    need_gpu()
    d = lib()
    g = torch.Generator("cuda").manual_seed(32)
    x = normal(g, p, rows, 8, dtype=dtype)
    w = normal(g, p, n_out, 8, dtype=dtype)
    dy, kg, ku = (normal(g, p, rows, n_out, dtype=dtype) for _ in range(3))
    dz, du = torch.empty_like(dy), torch.empty_like(dy)
    f32 = dict(dtype=torch.float32, device="cuda")
    dw, dw2 = (torch.empty(p, n_out, 8, **f32) for _ in range(2))
    opt = d.product_options(rows, 8, n_out, dtype, "float32", act)
    r = d.rows
    stream = torch.cuda.current_stream()

    def check(got, terms, slack):
        bound = (rows + 3) * 2.0 ** -24 * np.abs(terms).sum(1) + slack.sum(1)
        assert (np.abs(np64(got) - terms.sum(1)) <= bound).all()

    v, s = (np64(t) for t in (dy, kg))
    a, slope = ref.act(s, act)
    err = 0 * v if act in ("none", "relu") else \
        2.0 ** -20 * (1 + np.abs(s)) * np.abs(v)
    for split in (True, False):
        db, dbu = (torch.full((p, n_out), 7.0, **f32) for _ in range(2))
        n = d.dpar_product_workspace("linear_backward", p, opt)
        ws = torch.empty(max(n, 16), dtype=torch.uint8, device="cuda")
        ws = (ws, n) if split else (None, 0)
        d.dpar_linear_backward(
            r(dy), r(x), r(w), r(kg) if act != "none" else None, None, r(dw),
            r(db), r(dz) if act != "none" else None, p, opt, *ws, stream)
        check(db, v * slope, err)
        n = d.dpar_product_workspace("gated_backward", p, opt)
        ws = torch.empty(max(n, 16), dtype=torch.uint8, device="cuda")
        ws = (ws, n) if split else (None, 0)
        d.dpar_gated_backward(
            r(dy), r(x), r(w), r(w), r(kg), r(ku), None, r(dw), r(dw2), r(db),
            r(dbu), r(dz), r(du), p, opt, *ws, stream)
        check(db, v * np64(ku) * slope, err * np.abs(np64(ku)))
        check(dbu, v * a, err)


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
def test_single_rows_of_any_distance(dtype):
    """One row of x and dy, one of w, with odd distances that no second row
    uses: the results of packed ones."""
    need_gpu()
    d = lib()
    g = torch.Generator("cuda").manual_seed(33)
    r, stream = d.rows, torch.cuda.current_stream()
    for rows, n_in, n_out in ((1, 264, 136), (40, 264, 1)):
        x, w, dy = (normal(g, 1, *s, dtype=dtype) for s in
                    ((rows, n_in), (n_out, n_in), (rows, n_out)))
        got = []
        for far in ({}, {"ldx": 1, "ldy": 3, "lddx": 5} if rows == 1 else
                    {"ldw": 1, "lddw": 3}):
            opt = d.product_options(rows, n_in, n_out, dtype, **far)
            out = [torch.empty_like(t) for t in (x, w, dy)]
            d.dpar_linear_backward(r(dy), r(x), r(w), None, r(out[0]),
                                   r(out[1]), None, None, 1, opt,
                                   stream=stream)
            d.dpar_linear(r(x), r(w), None, None, r(out[2]), None, 1, opt,
                          stream=stream)
            got.append(out)
        for a, b in zip(*got):
            assert torch.equal(a, b)


@pytest.mark.parametrize("rows,n_out", [(1, 1), (3, 40), (70, 137), (65, 64),
                                        (130, 7)])
@pytest.mark.parametrize("far,shift", [(0, 0), (8, 0), (3, 5), (64, 4)])
@pytest.mark.parametrize("place", [None, "z", "dy"])
@pytest.mark.parametrize("dtype", ["bfloat16", "float16", "float32"])
@pytest.mark.parametrize("bias", [False, True])
def test_gradients_before_the_activation(rows, n_out, far, shift, place, dtype,
                                         bias):
    """dz, dg and du, which the calls hand out: within their own rounding, in
    place of what they may replace, and nothing between their rows."""
    need_gpu()
    d = lib()
    p, n_in = 2, 8
    g = torch.Generator("cuda").manual_seed(34)
    for op, act in (("linear", "gelu"), ("gated", "silu")):
        x, w = (Ranks(p, a, n_in, dtype, gen=g) for a in (rows, n_out))
        dy, kg, ku = (Ranks(p, rows, n_out, dtype, far, shift, g)
                      for _ in range(3))
        dw, dw2 = (Ranks(p, n_out, n_in, dtype) for _ in range(2))
        sums = [Ranks(p, 1, n_out, dtype) for _ in range(2)]
        db, db2 = (t.at if bias else None for t in sums)
        first = {None: Ranks(p, rows, n_out, dtype, far, shift), "z": kg,
                 "dy": dy}[place]
        second = ku if place else Ranks(p, rows, n_out, dtype, far, shift)
        opt = d.product_options(rows, n_in, n_out, dtype, act=act, ldy=dy.ld,
                                ldz=kg.ld)
        v, z, u = (np64(t.t) for t in (dy, kg, ku))
        a, slope = ref.act(z, act)
        if op == "linear":
            d.dpar_linear_backward(dy.at, x.at, w.at, kg.at, None, dw.at, db,
                                   first.at, p, opt)
            want = ref._slope(v, z, act, dtype)
        else:
            d.dpar_gated_backward(dy.at, x.at, w.at, w.at, kg.at, ku.at, None,
                                  dw.at, dw2.at, db, db2, first.at, second.at,
                                  p, opt)
            err = 2.0 ** -20 * (1 + np.abs(z)) * np.abs(v)
            want = ref._stored(v * u * slope, err * np.abs(u), dtype)
            close(second.t, ref._stored(v * a, err, dtype), "du")
            assert second.gaps_untouched()
        close(first.t, want, op)
        assert first.gaps_untouched()
