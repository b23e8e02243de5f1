"""Results in place of their residuals, at every kernel that adds them."""

import pytest
import torch

from oracle import products as ref
from tests._gpu import lib, need_gpu
from tests.test_gpu_products import Ranks, close, gen, np64, workspace

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows,n_in,n_out", [
    (1, 264, 48), (40, 520, 136), (70, 4104, 264), (300, 72, 520),
    (130, 201, 333), (1000, 200, 2000)])
@pytest.mark.parametrize("dtype,out", [("bfloat16", "bfloat16"),
                                       ("float16", "float32"),
                                       ("float32", "float32")])
@pytest.mark.parametrize("far", [0, 3])
def test_residual_in_place(rows, n_in, n_out, dtype, out, far):
    need_gpu()
    d, g, p = lib(), gen(41), 2
    x = Ranks(p, rows, n_in, dtype, far, 0, g)
    w = Ranks(p, n_out, n_in, dtype, far, 0, g, n_in ** -0.5)
    b = Ranks(p, 1, n_out, dtype, 0, 0, g)
    y = Ranks(p, rows, n_out, out, far, 0, g)
    given = [np64(y.t[i]) for i in range(p)]
    opt = d.product_options(rows, n_in, n_out, dtype, out, "gelu", ldx=x.ld,
                            ldw=w.ld, ldy=y.ld, ldr=y.ld)
    ws, n = workspace("linear", p, opt, True)
    d.dpar_linear(x.at, w.at, b.at, y.at, y.at, None, p, opt, ws, n,
                  torch.cuda.current_stream())
    for i in range(p):
        want = ref.linear(np64(x.t[i]), np64(w.t[i]), np64(b.t[i, 0]),
                          given[i], "gelu", dtype, out)
        close(y.t[i], want["y"], f"y of rank {i}")
    assert y.gaps_untouched()
