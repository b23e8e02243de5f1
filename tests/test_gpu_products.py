"""Layer products on the GPU against the definition in 64 bits (oracle/
products.py), element by element within the bound that 32-bit sums and the
stated roundings allow."""

import numpy as np
import pytest
import torch

from oracle import products as ref
from tests._gpu import lib, need_gpu

pytestmark = pytest.mark.gpu

TORCH = {"float32": torch.float32, "bfloat16": torch.bfloat16,
         "float16": torch.float16}
FILL = 77.0        # what lies between rows and after buffers


def np64(t):
    return t.double().cpu().numpy()


class Ranks:
    """p matrices of rows x cols in one buffer, `far` elements between rows and
    `shift` before the first; everything else holds FILL."""

    def __init__(self, p, rows, cols, dtype, far=0, shift=0, gen=None,
                 scale=1.0):
        self.ld = cols + far
        size = p * max(rows, 1) * self.ld + shift + 64
        self.flat = torch.full((size,), FILL, dtype=TORCH[dtype],
                               device="cuda")
        self.t = self.flat[shift:shift + p * rows * self.ld].view(
            p, rows, self.ld)[..., :cols]
        if gen is not None:
            self.t.copy_(torch.randn(p, rows, cols, generator=gen,
                                     device="cuda") * scale)
        self.at = lib().pointers([self.t.data_ptr() + i * rows * self.ld
                                  * self.flat.element_size()
                                  for i in range(p)])

    def gaps_untouched(self):
        mask = torch.ones_like(self.flat, dtype=torch.bool)
        n = self.t.numel()
        if n:
            start = self.t.storage_offset()
            mask[start:start + self.t.shape[0] * self.t.shape[1] * self.ld] \
                .view(self.t.shape[0], self.t.shape[1],
                      self.ld)[..., :self.t.shape[2]] = False
        return bool((self.flat[mask] == FILL).all())


def close(got, want, what):
    v, slack = want
    g = np64(got)
    assert g.shape == v.shape, (what, g.shape, v.shape)
    assert np.isfinite(g).all(), what
    bad = np.abs(g - v) > slack
    assert not bad.any(), (what, int(bad.sum()), np.argwhere(bad)[0],
                           g[bad][0], v[bad][0], slack[bad][0])


def gen(seed):
    return torch.Generator("cuda").manual_seed(seed)


def workspace(call, p, opt, split):
    n = lib().dpar_product_workspace(call, p, opt) if split else 0
    return (torch.empty(max(n, 16), dtype=torch.uint8, device="cuda"), n) \
        if n else (None, 0)


def run_linear(p, rows, n_in, n_out, dtype="bfloat16", out=None, act="none",
               bias=True, residual=True, keep=True, far=0, shift=0, split=True,
               seed=0):
    d = lib()
    out = out or dtype
    g = gen(seed)
    x = Ranks(p, rows, n_in, dtype, far, shift, g)
    w = Ranks(p, n_out, n_in, dtype, far, shift, g, max(n_in, 1) ** -0.5)
    b = Ranks(p, 1, n_out, dtype, 0, shift, g) if bias else None
    r = Ranks(p, rows, n_out, out, far, shift, g) if residual else None
    y = Ranks(p, rows, n_out, out, far, shift)
    z = Ranks(p, rows, n_out, dtype, far, shift) if keep else None
    opt = d.product_options(rows, n_in, n_out, dtype, out, act, ldx=x.ld,
                            ldw=w.ld, ldy=y.ld, ldr=n_out + far,
                            ldz=n_out + far)
    ws, n = workspace("linear", p, opt, split)
    at = [None if t is None else t.at for t in (x, w, b, r, y, z)]
    d.dpar_linear(*at, p, opt, ws, n, torch.cuda.current_stream())
    for i in range(p):
        want = ref.linear(np64(x.t[i]), np64(w.t[i]),
                          np64(b.t[i, 0]) if bias else None,
                          np64(r.t[i]) if residual else None, act, dtype, out)
        close(y.t[i], want["y"], f"y of rank {i}")
        if keep:
            close(z.t[i], want["z"], f"z of rank {i}")
    assert y.gaps_untouched() and (z is None or z.gaps_untouched())
    return y.t


def run_linear_backward(p, rows, n_in, n_out, dtype="bfloat16", out=None,
                        act="gelu", bias=True, far=0, shift=0, split=True,
                        seed=0, place=None):
    d = lib()
    out = out or dtype
    g = gen(seed)
    x = Ranks(p, rows, n_in, dtype, far, shift, g)
    w = Ranks(p, n_out, n_in, dtype, far, shift, g, max(n_in, 1) ** -0.5)
    dy = Ranks(p, rows, n_out, dtype, far, shift, g)
    z = Ranks(p, rows, n_out, dtype, far, shift, g, 1.5)
    dx = Ranks(p, rows, n_in, out, far, shift)
    dw = Ranks(p, n_out, n_in, out, far, shift)
    db = Ranks(p, 1, n_out, out, 0, shift) if bias else None
    dz = {None: Ranks(p, rows, n_out, dtype, far, shift), "z": z,
          "dy": dy}[place]
    opt = d.product_options(rows, n_in, n_out, dtype, out, act, ldx=x.ld,
                            ldw=w.ld, ldy=dy.ld, ldz=z.ld, lddx=dx.ld,
                            lddw=dw.ld)
    ws, n = workspace("linear_backward", p, opt, split)
    given = [(np64(dy.t[i]), np64(x.t[i]), np64(w.t[i]), np64(z.t[i]))
             for i in range(p)]
    at = [None if t is None else t.at for t in (dy, x, w, z, dx, dw, db, dz)]
    if act == "none":
        at[3] = at[7] = None
    d.dpar_linear_backward(*at, p, opt, ws, n, torch.cuda.current_stream())
    for i in range(p):
        want = ref.linear_backward(*given[i], act, dtype, out)
        close(dx.t[i], want["dx"], f"dx of rank {i}")
        close(dw.t[i], want["dwz"], f"dw of rank {i}")
        if bias:
            close(db.t[i, 0], want["dbz"], f"dbias of rank {i}")
    for t in (dx, dw, db):
        assert t is None or t.gaps_untouched()


def run_gated(p, rows, n_in, n_out, dtype="bfloat16", out=None, act="silu",
              bias=True, keep=True, far=0, shift=0, split=True, shared=False,
              seed=0):
    d = lib()
    out = out or dtype
    g = gen(seed)
    x = Ranks(1 if shared else p, rows, n_in, dtype, far, shift, g)
    wg, wu = (Ranks(p, n_out, n_in, dtype, far, shift, g,
                    max(n_in, 1) ** -0.5) for _ in range(2))
    bg, bu = (Ranks(p, 1, n_out, dtype, 0, shift, g) if bias else None
              for _ in range(2))
    h = Ranks(p, rows, n_out, out, far, shift)
    kg, ku = (Ranks(p, rows, n_out, dtype, far, shift) if keep else None
              for _ in range(2))
    opt = d.product_options(rows, n_in, n_out, dtype, out, act, ldx=x.ld,
                            ldw=wg.ld, ldy=h.ld, ldz=n_out + far)
    ws, n = workspace("gated", p, opt, split)
    at = [None if t is None else t.at for t in (x, wg, wu, bg, bu, h, kg, ku)]
    if shared:
        at[0] = d.pointers([x.t.data_ptr()] * p)
    d.dpar_gated(*at, p, opt, ws, n, torch.cuda.current_stream())
    for i in range(p):
        want = ref.gated(np64(x.t[0 if shared else i]), np64(wg.t[i]),
                         np64(wu.t[i]), np64(bg.t[i, 0]) if bias else None,
                         np64(bu.t[i, 0]) if bias else None, act, dtype, out)
        close(h.t[i], want["h"], f"h of rank {i}")
        if keep:
            close(kg.t[i], want["g"], f"g of rank {i}")
            close(ku.t[i], want["u"], f"u of rank {i}")
    for t in (h, kg, ku):
        assert t is None or t.gaps_untouched()


def run_gated_backward(p, rows, n_in, n_out, dtype="bfloat16", out=None,
                       act="silu", bias=True, far=0, shift=0, split=True,
                       seed=0, in_place=False):
    d = lib()
    out = out or dtype
    g = gen(seed)
    x = Ranks(p, rows, n_in, dtype, far, shift, g)
    wg, wu = (Ranks(p, n_out, n_in, dtype, far, shift, g,
                    max(n_in, 1) ** -0.5) for _ in range(2))
    dh = Ranks(p, rows, n_out, dtype, far, shift, g)
    kg, ku = (Ranks(p, rows, n_out, dtype, far, shift, g) for _ in range(2))
    dx = Ranks(p, rows, n_in, out, far, shift)
    dwg, dwu = (Ranks(p, n_out, n_in, out, far, shift) for _ in range(2))
    dbg, dbu = (Ranks(p, 1, n_out, out, 0, shift) if bias else None
                for _ in range(2))
    dg, du = (kg, ku) if in_place else (
        Ranks(p, rows, n_out, dtype, far, shift) for _ in range(2))
    opt = d.product_options(rows, n_in, n_out, dtype, out, act, ldx=x.ld,
                            ldw=wg.ld, ldy=dh.ld, ldz=kg.ld, lddx=dx.ld,
                            lddw=dwg.ld)
    ws, n = workspace("gated_backward", p, opt, split)
    given = [tuple(np64(t.t[i]) for t in (dh, x, wg, wu, kg, ku))
             for i in range(p)]
    at = [None if t is None else t.at for t in
          (dh, x, wg, wu, kg, ku, dx, dwg, dwu, dbg, dbu, dg, du)]
    d.dpar_gated_backward(*at, p, opt, ws, n, torch.cuda.current_stream())
    for i in range(p):
        want = ref.gated_backward(*given[i], act, dtype, out)
        close(dx.t[i], want["dx"], f"dx of rank {i}")
        close(dwg.t[i], want["dwg"], f"dwg of rank {i}")
        close(dwu.t[i], want["dwu"], f"dwu of rank {i}")
        if bias:
            close(dbg.t[i, 0], want["dbg"], f"dbg of rank {i}")
            close(dbu.t[i, 0], want["dbu"], f"dbu of rank {i}")
    for t in (dx, dwg, dwu, dbg, dbu):
        assert t is None or t.gaps_untouched()


RUNS = {"linear": run_linear, "linear_backward": run_linear_backward,
        "gated": run_gated, "gated_backward": run_gated_backward}
# rows, in, out: one of each, edges of the 16-, 64-, 128- and 256-wide tiles,
# of 16-byte pieces and of 128- and 512-byte steps of the contraction
SIZES = [(1, 1, 1), (1, 8, 8), (1, 64, 16), (2, 7, 3), (3, 64, 65),
         (15, 256, 17), (16, 264, 48), (17, 248, 33), (31, 520, 64),
         (33, 40, 129), (48, 72, 40), (49, 1000, 24), (64, 512, 56),
         (65, 63, 127), (66, 136, 128), (127, 65, 66), (129, 200, 257),
         (200, 31, 8)]


@pytest.mark.parametrize("op", RUNS)
@pytest.mark.parametrize("dtype", ["bfloat16", "float16", "float32"])
@pytest.mark.parametrize("rows,n_in,n_out", SIZES)
def test_sizes(op, dtype, rows, n_in, n_out):
    need_gpu()
    RUNS[op](2, rows, n_in, n_out, dtype, act="silu", seed=rows)


@pytest.mark.parametrize("op", RUNS)
@pytest.mark.parametrize("act", ["none", "relu", "gelu", "gelu_tanh", "silu"])
@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
def test_activations(op, act, dtype):
    need_gpu()
    RUNS[op](1, 70, 96, 72, dtype, act=act, seed=3)


@pytest.mark.parametrize("op", RUNS)
@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("rows", [5, 40, 100, 300])
def test_results_in_32_bits(op, dtype, rows):
    need_gpu()
    RUNS[op](2, rows, 136, 80, dtype, "float32", act="silu", seed=4)


@pytest.mark.parametrize("op", RUNS)
@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("far,shift", [(8, 0), (1, 0), (0, 1), (3, 5),
                                       (16, 8), (64, 4)])
@pytest.mark.parametrize("rows", [3, 70, 130])
def test_row_distances_and_alignments(op, dtype, far, shift, rows):
    """Rows apart, off 16 bytes, off everything but their element; nothing
    between or around them changes."""
    need_gpu()
    RUNS[op](2, rows, 72, 40, dtype, act="gelu_tanh", far=far, shift=shift)


@pytest.mark.parametrize("op", RUNS)
@pytest.mark.parametrize("rows,n_in,n_out", [
    (256, 256, 256), (512, 320, 768), (300, 4096, 264), (257, 72, 520),
    (1000, 200, 1304)])
def test_large_tiles(op, rows, n_in, n_out):
    """Enough ranks that the 256 x 256 tiles run."""
    need_gpu()
    RUNS[op](36, rows, n_in, n_out, act="silu", seed=5) \
        if rows * n_in * n_out < 2e7 else \
        RUNS[op](8, rows, n_in, n_out, act="silu", seed=5)


@pytest.mark.parametrize("op", RUNS)
@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("rows,n_in,n_out", [
    (70, 4000, 40), (100, 40, 4000), (4000, 40, 70), (2000, 1000, 24),
    (66, 2056, 2056)])
def test_long_sums_split_and_unsplit(op, dtype, rows, n_in, n_out):
    """Few results and a long sum, with a workspace and without one."""
    need_gpu()
    for split in (True, False):
        RUNS[op](1, rows, n_in, n_out, dtype, split=split, seed=6)


@pytest.mark.parametrize("op", RUNS)
@pytest.mark.parametrize("p", [1, 3, 47, 48, 49, 97])
def test_ranks(op, p):
    """More ranks than one launch takes."""
    need_gpu()
    RUNS[op](p, 9, 24, 40, seed=7)


@pytest.mark.parametrize("rows", [1, 30, 80])
def test_shared_input(rows):
    need_gpu()
    run_gated(5, rows, 64, 48, shared=True)


@pytest.mark.parametrize("place", ["z", "dy"])
@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
def test_slope_in_place(place, dtype):
    need_gpu()
    run_linear_backward(2, 70, 48, 56, dtype, place=place)


@pytest.mark.parametrize("dtype", ["float16", "float32"])
def test_gated_slopes_in_place(dtype):
    need_gpu()
    run_gated_backward(2, 70, 48, 56, dtype, in_place=True)


@pytest.mark.parametrize("op", RUNS)
def test_without_biases(op):
    need_gpu()
    RUNS[op](2, 20, 40, 24, bias=False)
    RUNS[op](2, 140, 40, 24, bias=False)


def test_bias_and_residual_on_one_rank_only():
    """The other ranks' entries are null: partial sums of a split layer."""
    need_gpu()
    d = lib()
    g = gen(8)
    for rows in (4, 80):
        x, w, y = (Ranks(3, a, b, "bfloat16", gen=g) for a, b in
                   ((rows, 32), (24, 32), (rows, 24)))
        out = Ranks(3, rows, 24, "float32")
        b = Ranks(1, 1, 24, "bfloat16", gen=g)
        r = Ranks(1, rows, 24, "float32", gen=g)
        opt = d.product_options(rows, 32, 24, "bfloat16", "float32")
        d.dpar_linear(x.at, w.at, [0, b.t.data_ptr(), 0],
                      [0, 0, r.t.data_ptr()], out.at, None, 3, opt)
        for i in range(3):
            want = ref.linear(np64(x.t[i]), np64(w.t[i]),
                              np64(b.t[0, 0]) if i == 1 else None,
                              np64(r.t[0]) if i == 2 else None, "none",
                              "bfloat16", "float32")
            close(out.t[i], want["y"], f"rank {i}")


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("rows,n_in,n_out", [(5, 0, 24), (80, 0, 24),
                                             (300, 0, 300)])
def test_empty_contraction(dtype, rows, n_in, n_out):
    """No inputs: act(bias) + residual, and bias gradients."""
    need_gpu()
    run_linear(2, rows, n_in, n_out, dtype, act="silu")
    run_gated(2, rows, n_in, n_out, dtype)
    run_linear_backward(2, rows, n_in, n_out, dtype)
    run_gated_backward(2, rows, n_in, n_out, dtype)


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("n_in,n_out", [(24, 40), (300, 300)])
def test_no_rows_give_zero_gradients(dtype, n_in, n_out):
    need_gpu()
    run_linear_backward(2, 0, n_in, n_out, dtype)
    run_gated_backward(2, 0, n_in, n_out, dtype)
    run_linear(2, 0, n_in, n_out, dtype)


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
def test_no_outputs_give_zero_input_gradients(dtype):
    need_gpu()
    run_linear_backward(2, 70, 24, 0, dtype)
    run_gated_backward(2, 70, 24, 0, dtype)


@pytest.mark.parametrize("rows", [4, 40, 70, 300])
@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
def test_values_that_are_not_finite_stay_in_their_rows(rows, dtype):
    """NaN and infinities in one row of x and one of w reach that row and that
    column only, whatever lies past the rows' ends; between rows lie NaNs."""
    need_gpu()
    d = lib()
    n_in, n_out, far = 72, 40, 8
    g = gen(9)
    x, w = (Ranks(1, a, n_in, dtype, far, 0, g) for a in (rows, n_out))
    for t in (x, w):
        t.flat[t.flat == FILL] = float("nan")
    y = Ranks(1, rows, n_out, dtype)
    opt = d.product_options(rows, n_in, n_out, dtype, ldx=x.ld, ldw=w.ld)

    def run():
        d.dpar_linear(x.at, w.at, None, None, y.at, None, 1, opt)
        return np64(y.t[0])

    assert np.isfinite(run()).all()
    x.t[0, 1, n_in - 1] = float("nan")
    w.t[0, 2, 0] = float("inf")
    got = run()
    assert np.isnan(got[1]).all() and not np.isfinite(got[:, 2]).any()
    rest = np.delete(np.delete(got, 1, 0), 2, 1)
    assert np.isfinite(rest).all()


@pytest.mark.parametrize("dtype", ["bfloat16", "float16", "float32"])
def test_activations_at_their_limits(dtype):
    """Infinities, the type's largest and smallest values and NaN through a
    1 x 1 identity: limits, and NaN stays NaN."""
    need_gpu()
    d = lib()
    big = torch.finfo(TORCH[dtype]).max
    v = [0.0, -0.0, 1e-7, -1e-7, 20.0, -20.0, 150.0, -150.0, big, -big,
         float("inf"), float("-inf"), float("nan")]
    x = torch.tensor(v, dtype=TORCH[dtype], device="cuda")[:, None]
    w = torch.ones(1, 1, dtype=TORCH[dtype], device="cuda")
    one = torch.ones_like(x)
    for act in ("relu", "gelu", "gelu_tanh", "silu"):
        y, z = d.linear(x, w, act=act, keep=True)
        got = np64(y)[:, 0]
        zs = np64(x)[:, 0]
        for k, t in enumerate(zs):
            if np.isnan(t):
                assert np.isnan(got[k]), (act, t)
            elif t >= 20:
                assert got[k] == t, (act, t, got[k])
            elif t <= -20:
                assert abs(got[k]) < 1e-6, (act, t, got[k])
        dx, dw = d.linear_backward(one, one, w, z, act=act)
        slope = np64(dx)[:, 0]
        for k, t in enumerate(zs):
            if np.isnan(t):
                assert np.isnan(slope[k]), (act, t)
            elif t >= 20:
                assert slope[k] == 1, (act, t, slope[k])
            elif t <= -20:
                assert abs(slope[k]) < 1e-6, (act, t, slope[k])


def test_relu_slope_at_zero():
    need_gpu()
    d = lib()
    x = torch.ones(3, 1, device="cuda")
    w = torch.ones(1, 1, device="cuda")
    z = torch.tensor([[0.0], [-0.0], [1e-30]], device="cuda")
    dx, _ = d.linear_backward(x, x, w, z, act="relu")
    assert dx[:, 0].tolist() == [0.0, 0.0, 1.0]


@pytest.mark.parametrize("act", ["gelu", "gelu_tanh", "silu"])
def test_gradients_against_differences(act):
    """32-bit gradients against central differences of the forward pass in 64
    bits: loss = sum(dy y).  Steps of 1e-4 leave differences 1e-6 off."""
    need_gpu()
    d = lib()
    rows, n_in, n_out = 5, 7, 6
    g = gen(10)
    x, wg, wu = (torch.randn(a, b, generator=g, device="cuda") for a, b in
                 ((rows, n_in), (n_out, n_in), (n_out, n_in)))
    bg, bu = (torch.randn(n_out, generator=g, device="cuda")
              for _ in range(2))
    dy = torch.randn(rows, n_out, generator=g, device="cuda")
    _, z = d.linear(x, wg, bg, act=act, keep=True)
    got = list(d.linear_backward(dy, x, wg, z, act=act, bias=True))
    _, kg, ku = d.gated(x, wg, wu, bg, bu, act=act, keep=True)
    got2 = list(d.gated_backward(dy, x, wg, wu, kg, ku, act=act, bias=True))

    def loss1(a):
        return (np64(dy) * ref.act(a[0] @ a[1].T + a[2], act)[0]).sum()

    def loss2(a):
        return (np64(dy) * ref.act(a[0] @ a[1].T + a[3], act)[0]
                * (a[0] @ a[2].T + a[4])).sum()

    for loss, args, grads in ((loss1, (x, wg, bg), got),
                              (loss2, (x, wg, wu, bg, bu), got2)):
        a = [np64(t) for t in args]
        for k, grad in enumerate(grads):
            want = np.zeros_like(a[k])
            for at in np.ndindex(*a[k].shape):
                keep = a[k][at]
                a[k][at] = keep + 1e-4
                up = loss(a)
                a[k][at] = keep - 1e-4
                want[at] = (up - loss(a)) / 2e-4
                a[k][at] = keep
            err = np.abs(np64(grad) - want).max()
            assert err < 2e-5 * (1 + np.abs(want).max()), (k, err)


@pytest.mark.parametrize("op", RUNS)
def test_same_results_every_time(op):
    need_gpu()
    d = lib()
    g = gen(11)
    x = torch.randn(2, 300, 520, generator=g, device="cuda").bfloat16()
    w, w2 = (torch.randn(2, 136, 520, generator=g, device="cuda").bfloat16()
             for _ in range(2))
    dy = torch.randn(2, 300, 136, generator=g, device="cuda").bfloat16()

    def run():
        if op == "linear":
            return d.linear(x, w, act="gelu", keep=True)
        if op == "gated":
            return d.gated(x, w, w2, keep=True)
        if op == "linear_backward":
            return d.linear_backward(dy, x, w, dy, act="gelu", bias=True)
        return d.gated_backward(dy, x, w, w2, dy, dy * 2, bias=True)

    first = run()
    for _ in range(5):
        for a, b in zip(first, run()):
            assert torch.equal(a, b)


def test_front_ends_of_one_matrix_and_views():
    """Two-dimensional tensors, rows taken from wider ones, one x for all
    ranks."""
    need_gpu()
    d = lib()
    g = gen(12)
    wide = torch.randn(30, 100, generator=g, device="cuda")
    x, w, w2 = wide[:20, :24], wide[5:13, 30:54], wide[10:18, 60:84]
    y = d.linear(x, w, wide[0, :8], wide[:20, 90:98], act="relu")
    want = ref.linear(np64(x), np64(w), np64(wide[0, :8]),
                      np64(wide[:20, 90:98]), "relu", "float32", "float32")
    close(y, want["y"], "y")
    h = d.gated(x, w[:, :24].contiguous(), w2.contiguous())
    want = ref.gated(np64(x), np64(w), np64(w2), None, None, "silu",
                     "float32", "float32")
    close(h, want["h"], "h")
    ranks = torch.stack([w, w2])
    y = d.linear(x, ranks)
    for i in range(2):
        want = ref.linear(np64(x), np64(ranks[i]), None, None, "none",
                          "float32", "float32")
        close(y[i], want["y"], "y of a rank")


def test_calls_on_two_streams():
    """Each stream with its own buffers and workspace, in flight together."""
    need_gpu()
    d = lib()
    streams = [torch.cuda.Stream() for _ in range(2)]
    g = gen(13)
    jobs = []
    for s in streams:
        x = torch.randn(70, 4096, generator=g, device="cuda").bfloat16()
        w = torch.randn(64, 4096, generator=g, device="cuda").bfloat16()
        jobs.append((s, x, w, []))
    torch.cuda.synchronize()
    for _ in range(20):
        for s, x, w, out in jobs:
            with torch.cuda.stream(s):
                out.append(d.linear(x, w, act="silu"))
    torch.cuda.synchronize()
    for _, x, w, out in jobs:
        want = ref.linear(np64(x), np64(w), None, None, "silu", "bfloat16",
                          "bfloat16")
        for y in out:
            close(y, want["y"], "y")


def test_calls_in_a_graph():
    """Recorded once (the split sum's workspace with them), replayed with new
    inputs and eager work in between."""
    need_gpu()
    d = lib()
    g = gen(14)
    x = torch.randn(66, 2048, generator=g, device="cuda").bfloat16()
    w, w2 = (torch.randn(96, 2048, generator=g, device="cuda").bfloat16()
             for _ in range(2))
    d.gated(x, w, w2)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        h, kg, ku = d.gated(x, w, w2, keep=True)
        grads = d.gated_backward(h, x, w, w2, kg, ku, bias=True)
    for k in range(4):
        x.copy_(torch.randn(66, 2048, generator=g, device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        h2, kg2, ku2 = d.gated(x, w, w2, keep=True)
        for a, b in zip((h, kg, ku) + grads, (h2, kg2, ku2)
                        + d.gated_backward(h2, x, w, w2, kg2, ku2,
                                           bias=True)):
            assert torch.equal(a, b)


@pytest.mark.parametrize("far", [(1 << 23) - 72, (1 << 23) + 8])
def test_rows_far_apart(far):
    """Row distances on both sides of where 256 rows leave 32-bit offsets; the
    last rows start past 2^32 bytes."""
    need_gpu()
    d = lib()
    rows, n_in, n_out = 280, 64, 24
    ld = n_in + far
    g = gen(15)
    buf = torch.empty((rows - 1) * ld + n_in, dtype=torch.bfloat16,
                      device="cuda")
    x = buf.as_strided((rows, n_in), (ld, 1))
    x.copy_(torch.randn(rows, n_in, generator=g, device="cuda"))
    w = torch.randn(n_out, n_in, generator=g, device="cuda").bfloat16()
    dy = torch.randn(rows, n_out, generator=g, device="cuda").bfloat16()
    want = ref.linear(np64(x), np64(w), None, None, "none", "bfloat16",
                      "bfloat16")
    close(d.linear(x, w), want["y"], "y")
    close(d.linear(x[-20:], w), tuple(v[-20:] for v in want["y"]), "last y")
    want = ref.linear_backward(np64(dy), np64(x), np64(w), None, "none",
                               "bfloat16", "bfloat16")
    dx, dw = d.linear_backward(dy, x, w)
    close(dx, want["dx"], "dx")
    close(dw, want["dwz"], "dw")


@pytest.mark.parametrize("p,rows,width,hidden", [(4, 24, 64, 96),
                                                 (2, 130, 72, 48),
                                                 (1, 5, 16, 16)])
def test_layer_split_over_ranks(p, rows, width, hidden):
    """The example: gated layer, reduction, gradients and their reduction,
    replayed from one graph, against the unsplit layer in 64 bits.  The hidden
    layer and its gradients are rounded to bfloat16 (2^-9, and the products
    that read them average it out), weights' and inputs' gradients follow."""
    need_gpu()
    import os
    import sys
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    sys.path.insert(0, os.path.join(root, "examples"))
    try:
        import split_layer
    finally:
        sys.path.pop(0)
    worst = split_layer.main(p, rows, width, hidden)
    assert worst["y"] < 2e-3
    for k in ("dx", "dwg", "dwu", "dw2"):
        assert worst[k] < 1e-2, (k, worst[k])
