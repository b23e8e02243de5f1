"""8-bit layer products on the GPU against the definition in 64 bits (oracle/
products.py): quantised rows bit for bit, products element by element within the
bound of the stated roundings."""

import numpy as np
import pytest
import torch

from oracle import products as ref
from tests._gpu import lib, need_gpu

pytestmark = pytest.mark.gpu

TORCH = {"float32": torch.float32, "bfloat16": torch.bfloat16,
         "float16": torch.float16, "int8": torch.int8}
FILL = 77          # what lies between rows and after buffers


@pytest.fixture(autouse=True)
def gpu():
    need_gpu()


def np64(t):
    return t.double().cpu().numpy()


def gen(seed):
    return torch.Generator("cuda").manual_seed(seed)


class Ranks:
    """p matrices of rows x cols in one buffer, `far` elements between rows and
    `shift` before the first; everything else holds FILL."""

    def __init__(self, p, rows, cols, dtype, far=0, shift=0):
        self.ld = cols + far
        size = p * max(rows, 1) * self.ld + shift + 64
        self.flat = torch.full((size,), FILL, dtype=TORCH[dtype],
                               device="cuda")
        self.t = self.flat[shift:shift + p * rows * self.ld].view(
            p, rows, self.ld)[..., :cols]
        self.at = lib().pointers([self.t.data_ptr() + i * rows * self.ld
                                  * self.flat.element_size()
                                  for i in range(p)])

    def normal(self, g, scale=1.0):
        if self.flat.dtype == torch.int8:
            self.t.copy_(torch.randint(-128, 128, self.t.shape, generator=g,
                                       device="cuda", dtype=torch.int8))
        else:
            self.t.copy_(torch.randn(self.t.shape, generator=g,
                                     device="cuda") * scale)
        return self

    def gaps_untouched(self):
        mask = torch.ones_like(self.flat, dtype=torch.bool)
        p, rows, cols = self.t.shape
        start = self.t.storage_offset()
        if self.t.numel():
            mask[start:start + p * rows * self.ld].view(
                p, rows, self.ld)[..., :cols] = False
        return bool((self.flat[mask] == FILL).all())


def close(got, want, what):
    v, slack = want
    g = np64(got)
    assert g.shape == v.shape, (what, g.shape, v.shape)
    assert np.isfinite(g).all(), what
    bad = np.abs(g - v) > slack
    assert not bad.any(), (what, int(bad.sum()), np.argwhere(bad)[0],
                           g[bad][0], v[bad][0], slack[bad][0])


# ------------------------------------------------------------- quantisation

def run_quantize(x, far=0, shift=0):
    """x: [p, rows, cols] on the CPU, float32 values of `dtype`."""
    d = lib()
    p, rows, cols = x.shape
    name = {v: k for k, v in TORCH.items()}[x.dtype]
    xs = Ranks(p, rows, cols, name, far, shift)
    xs.t.copy_(x)
    q = Ranks(p, rows, cols, "int8", far, shift)
    s = Ranks(p, 1, rows, "float32", 0, shift)
    d.dpar_quantize(xs.at, q.at, s.at, p, d.quantize_options(
        rows, cols, name, xs.ld, q.ld), torch.cuda.current_stream())
    for i in range(p):
        want, scale = ref.quantize(np64(x[i]))
        np.testing.assert_array_equal(s.t[i, 0].cpu().numpy(), scale)
        np.testing.assert_array_equal(np64(q.t[i]), want)
    assert q.gaps_untouched() and s.gaps_untouched()


@pytest.mark.parametrize("dtype", ["bfloat16", "float16", "float32"])
@pytest.mark.parametrize("p,rows,cols,far,shift", [
    (1, 1, 1, 0, 0), (1, 1, 4096, 0, 0), (2, 3, 7, 1, 1), (1, 5, 8, 0, 0),
    (3, 17, 1001, 0, 0), (1, 2, 8191, 5, 3), (1, 3, 8200, 0, 0),
    (1, 2, 33000, 8, 0), (1, 2047, 65, 0, 0), (1, 2048, 64, 0, 0),
    (2, 2050, 515, 3, 1), (1, 2049, 4104, 0, 0), (50, 2, 100, 0, 0)])
def test_quantize(dtype, p, rows, cols, far, shift):
    g = torch.Generator().manual_seed(rows * cols)
    x = torch.randn(p, rows, cols, generator=g) \
        * torch.exp(3 * torch.randn(p, rows, 1, generator=g))
    run_quantize(x.to(TORCH[dtype]), far, shift)


@pytest.mark.parametrize("rows", [1, 2048])
@pytest.mark.parametrize("dtype", ["bfloat16", "float16", "float32"])
def test_quantize_halves(dtype, rows):
    """Quotients at and next to n + 1/2: the largest value 127 makes the scale
    1, other powers of two make it exact, and the rest lie beside a half."""
    half = torch.arange(-254, 255).float() / 2
    for most in (127.0, 63.5, 254.0, 0.99609375, 100.0):
        x = (half / 127 * most).to(TORCH[dtype])
        run_quantize(x.repeat(rows, 1)[None])
    x = half.clone().to(TORCH[dtype])
    if dtype == "float32":
        for step in (1, -1):
            near = torch.nextafter(half, torch.full_like(half, 1e9 * step))
            near[0] = -127
            near[-1] = 127
            run_quantize(near.clamp(-127, 127).repeat(rows, 1)[None])


@pytest.mark.parametrize("dtype", ["bfloat16", "float16", "float32"])
def test_quantize_smallest_and_largest(dtype):
    t = TORCH[dtype]
    fi = torch.finfo(t)
    tiny = {"float32": 2.0 ** -149, "bfloat16": 2.0 ** -133,
            "float16": 2.0 ** -24}[dtype]
    rows = [[0, 0, 0], [tiny, 0, -tiny], [63 * tiny, tiny, -tiny],
            [64 * tiny, 32 * tiny, -tiny], [190 * tiny, -189 * tiny, tiny],
            [fi.max, -fi.max, 1], [fi.tiny, fi.tiny / 2, -fi.tiny],
            [fi.max, fi.tiny, 0], [-0.0, 0.0, -0.0]]
    run_quantize(torch.tensor(rows, dtype=torch.float64).to(t)[None])


def test_quantize_infinities_and_nan():
    inf, nan = float("inf"), float("nan")
    run_quantize(torch.tensor([[[1.0, inf, 2], [nan, 1, 1], [1, 2, -inf],
                                [inf, nan, 0], [3, 4, 5]]]))


def test_quantize_nothing():
    d = lib()
    s = torch.full((3,), 5.0, device="cuda")
    d.dpar_quantize([0], [0], [s], 1, d.quantize_options(3, 0, "float16"),
                    torch.cuda.current_stream())
    assert (s == 0).all()
    d.dpar_quantize([0], [0], [0], 1, d.quantize_options(0, 5, "float16"),
                    torch.cuda.current_stream())


# ----------------------------------------------------------------- products

def scales(g, p, n, size, shift=0):
    """Of both signs, a zero among them."""
    r = Ranks(p, 1, n, "float32", 0, shift)
    r.normal(g, size)
    if n > 2:
        r.t[:, 0, n // 2] = 0
    return r


def operands(call, p, rows, n_in, n_out, out, bias, residual, far, shift,
             seed, shared):
    g = gen(seed)
    n = 2 if call == "gated" else 1
    x = Ranks(1 if shared else p, rows, n_in, "int8", far, shift).normal(g)
    sx = scales(g, 1 if shared else p, rows, 1 / 74, shift)
    w, sw, b = [], [], []
    for _ in range(n):
        w.append(Ranks(p, n_out, n_in, "int8", far, shift).normal(g))
        sw.append(scales(g, p, n_out, max(n_in, 1) ** -0.5 / 74, shift))
        b.append(Ranks(p, 1, n_out, out, 0, shift).normal(g) if bias
                 else None)
    r = Ranks(p, rows, n_out, out, far, shift).normal(g) if residual else None
    return x, sx, w, sw, b, r


def run_int8(call, p, rows, n_in, n_out, out="bfloat16", act="silu",
             bias=True, residual=True, far=0, shift=0, split=True,
             shared=False, seed=0):
    d = lib()
    residual = residual and call == "linear"
    x, sx, w, sw, b, r = operands(call, p, rows, n_in, n_out, out, bias,
                                  residual, far, shift, seed, shared)
    y = Ranks(p, rows, n_out, out, far, shift)
    opt = d.product_options(rows, n_in, n_out, "int8", out, act, ldx=x.ld,
                            ldw=w[0].ld, ldy=y.ld, ldr=n_out + far)
    n = d.dpar_product_workspace(call, p, opt) if split else 0
    ws = torch.empty(max(n, 16), dtype=torch.uint8, device="cuda") if n \
        else None

    def at(t):
        if t is None:
            return None
        return t.at if t.t.shape[0] == p else d.pointers(
            [t.t.data_ptr()] * p)

    stream = torch.cuda.current_stream()
    if call == "gated":
        d.dpar_gated_int8(at(x), at(sx), at(w[0]), at(sw[0]), at(w[1]),
                          at(sw[1]), at(b[0]), at(b[1]), y.at, p, opt, ws, n,
                          stream)
    else:
        d.dpar_linear_int8(at(x), at(sx), at(w[0]), at(sw[0]), at(b[0]),
                           at(r), y.at, p, opt, ws, n, stream)
    for i in range(p):
        j = 0 if shared else i
        one = [np64(x.t[j]), np64(sx.t[j, 0])]
        for k in range(len(w)):
            one += [np64(w[k].t[i]), np64(sw[k].t[i, 0])]
        one += [np64(t.t[i, 0]) if bias else None for t in b]
        if call == "gated":
            want = ref.gated_int8(*one, act, out)
        else:
            want = ref.linear_int8(*one, np64(r.t[i]) if residual else None,
                                   act, out)
        close(y.t[i], want, f"rank {i}")
    assert y.gaps_untouched()
    return y.t


ACTS = ["none", "relu", "gelu", "gelu_tanh", "silu"]
OUTS = ["bfloat16", "float16", "float32"]
# rows, in, out: one row to tiles of every size, whole pieces and odd widths
SIZES = [(1, 1, 1), (1, 16, 16), (1, 4096, 40), (3, 515, 33), (16, 1024, 200),
         (17, 512, 64), (31, 4112, 48), (33, 2000, 100), (48, 1040, 4096),
         (64, 512, 4096), (65, 300, 129), (128, 128, 64), (130, 1001, 257),
         (200, 2048, 384), (257, 784, 520)]


@pytest.mark.parametrize("k", range(len(SIZES)), ids=map(str, SIZES))
@pytest.mark.parametrize("call", ["linear", "gated"])
def test_products(call, k):
    run_int8(call, 1 + k % 3, *SIZES[k], out=OUTS[k % 3], act=ACTS[k % 5],
             seed=k)


@pytest.mark.parametrize("call", ["linear", "gated"])
@pytest.mark.parametrize("far,shift", [(1, 0), (16, 0), (5, 3), (0, 1)])
@pytest.mark.parametrize("rows,n_in,n_out", [(2, 528, 48), (70, 256, 72),
                                             (300, 640, 144)])
def test_distances_and_alignment(call, far, shift, rows, n_in, n_out):
    run_int8(call, 2, rows, n_in, n_out, out=OUTS[shift % 3], far=far,
             shift=shift, seed=rows)


@pytest.mark.parametrize("call", ["linear", "gated"])
@pytest.mark.parametrize("rows,n_in,n_out", [
    (256, 1024, 12288), (1024, 1152, 3328), (2048, 640, 4096)])
def test_large_tiles(call, rows, n_in, n_out):
    run_int8(call, 1, rows, n_in, n_out, out="bfloat16", seed=rows)


@pytest.mark.parametrize("call", ["linear", "gated"])
@pytest.mark.parametrize("rows,n_in,n_out", [(100, 16384, 64),
                                             (66, 9000, 100)])
def test_with_and_without_a_workspace(call, rows, n_in, n_out):
    """Integer sums: the same bits, however they are split."""
    for out in OUTS:
        a = run_int8(call, 2, rows, n_in, n_out, out=out)
        b = run_int8(call, 2, rows, n_in, n_out, out=out, split=False)
        assert torch.equal(a, b)


@pytest.mark.parametrize("call", ["linear", "gated"])
def test_empty_sizes(call):
    run_int8(call, 2, 5, 0, 7)
    run_int8(call, 2, 0, 5, 7)
    run_int8(call, 2, 5, 7, 0)


@pytest.mark.parametrize("rows", [1, 40, 300])
def test_largest_sums(rows):
    """-128 x -128 over the longest contraction: 2^31 - 2^14."""
    d = lib()
    n_in, n_out = 131071, 24
    x = torch.full((rows, n_in), -128, dtype=torch.int8, device="cuda")
    w = torch.full((n_out, n_in), -128, dtype=torch.int8, device="cuda")
    one = torch.ones(max(rows, n_out), device="cuda")
    y = d.linear_int8(x, one[:rows], w, one[:n_out], out_dtype=torch.float32)
    assert (y.double() == float(np.float32(131071 * 16384))).all()


@pytest.mark.parametrize("p", [48, 49, 100])
def test_many_ranks(p):
    run_int8("linear", p, 3, 64, 32, seed=p)
    run_int8("gated", p, 3, 48, 24, out="float32", seed=p, shared=True)


def test_scales_that_are_not_finite_stay_in_their_row():
    d = lib()
    g = gen(3)
    x = torch.randint(-9, 9, (20, 64), generator=g, device="cuda",
                      dtype=torch.int8)
    w = torch.randint(-9, 9, (32, 64), generator=g, device="cuda",
                      dtype=torch.int8)
    sx, sw = torch.ones(20, device="cuda"), torch.ones(32, device="cuda")
    clean = d.linear_int8(x, sx, w, sw, act="gelu")
    sx[4], sw[7] = float("nan"), float("inf")
    y = d.linear_int8(x, sx, w, sw, act="gelu")
    keep = torch.ones_like(y, dtype=torch.bool)
    keep[4] = False
    keep[:, 7] = False
    assert y[4].isnan().all() and torch.equal(y[keep], clean[keep])


def test_result_in_place_of_the_residual():
    d = lib()
    g = gen(5)
    x = torch.randint(-100, 100, (9, 256), generator=g, device="cuda",
                      dtype=torch.int8)
    w = torch.randint(-100, 100, (40, 256), generator=g, device="cuda",
                      dtype=torch.int8)
    sx, sw = torch.rand(9, device="cuda"), torch.rand(40, device="cuda")
    r = torch.randn(9, 40, generator=g, device="cuda").bfloat16()
    want = d.linear_int8(x, sx, w, sw, residual=r)
    opt = d.product_options(9, 256, 40, "int8", "bfloat16")
    d.dpar_linear_int8([x], [sx], [w], [sw], None, [r], [r], 1, opt, None, 0,
                       torch.cuda.current_stream())
    assert torch.equal(r, want)


def test_streams_and_a_graph():
    """Two streams with a workspace each, and a captured call that is replayed
    between eager ones."""
    d = lib()
    g = gen(7)
    rows, n_in, n_out = 96, 8192, 128
    x = torch.randn(rows, n_in, generator=g, device="cuda")
    w, sw = d.quantize(torch.randn(n_out, n_in, generator=g, device="cuda"))

    def layer(t):
        q, s = d.quantize(t)
        return d.linear_int8(q, s, w, sw, act="silu")

    want = layer(x)
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            got.append([layer(x) for _ in range(3)])
    for s in streams:
        torch.cuda.current_stream().wait_stream(s)
    assert all(torch.equal(y, want) for ys in got for y in ys)
    graph = torch.cuda.CUDAGraph()
    held = x.clone()
    with torch.cuda.graph(graph):
        y = layer(held)
    for k in range(4):
        held.copy_(x * (k + 1))
        graph.replay()
        assert torch.equal(y, layer(held))


def test_front_ends():
    d = lib()
    g = gen(11)
    x = torch.randn(2, 10, 96, generator=g, device="cuda").half()
    wide = torch.randn(10, 128, generator=g, device="cuda")
    q, s = d.quantize(x)
    assert q.shape == x.shape and s.shape == (2, 10)
    for i in range(2):
        a, b = d.quantize(x[i])
        assert torch.equal(a, q[i]) and torch.equal(b, s[i])
    a, b = d.quantize(wide[:, :96])
    c, e = d.quantize(wide[:, :96].contiguous())
    assert torch.equal(a, c) and torch.equal(b, e)
    w = torch.randint(-127, 128, (2, 40, 96), generator=g, device="cuda",
                      dtype=torch.int8)
    sw = torch.rand(2, 40, generator=g, device="cuda")
    y = d.linear_int8(q, s, w, sw)
    h = d.gated_int8(q, s, w, sw, w, sw, out_dtype=torch.float32)
    assert y.dtype == torch.bfloat16 and h.dtype == torch.float32
    for i in range(2):
        assert torch.equal(y[i], d.linear_int8(q[i], s[i], w[i], sw[i]))
        assert torch.equal(h[i], d.gated_int8(q[i], s[i], w[i], sw[i], w[i],
                                              sw[i],
                                              out_dtype=torch.float32))


def test_quantize_many_rows():
    """More workgroups than a launch has along its first axis."""
    d = lib()
    for rows, cols in ((2 ** 24 + 9, 3), (2 ** 22 + 3, 1025)):
        x = torch.randn(rows, cols, generator=gen(rows), device="cuda").half()
        q, scale = d.quantize(x)
        for part in (slice(0, 1000), slice(2 ** 22 - 500, 2 ** 22 + 500),
                     slice(rows - 1000, rows)):
            want, s = ref.quantize(np64(x[part]))
            np.testing.assert_array_equal(scale[part].cpu().numpy(), s)
            np.testing.assert_array_equal(np64(q[part]), want)


def apart(t, distance):
    """A copy of the rows of a matrix, `distance` elements apart."""
    n, cols = t.shape
    flat = torch.empty((n - 1) * distance + cols, dtype=t.dtype, device="cuda")
    far = flat.as_strided((n, cols), (distance, 1))
    far.copy_(t)
    return far


@pytest.mark.parametrize("n_in", [512, 515])
def test_distances_past_32_bits(n_in):
    d = lib()
    g = gen(5)
    x = torch.randn(9, n_in, generator=g, device="cuda").bfloat16()
    w = torch.randn(40, n_in, generator=g, device="cuda")
    r = torch.randn(9, 40, generator=g, device="cuda").bfloat16()
    far = apart(x, 2 ** 28 + 16)
    q, s = d.quantize(x)
    for a, b in zip(d.quantize(far), (q, s)):
        assert torch.equal(a, b)
    wq, sw = d.quantize(w)
    want = d.linear_int8(q, s, wq, sw, residual=r, act="gelu")
    got = d.linear_int8(apart(q, 2 ** 29 + 16), s, apart(wq, 2 ** 27 + 16), sw,
                        residual=apart(r, 2 ** 28 + 8), act="gelu")
    assert torch.equal(got, want)
    want = d.gated_int8(q, s, wq, sw, wq.flip(0).contiguous(), sw)
    got = d.gated_int8(apart(q, 2 ** 29 + 3), s, apart(wq, 2 ** 27 + 5), sw,
                       apart(wq.flip(0).contiguous(), 2 ** 27 + 5), sw)
    assert torch.equal(got, want)


@pytest.mark.parametrize("rows", [2, 40])
def test_values_between_rows_are_not_read(rows):
    """Scales and residual beside NaN, rows beside others."""
    d = lib()
    g = gen(6)
    nan = float("nan")
    x = torch.full((rows, 600), nan, device="cuda")
    x[:, :515] = torch.randn(rows, 515, generator=g, device="cuda")
    q, s = d.quantize(x[:, :515])
    assert torch.equal(q, d.quantize(x[:, :515].contiguous())[0])
    wq, sw = d.quantize(torch.randn(33, 515, generator=g, device="cuda"))
    r = torch.full((rows, 40), nan, device="cuda").bfloat16()
    r[:, :33] = 1
    got = d.linear_int8(q, s, wq, sw, residual=r[:, :33])
    assert torch.equal(got, d.linear_int8(q, s, wq, sw,
                                          residual=r[:, :33].contiguous()))
    assert got.isfinite().all()
