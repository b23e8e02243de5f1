"""The mixture-of-experts layer on the GPU against the definition in 64 bits
(oracle/products.py): the choice exactly, results element by element within the
bound of the stated roundings."""

import numpy as np
import pytest
import torch

from oracle import products as ref
from tests._gpu import lib, need_gpu
from tests.test_gpu_int8 import TORCH, Ranks, close, gen, np64

pytestmark = pytest.mark.gpu
INF, NAN = float("inf"), float("nan")


@pytest.fixture(autouse=True)
def gpu():
    need_gpu()


class Layer:
    """Operands of a layer whose matrices, rows and buffers may lie apart."""

    def __init__(self, p, tokens, n_in, hidden, experts, top,
                 dtype="bfloat16", weights=None, out=None, act="silu",
                 route="softmax", normalize=True, scale=1.0, residual=True,
                 far=0, shift=0, seed=0):
        d = lib()
        g = self.g = gen(seed)
        weights, out = weights or dtype, out or dtype
        self.p, self.tokens, self.top, self.experts = p, tokens, top, experts
        self.dtype, self.out, self.act = dtype, out, act
        self.route, self.normalize, self.scale = route, normalize, scale
        self.x = Ranks(1, tokens, n_in, dtype, far, shift).normal(g)
        eight = weights == "int8"

        def matrices(rows, cols):
            # `far` elements between rows, `far` between matrices too
            r = Ranks(p * experts, rows + (1 if far else 0), cols, weights,
                      far, shift)
            r.normal(g, max(cols, 1) ** -0.5)
            r.per = (rows + (1 if far else 0)) * r.ld
            r.ranks = d.pointers([
                r.t.data_ptr() + i * experts * r.per * r.t.element_size()
                for i in range(p)])
            r.m = r.t[:, :rows]
            return r

        def scales(n, size):
            r = Ranks(p, experts, n, "float32", 0, shift)
            r.normal(g, max(size, 1) ** -0.5 / 74)
            return r

        self.wg, self.wu = matrices(hidden, n_in), matrices(hidden, n_in)
        self.wd = matrices(n_in, hidden)
        self.s = [scales(hidden, n_in), scales(hidden, n_in),
                  scales(n_in, hidden)] if eight else None
        self.r = Ranks(p, tokens, n_in, out, far, shift).normal(g) \
            if residual else None
        self.y = Ranks(p, tokens, n_in, out, far, shift)
        self.logits = Ranks(1, tokens, p * experts, "float32", far,
                            shift).normal(g, 2.0)
        self.opt = d.moe_options(
            tokens, n_in, hidden, experts, top, dtype, weights, out, act,
            route, normalize, scale, self.x.ld, self.logits.ld, self.wg.ld,
            self.wd.ld, self.wg.per, self.wd.per, self.y.ld, n_in + far)
        n = d.dpar_moe_workspace(p, self.opt)
        self.ws = torch.full((max(n, 16),), 0xff, dtype=torch.uint8,
                             device="cuda")
        self.index = torch.full((tokens, top), 99, dtype=torch.int32,
                                device="cuda")
        self.weight = torch.full((tokens, top), 99.0, device="cuda")

    def run(self, given=None, stream=None, y=None):
        """given: (index, weight), the choice as an input."""
        d, p = lib(), self.p

        def every(t):
            return d.pointers([t.data_ptr()] * p)

        if given is None:
            choice = [d.pointers([t.data_ptr()] + [0] * (p - 1))
                      for t in (self.index, self.weight)]
        else:
            self.index, self.weight = given
            choice = [every(t) for t in given]
        d.dpar_moe(every(self.x.t), None if given else every(self.logits.t),
                   self.wg.ranks, self.wu.ranks, self.wd.ranks,
                   *([t.at for t in self.s] if self.s else [None] * 3),
                   self.r.at if self.r else None, y or self.y.at, *choice, p,
                   self.opt, self.ws, self.ws.numel(),
                   stream or torch.cuda.current_stream())

    def check(self, given=None):
        if given is None:
            index, weight = ref.choice(np64(self.logits.t[0]), self.top,
                                       self.route, self.normalize, self.scale)
            np.testing.assert_array_equal(self.index.cpu().numpy(), index)
            np.testing.assert_allclose(np64(self.weight), weight,
                                       rtol=2.0 ** -20, atol=2.0 ** -126)
        else:
            index, weight = given[0].cpu().numpy(), np64(given[1])
        n = self.experts
        for i in range(self.p):
            part = slice(i * n, (i + 1) * n)
            want = ref.moe(
                np64(self.x.t[0]), index, weight, np64(self.wg.m[part]),
                np64(self.wu.m[part]), np64(self.wd.m[part]),
                [np64(t.t[i]) for t in self.s] if self.s else None,
                np64(self.r.t[i]) if self.r else None, self.act, self.dtype,
                self.out, i * n, given is None)
            close(self.y.t[i], want, f"rank {i}")
        assert self.y.gaps_untouched()


def run_moe(*args, edit=None, **kw):
    layer = Layer(*args, **kw)
    if edit:
        edit(layer.logits.t[0])
    layer.run()
    layer.check()
    return layer


TYPES = [("bfloat16", "bfloat16", "bfloat16"),
         ("bfloat16", "bfloat16", "float32"),
         ("float16", "float16", "float16"), ("float16", "float16", "float32"),
         ("float32", "float32", "float32"), ("bfloat16", "int8", "bfloat16"),
         ("bfloat16", "int8", "float32"), ("float16", "int8", "float16"),
         ("float16", "int8", "float32")]
ACTS = ["none", "relu", "gelu", "gelu_tanh", "silu"]


@pytest.mark.parametrize("dtype,weights,out", TYPES)
@pytest.mark.parametrize("p,tokens,n_in,hidden,experts,top", [
    (1, 1, 64, 48, 4, 2), (1, 1, 1024, 528, 9, 3), (2, 5, 256, 64, 3, 4),
    (1, 16, 512, 128, 8, 2), (1, 17, 272, 80, 5, 5), (4, 33, 144, 176, 2, 3),
    (1, 128, 128, 96, 3, 2), (1, 100, 64, 32, 70, 6)])
def test_layer(dtype, weights, out, p, tokens, n_in, hidden, experts, top):
    run_moe(p, tokens, n_in, hidden, experts, top, dtype, weights, out,
            act=ACTS[tokens % 5], route=["softmax", "sigmoid"][top % 2],
            normalize=hidden % 32 == 0, scale=[1.0, 2.5][p % 2],
            residual=tokens % 2 == 1, seed=tokens)


@pytest.mark.parametrize("dtype,weights,out", TYPES)
@pytest.mark.parametrize("tokens,n_in,hidden,far,shift", [
    (1, 1, 1, 0, 0), (3, 33, 15, 0, 0), (20, 1001, 501, 0, 0),
    (2, 64, 48, 16, 0), (2, 64, 48, 5, 0), (2, 64, 48, 0, 1),
    (40, 65, 64, 0, 0), (40, 64, 65, 0, 0), (7, 2064, 1040, 0, 0)])
def test_odd_sizes_distances_and_alignment(dtype, weights, out, tokens, n_in,
                                           hidden, far, shift):
    run_moe(2, tokens, n_in, hidden, 3, 2, dtype, weights, out, far=far,
            shift=shift, seed=n_in)


@pytest.mark.parametrize("tokens", [1, 16, 64, 65, 128])
@pytest.mark.parametrize("dtype,weights", [("bfloat16", "bfloat16"),
                                           ("float32", "float32"),
                                           ("float16", "int8")])
@pytest.mark.parametrize("n_in,hidden", [(528, 272), (101, 67)])
def test_every_token_in_one_expert(tokens, dtype, weights, n_in, hidden):
    def one(logits):
        logits[:] = -INF
        logits[:, 2] = torch.arange(logits.shape[0])

    layer = run_moe(1, tokens, n_in, hidden, 4, 3, dtype, weights, edit=one)
    assert (layer.index == torch.tensor([2, -1, -1], device="cuda")).all()


@pytest.mark.parametrize("route", ["softmax", "sigmoid"])
@pytest.mark.parametrize("normalize", [False, True])
def test_masked_logits_ties_and_empty_tokens(route, normalize):
    def edit(logits):
        logits.copy_(torch.round(logits))            # ties
        logits[1] = -INF                             # no expert
        logits[2, 1:] = -INF                         # one
        logits[3] = 0
        logits[3, ::2] = -0.0                        # equal to 0
        logits[4] = 1e30
        logits[5] = -1e30
        logits[6, 3] = 1e38
        logits[7] = torch.finfo(torch.float32).min
        logits[8, :5] = -INF

    # by a launch of the choice, and by every expert's workgroups
    run_moe(2, 11, 64, 48, 12, 4, route=route, normalize=normalize, edit=edit,
            seed=3)
    layer = run_moe(2, 11, 64, 48, 6, 4, route=route, normalize=normalize,
                    edit=edit, seed=3)
    assert (layer.index[1] == -1).all() and (layer.weight[1] == 0).all()
    assert torch.equal(layer.y.t[0, 1], layer.r.t[0, 1])
    assert layer.index[3].tolist() == [0, 1, 2, 3]


def test_tokens_without_experts_only():
    def edit(logits):
        logits[:] = -INF

    layer = run_moe(1, 5, 64, 48, 6, 4, residual=False, edit=edit)
    assert (layer.y.t == 0).all()


@pytest.mark.parametrize("route", ["softmax", "sigmoid"])
@pytest.mark.parametrize("tokens", [6, 9])     # two ways of the choice
def test_infinities_and_nan_among_logits(route, tokens):
    layer = Layer(1, tokens, 64, 48, 5, 2, route=route)
    l = layer.logits.t[0]
    l[1, 3] = NAN
    l[2, 4] = INF
    l[3, 0], l[3, 2] = -INF, NAN
    l[4] = NAN
    layer.run()
    index, weight = ref.choice(np64(l), 2, route, True)
    np.testing.assert_array_equal(layer.index.cpu().numpy(), index)
    np.testing.assert_allclose(np64(layer.weight), weight, rtol=2.0 ** -20)
    y = layer.y.t[0]
    assert y[0].isfinite().all() and y[5].isfinite().all()
    for t in (1, 3, 4):
        assert y[t].isnan().all()


@pytest.mark.parametrize("weights", ["bfloat16", "int8"])
def test_values_that_are_not_finite_stay_in_their_token(weights):
    clean = Layer(1, 20, 72, 40, 4, 2, weights=weights, seed=5)
    clean.run()
    for v in (INF, NAN):
        layer = Layer(1, 20, 72, 40, 4, 2, weights=weights, seed=5)
        layer.x.t[0, 7, 3] = v
        layer.run()
        keep = torch.arange(20, device="cuda") != 7
        assert torch.equal(layer.y.t[0, keep], clean.y.t[0, keep])
        assert not layer.y.t[0, 7].isfinite().all()


@pytest.mark.parametrize("dtype,weights,out", TYPES)
def test_choice_as_an_input(dtype, weights, out):
    layer = Layer(2, 30, 128, 64, 4, 5, dtype, weights, out, seed=9)
    g = layer.g
    index = torch.randint(-2, 10, (30, 5), generator=g, device="cuda",
                          dtype=torch.int32)
    index[3] = 6                                   # the same one five times
    index[4] = torch.tensor([1, 7, 1, 7, 1])
    index[5] = -1
    index[6, 0], index[6, 1] = 2 ** 31 - 1, -2 ** 31
    weight = torch.randn(30, 5, generator=g, device="cuda")
    held = index.clone(), weight.clone()
    layer.run((index, weight))
    layer.check((index, weight))
    assert torch.equal(index, held[0]) and torch.equal(weight, held[1])


@pytest.mark.parametrize("p,tokens,experts,top", [
    (3, 1, 5, 4), (2, 8, 40, 3), (3, 30, 4, 2), (2, 20, 100, 5),
    (34, 3, 2, 4), (35, 40, 1, 3)])
@pytest.mark.parametrize("given", [False, True])
def test_ranks_with_a_choice_of_their_own(p, tokens, experts, top, given):
    """Every rank chooses from its own logits (or by its own index and weight)
    and sums what its experts contribute by that choice."""
    d = lib()
    layer = Layer(p, tokens, 72, 40, experts, top, seed=tokens)
    g = layer.g
    every = d.pointers([layer.x.t.data_ptr()] * p)
    logits = torch.randn(p, tokens, p * experts, generator=g, device="cuda")
    index = torch.full((p, tokens, top), 99, dtype=torch.int32, device="cuda")
    weight = torch.zeros(p, tokens, top, device="cuda")
    if given:
        index = torch.randint(-1, p * experts, index.shape, generator=g,
                              device="cuda", dtype=torch.int32)
        weight = torch.randn(weight.shape, generator=g, device="cuda")
    layer.opt.ldl = 0
    d.dpar_moe(every, None if given else d.rows(logits), layer.wg.ranks,
               layer.wu.ranks, layer.wd.ranks, None, None, None, layer.r.at,
               layer.y.at, d.rows(index), d.rows(weight), p, layer.opt,
               layer.ws, layer.ws.numel(), torch.cuda.current_stream())
    for i in range(p):
        if given:
            chosen = index[i].cpu().numpy(), np64(weight[i])
        else:
            chosen = ref.choice(np64(logits[i]), top, "softmax", True)
            np.testing.assert_array_equal(index[i].cpu().numpy(), chosen[0])
            np.testing.assert_allclose(np64(weight[i]), chosen[1],
                                       rtol=2.0 ** -20)
        part = slice(i * experts, (i + 1) * experts)
        want = ref.moe(np64(layer.x.t[0]), *chosen, np64(layer.wg.m[part]),
                       np64(layer.wu.m[part]), np64(layer.wd.m[part]), None,
                       np64(layer.r.t[i]), "silu", "bfloat16", "bfloat16",
                       i * experts, not given)
        close(layer.y.t[i], want, f"rank {i}")


def test_given_as_chosen():
    a = run_moe(4, 21, 64, 80, 5, 3, seed=1)
    b = Layer(4, 21, 64, 80, 5, 3, seed=1)
    b.run((a.index, a.weight))
    assert torch.equal(a.y.t, b.y.t)


def test_largest_counts():
    run_moe(1, 128, 32, 16, 1024, 16, seed=2)
    run_moe(64, 9, 32, 32, 16, 16, out="float32", seed=3)
    run_moe(33, 2, 32, 16, 1, 16, seed=4)


@pytest.mark.parametrize("tokens,n_in,hidden", [(0, 64, 48), (3, 0, 48),
                                                (3, 64, 0)])
def test_empty_sizes(tokens, n_in, hidden):
    run_moe(2, tokens, n_in, hidden, 3, 2)


def test_wide_layers():
    run_moe(1, 3, 8192, 48, 3, 2, seed=1)
    run_moe(1, 3, 48, 8192, 3, 2, out="float32", seed=2)
    run_moe(1, 20, 4100, 2052, 2, 1, "float16", seed=3)


def test_runs_are_the_same_bits():
    for kw in (dict(p=1, tokens=50, n_in=256, hidden=512, experts=16, top=4),
               dict(p=1, tokens=1, n_in=1024, hidden=512, experts=16, top=4)):
        layer = run_moe(**kw, out="float32")
        first = layer.y.t.clone()
        for _ in range(10):
            layer.ws.fill_(0x5a)
            layer.run()
            assert torch.equal(layer.y.t, first)


def test_result_in_place_of_the_residual():
    a = run_moe(2, 9, 64, 48, 3, 2, seed=6)
    b = Layer(2, 9, 64, 48, 3, 2, seed=6)
    b.run(y=b.r.at)
    assert torch.equal(b.r.t, a.y.t)


def test_streams_and_a_graph():
    layers = [Layer(1, t, 512, 256, 16, 4, seed=t) for t in (1, 24)]
    want = []
    for layer in layers:
        layer.run()
        want.append(layer.y.t.clone())
    streams = [torch.cuda.Stream() for _ in layers]
    for s, layer in zip(streams, layers):
        layer.y.t.zero_()
        s.wait_stream(torch.cuda.current_stream())
        for _ in range(5):
            layer.run(stream=s)
    for s, layer, w in zip(streams, layers, want):
        torch.cuda.current_stream().wait_stream(s)
        assert torch.equal(layer.y.t, w)
    for layer in layers:
        layer.run()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            layer.run()
        for k in range(4):
            layer.logits.t.copy_(layer.logits.t.roll(1, -1))
            layer.run()
            eager, index = layer.y.t.clone(), layer.index.clone()
            layer.y.t.zero_()
            graph.replay()
            assert torch.equal(layer.y.t, eager)
            assert torch.equal(layer.index, index)


def test_a_workspace_shared_in_turn():
    """A capture's workspace that an eager call of another size uses between
    replays."""
    d = lib()
    a, b = Layer(1, 8, 256, 64, 8, 2), Layer(1, 30, 128, 96, 4, 3, seed=2)
    a.ws = b.ws = torch.empty(max(a.ws.numel(), b.ws.numel()),
                              dtype=torch.uint8, device="cuda")
    a.run()
    want = a.y.t.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a.run()
    for _ in range(3):
        b.run()
        b.check()
        a.y.t.zero_()
        graph.replay()
        assert torch.equal(a.y.t, want)
    assert d.dpar_last_error() == ""


def test_front_end():
    d = lib()
    g = gen(4)

    def normal(*shape, dtype=torch.bfloat16):
        return (torch.randn(*shape, generator=g, device="cuda")
                * shape[-1] ** -0.5).to(dtype)

    x = normal(6, 64) * 8
    wg, wu, wd = normal(4, 48, 64), normal(4, 48, 64), normal(4, 64, 48)
    logits = normal(6, 4, dtype=torch.float32)
    y, index, weight = d.moe(x, logits, wg, wu, wd, 2)
    again, _, _ = d.moe(x, None, wg, wu, wd, index=index, weight=weight)
    assert torch.equal(y, again)
    ranks = [t.view(2, 2, *t.shape[1:]) for t in (wg, wu, wd)]
    parts, i2, w2 = d.moe(x, logits, *ranks, 2, out_dtype=torch.float32)
    assert parts.shape == (2, 6, 64) and torch.equal(i2, index)
    whole, _, _ = d.moe(x, logits, wg, wu, wd, 2, out_dtype=torch.float32)
    assert torch.allclose(parts.sum(0), whole, rtol=0, atol=1e-5)
    # 8-bit weights as dpar.quantize makes them
    q = [d.quantize(t) for t in (wg, wu, wd)]
    near, _, _ = d.moe(x, logits, *(a for a, _ in q), 2, *(b for _, b in q),
                       residual=y)
    assert near.shape == y.shape
    assert ((near - y).float() - y.float()).norm() < 0.05 * y.float().norm()


def poison_gaps(r):
    """NaN between a matrix's rows and after it."""
    keep = r.t.clone()
    r.flat.fill_(NAN)
    r.t.copy_(keep)


@pytest.mark.parametrize("dtype", ["bfloat16", "float16", "float32"])
@pytest.mark.parametrize("tokens,n_in,hidden,far,shift", [
    (1, 72, 40, 8, 0), (5, 101, 67, 3, 1), (30, 264, 136, 8, 0),
    (30, 333, 77, 5, 3), (100, 67, 131, 1, 0)])
def test_nan_between_rows_and_matrices(dtype, tokens, n_in, hidden, far,
                                       shift):
    layer = Layer(2, tokens, n_in, hidden, 4, 3, dtype, far=far, shift=shift)
    for r in (layer.x, layer.r, layer.logits):
        poison_gaps(r)
    for r in (layer.wg, layer.wu, layer.wd):
        poison_gaps(r)
        r.t[:, r.m.shape[1]:] = NAN
    layer.run()
    layer.check()


# tokens: the choice within the projections, by a launch, by every expert
@pytest.mark.parametrize("tokens,experts", [(1, 8), (6, 8), (20, 32), (40, 8)])
@pytest.mark.parametrize("dtype", ["bfloat16", "float16", "float32"])
def test_experts_that_nobody_chose_are_not_read(dtype, tokens, experts):
    clean = Layer(1, tokens, 128, 64, experts, 2, dtype, seed=7)
    clean.logits.t[..., ::2] = -INF
    clean.run()
    clean.check()
    layer = Layer(1, tokens, 128, 64, experts, 2, dtype, seed=7)
    layer.logits.t[..., ::2] = -INF
    for r in (layer.wg, layer.wu, layer.wd):
        r.m[::2] = NAN
    layer.run()
    assert torch.equal(layer.y.t, clean.y.t)


@pytest.mark.parametrize("tokens", [1, 6, 20, 40])
@pytest.mark.parametrize("dtype", ["bfloat16", "float16", "float32"])
def test_weights_that_are_not_finite_stay_with_their_expert(dtype, tokens):
    clean = Layer(1, tokens, 128, 64, 6, 2, dtype, seed=8)
    clean.run()
    for which in (0, 2):
        for v in (INF, NAN):
            layer = Layer(1, tokens, 128, 64, 6, 2, dtype, seed=8)
            (layer.wg, layer.wu, layer.wd)[which].m[3, 17, 5] = v
            layer.run()
            chose = (layer.index == 3).any(1)
            touched = torch.zeros_like(layer.y.t[0], dtype=torch.bool)
            if which == 2:
                touched[chose, 17] = True
                assert not layer.y.t[0, chose, 17].isfinite().any()
            else:
                touched[chose] = True
                # (silu of -inf is 0, so an infinity may leave no trace)
                if v != v:
                    assert layer.y.t[0, chose].isnan().all()
            assert torch.equal(layer.y.t[0][~touched], clean.y.t[0][~touched])


def apart(t, distance):
    """A copy of the rows of a matrix, `distance` elements apart."""
    n = t.shape[0]
    flat = torch.empty((n - 1) * distance + t[0].numel(), dtype=t.dtype,
                       device="cuda")
    far = flat.as_strided(t.shape, (distance,) + t[0].stride())
    far.copy_(t)
    return far


@pytest.mark.parametrize("tokens,dtype,n_in,hidden", [
    (2, "bfloat16", 128, 64), (9, "bfloat16", 136, 72), (9, "float16", 101, 67),
    (3, "float32", 64, 36)])
def test_distances_past_32_bits(tokens, dtype, n_in, hidden):
    """Rows and experts more than 2^32 bytes apart in all."""
    d = lib()
    g = gen(9)
    t = TORCH[dtype]

    def normal(*shape, dtype=t):
        return (torch.randn(*shape, generator=g, device="cuda")
                * shape[-1] ** -0.5).to(dtype)

    x, r = normal(tokens, n_in) * 8, normal(tokens, n_in)
    logits = normal(tokens, 3, dtype=torch.float32)
    w = [normal(3, hidden, n_in), normal(3, hidden, n_in),
         normal(3, n_in, hidden)]
    want, index, weight = d.moe(x, logits, *w, 2, residual=r)
    rows = (2 ** 32 // (tokens - 1) // x.element_size() // 16 + 5) * 16
    far = [apart(m, 2 ** 32 // x.element_size() // 2 + 48) for m in w]
    got = d.moe(apart(x, rows), apart(logits, 2 ** 30 // (tokens - 1) + 3),
                *far, 2, residual=apart(r, rows))
    for a, b in zip(got, (want, index, weight)):
        assert torch.equal(a, b)


CHOICES = [(1, 64, 8), (6, 8, 2), (16, 64, 2), (40, 8, 2)]


@pytest.mark.parametrize("n_in,hidden", [(512, 256), (333, 131)])
def test_every_way_of_the_choice_on_streams_and_in_graphs(n_in, hidden):
    """Layers of every kind in turn on two streams, then recorded together, with
    a workspace each, and replayed beside an eager call on another stream."""
    layers = [Layer(1, t, n_in, hidden, e, k, seed=t) for t, e, k in CHOICES]
    other = [Layer(1, t, n_in, hidden, e, k, seed=t) for t, e, k in CHOICES]
    want = []
    for layer in layers:
        layer.run()
        layer.check()
        want.append(layer.y.t.clone())
    streams = [torch.cuda.Stream() for _ in range(2)]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        for a, b in zip(layers, reversed(other)):
            a.run(stream=streams[0])
            b.run(stream=streams[1])
    for s in streams:
        torch.cuda.current_stream().wait_stream(s)
    for a, b, w in zip(layers, other, want):
        assert torch.equal(a.y.t, w) and torch.equal(b.y.t, w)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for layer in layers:
            layer.run()
    for k in range(3):
        for a, b in zip(layers, other):
            rolled = a.logits.t.roll(k + 1, -1)
            a.logits.t.copy_(rolled)
            b.logits.t.copy_(rolled)
            a.y.t.zero_()
        streams[0].wait_stream(torch.cuda.current_stream())
        graph.replay()
        for b in other:
            b.run(stream=streams[0])
        torch.cuda.current_stream().wait_stream(streams[0])
        for a, b in zip(layers, other):
            b.check()
            assert torch.equal(a.y.t, b.y.t)
            assert torch.equal(a.index, b.index)


# tokens: by token, by expert with one and with two tiles of pairs
@pytest.mark.parametrize("tokens,experts,top", [(1, 4, 2), (6, 16, 3),
                                                (40, 64, 3), (48, 4, 2)])
@pytest.mark.parametrize("dtype,weights", [
    ("bfloat16", "bfloat16"), ("float16", "float16"), ("bfloat16", "int8"),
    ("float16", "int8")])
@pytest.mark.parametrize("n_in,hidden", [(256, 1024), (101, 67)])
def test_16_bit_results_are_32_bit_ones_rounded(tokens, experts, top, dtype,
                                                weights, n_in, hidden):
    """Nothing between the sums is held to fewer than 32 bits."""
    args = (1, tokens, n_in, hidden, experts, top, dtype, weights)
    one, whole = (run_moe(*args, out, residual=False, seed=tokens)
                  for out in (dtype, "float32"))
    assert torch.equal(one.y.t, whole.y.t.to(TORCH[dtype]))


@pytest.mark.parametrize("tokens,experts", [(1, 2), (6, 2), (20, 16), (40, 2)])
@pytest.mark.parametrize("n_in,hidden", [(256, 128), (101, 67), (48, 256)])
@pytest.mark.parametrize("dtype", ["bfloat16", "float16", "float32"])
@pytest.mark.parametrize("out", ["same", "float32"])
def test_infinities_of_the_second_product(tokens, experts, n_in, hidden,
                                          dtype, out):
    """An infinity of wd gives one of the sum's sign (it meets values of few
    bits too), two of opposite signs NaN, and one beside a hidden value of 0
    NaN."""
    layer = Layer(1, tokens, n_in, hidden, experts, 1, dtype,
                  out=dtype if out == "same" else out, act="none",
                  residual=False, seed=3)
    layer.logits.t.fill_(-1)
    layer.logits.t[..., 1] = 1
    # hidden values 1, 2, 3 ..: of few bits; the fifth one is 0
    layer.x.t.zero_()
    layer.x.t[..., 0] = 1
    layer.wg.m.zero_()
    layer.wu.m.zero_()
    values = torch.arange(hidden, device="cuda") % 7 + 1.0
    values[::2] *= -1
    layer.wg.m[1, :, 0] = values.to(layer.wg.t.dtype)
    layer.wu.m[1, :, 0] = 1
    layer.wg.m[1, 4, 0] = 0
    h = layer.wg.m[1, :, 0].float()
    w = layer.wd.m[1]
    w[3, 1] = INF
    w[5, 2] = INF
    w[7, hidden - 1] = -INF
    w[11, 8], w[11, 9] = INF, INF               # opposite signs of h
    w[13, 4] = INF                              # beside 0
    w[17, 6] = NAN
    layer.run()
    want = (w.float() * h).sum(1)
    assert want[3] == INF and want[5] == -INF and want[11].isnan()
    assert want[13].isnan() and want[17].isnan()
    y = layer.y.t[0].float()
    special = ~want.isfinite()
    assert y[:, ~special].isfinite().all()
    for t in range(tokens):
        assert torch.equal(y[t, special].nan_to_num(nan=5.0),
                           want[special].nan_to_num(nan=5.0)), t


@pytest.mark.parametrize("tokens,experts", [(1, 2), (6, 2), (20, 16), (40, 2)])
@pytest.mark.parametrize("dtype,weights", [
    ("bfloat16", "bfloat16"), ("float16", "float16"), ("float32", "float32"),
    ("bfloat16", "int8"), ("float16", "int8")])
@pytest.mark.parametrize("n_in,hidden", [(128, 64), (32, 256)])
@pytest.mark.parametrize("out", ["same", "float32"])
def test_an_infinite_hidden_value(tokens, experts, dtype, weights, n_in,
                                  hidden, out):
    """Beside weights of few bits, of either sign and of 0."""
    layer = Layer(1, tokens, n_in, hidden, experts, 1, dtype, weights,
                  out=dtype if out == "same" else out, act="none",
                  residual=False, seed=3)
    layer.logits.t.fill_(-1)
    layer.logits.t[..., 1] = 1
    layer.x.t.fill_(0)
    layer.x.t[..., 0] = 1
    layer.x.t[0, 0, 1] = INF                    # of the first token
    for r in (layer.wg, layer.wu):
        r.m.zero_()
        r.m[1, :, :2] = 1
    if layer.s:
        for s in layer.s:
            s.t.fill_(1)
    w = layer.wd.m[1]
    w[:, 1:] = w[:, :1]                         # one sign a row
    w[9] = 0
    w[10] = 1
    w[10, 3] = -1
    layer.run()
    want = (w.float() * INF).sum(1)
    assert want[9].isnan() and want[10].isnan()
    assert (want == INF).any() and (want == -INF).any()
    y = layer.y.t[0].float()
    assert torch.equal(y[0].nan_to_num(nan=5.0), want.nan_to_num(nan=5.0))
    assert y[1:].isfinite().all()
