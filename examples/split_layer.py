"""A gated feed-forward layer split over p ranks:
y = x + W2 (silu(Wg x) * Wu x).

Each rank holds n_hidden / p columns of the hidden layer: rows of Wg and Wu,
columns of W2.  Forward: the gated projections and the second product of all
ranks (two calls), the second with 32-bit partial sums, rank 0's with x added;
dpar_allreduce sums them and gives every rank the result.  Backward: the same
backwards, and dpar_allreduce sums the ranks' gradients of x.  All calls are
recorded into one HIP graph, which is replayed as a training program would.

    python examples/split_layer.py [ranks tokens width hidden]
"""

import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2109_12626_amd import dpar  # noqa: E402


class SplitLayer:
    """Weights, buffers and address arrays of one layer on one GPU."""

    def __init__(self, p, rows, width, hidden, seed=0, dtype=torch.bfloat16):
        if hidden % p:
            raise ValueError("the ranks share the hidden layer evenly")
        self.p, self.rows, self.width = p, rows, width
        self.part = part = hidden // p
        g = torch.Generator("cuda").manual_seed(seed)

        def normal(*shape, scale):
            return (torch.randn(*shape, generator=g, device="cuda")
                    * scale).to(dtype)

        def empty(*shape, dtype=dtype):
            return torch.empty(*shape, device="cuda", dtype=dtype)

        f32 = torch.float32
        self.wg, self.wu = (normal(p, part, width, scale=width ** -0.5)
                            for _ in range(2))
        self.w2 = normal(p, width, part, scale=hidden ** -0.5)
        self.x, self.dy = empty(rows, width), empty(rows, width)
        self.x32 = empty(rows, width, dtype=f32)
        self.h, self.g, self.u, self.dh, self.dg, self.du = (
            empty(p, rows, part) for _ in range(6))
        self.partial, self.y, self.dx_partial, self.dx = (
            empty(p, rows, width, dtype=f32) for _ in range(4))
        self.dwg, self.dwu = (empty(p, part, width, dtype=f32)
                              for _ in range(2))
        self.dw2 = torch.empty_like(self.w2)

        # addresses, options and workspace: made once, kept with the layer
        self.at = {k: dpar.rows(t) for k, t in vars(self).items()
                   if isinstance(t, torch.Tensor) and t.dim() == 3}
        for k in ("x", "dy"):
            self.at[k] = dpar.pointers([getattr(self, k).data_ptr()] * p)
        # only rank 0 adds x
        self.at["residual"] = dpar.pointers([self.x32.data_ptr()]
                                            + [0] * (p - 1))
        name = {torch.bfloat16: "bfloat16", torch.float16: "float16",
                torch.float32: "float32"}[dtype]
        opt = dpar.product_options
        self.first = opt(rows, width, part, name, act="silu")
        self.second = opt(rows, part, width, name, "float32")
        # gradients of the hidden layer and w2 in their type; of x, which the
        # reduction sums, and of the first weights in 32 bits
        self.second_back = opt(rows, part, width, name)
        self.first_back = opt(rows, width, part, name, "float32", act="silu")
        self.bytes = max(dpar.dpar_product_workspace(c, p, o) for c, o in (
            ("gated", self.first), ("linear", self.second),
            ("linear_backward", self.second_back),
            ("gated_backward", self.first_back)))
        self.ws = empty(max(self.bytes, 16), dtype=torch.uint8)

    def forward(self):
        a, s = self.at, torch.cuda.current_stream()
        ws = (self.ws, self.ws.numel(), s)
        self.x32.copy_(self.x)
        dpar.dpar_gated(a["x"], a["wg"], a["wu"], None, None, a["h"], a["g"],
                        a["u"], self.p, self.first, *ws)
        dpar.dpar_linear(a["h"], a["w2"], None, a["residual"], a["partial"],
                         None, self.p, self.second, *ws)
        dpar.dpar_allreduce(a["partial"], a["y"], self.p,
                            self.rows * self.width, "float32", "sum", 0, s)
        return self.y

    def backward(self):
        """dy -> dx (every rank's row), dwg, dwu, dw2."""
        a, s = self.at, torch.cuda.current_stream()
        ws = (self.ws, self.ws.numel(), s)
        dpar.dpar_linear_backward(a["dy"], a["h"], a["w2"], None, a["dh"],
                                  a["dw2"], None, None, self.p,
                                  self.second_back, *ws)
        dpar.dpar_gated_backward(a["dh"], a["x"], a["wg"], a["wu"], a["g"],
                                 a["u"], a["dx_partial"], a["dwg"], a["dwu"],
                                 None, None, a["dg"], a["du"], self.p,
                                 self.first_back, *ws)
        dpar.dpar_allreduce(a["dx_partial"], a["dx"], self.p,
                            self.rows * self.width, "float32", "sum", 0, s)
        self.dx += self.dy                     # the residual's path
        return self.dx

    def graph(self):
        """Both passes as one HIP graph (after an eager pass, which builds the
        reduction's tables)."""
        self.forward()
        self.backward()
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            self.forward()
            self.backward()
        return g


def reference(layer):
    """The unsplit layer in 64 bits: y, dx, dwg, dwu, dw2."""
    x, dy = layer.x.double(), layer.dy.double()
    wg, wu = (w.double().flatten(0, 1) for w in (layer.wg, layer.wu))
    w2 = layer.w2.double().transpose(0, 1).flatten(1)
    g, u = x @ wg.t(), x @ wu.t()
    s = torch.sigmoid(g)
    h = g * s * u
    dh = dy @ w2
    dg, du = dh * u * s * (1 + g * (1 - s)), dh * g * s
    dw2 = (dy.t() @ h).view(layer.width, layer.p, -1).transpose(0, 1)
    return {"y": x + h @ w2.t(), "dx": dy + dg @ wg + du @ wu,
            "dwg": (dg.t() @ x).view_as(layer.wg),
            "dwu": (du.t() @ x).view_as(layer.wu), "dw2": dw2}


def main(p=8, rows=1024, width=4096, hidden=16384, replays=3, seed=1):
    layer = SplitLayer(p, rows, width, hidden, seed)
    gen = torch.Generator("cuda").manual_seed(seed + 1)
    layer.x.normal_(generator=gen)
    layer.dy.normal_(generator=gen)
    graph = layer.graph()
    worst = {}
    for _ in range(replays):
        layer.x.normal_(generator=gen)
        layer.dy.normal_(generator=gen)
        graph.replay()
        torch.cuda.synchronize()
        want = reference(layer)
        got = {k: getattr(layer, k) for k in want}
        for i in range(p):                     # every rank holds y and dx
            for k in ("y", "dx"):
                if not torch.equal(got[k][i], got[k][0]):
                    raise AssertionError(f"{k} of rank {i} differs")
        got["y"], got["dx"] = got["y"][0], got["dx"][0]
        for k, v in want.items():
            e = float((got[k].double() - v).norm() / v.norm())
            worst[k] = max(worst.get(k, 0.0), e)
    begin, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    begin.record()
    for _ in range(10):
        graph.replay()
    end.record()
    end.synchronize()
    print(f"{p} ranks, {rows} x {width}, hidden {hidden}: "
          f"{begin.elapsed_time(end) / 10:.3f} ms per step; relative errors "
          + ", ".join(f"{k} {e:.1e}" for k, e in worst.items()), flush=True)
    return worst


if __name__ == "__main__":
    main(*[int(v) for v in sys.argv[1:5]])
