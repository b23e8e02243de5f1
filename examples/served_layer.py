"""A served block split over p ranks: a gated feed-forward layer with 8-bit
weights and activations, and a mixture-of-experts layer with 8-bit experts,

    y = x + W2 (silu(Wg x) * Wu x),    out = y + MoE(y).

Each rank holds n_hidden / p columns of the first layer and n_experts / p experts
of the second.  First layer: the tokens to 8 bits, the gated projections, their
result to 8 bits, the second product with 32-bit partial sums, rank 0's with x
added; dpar_allreduce sums them.  Second: the router's logits (one 16-bit
product), every rank's experts with 32-bit partial sums, rank 0's with y added;
dpar_allreduce again.  All calls are recorded into one HIP graph, which is
replayed as a serving program would.

    python examples/served_layer.py [ranks tokens width hidden experts top]
"""

import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2109_12626_amd import dpar  # noqa: E402


class ServedBlock:
    """Weights, buffers and address arrays of one block on one GPU."""

    def __init__(self, p, tokens, width, hidden, experts, inner, top, seed=0):
        if hidden % p or experts % p:
            raise ValueError("the ranks share hidden layer and experts evenly")
        self.p, self.tokens, self.width = p, tokens, width
        g = torch.Generator("cuda").manual_seed(seed)
        part, own = hidden // p, experts // p

        def normal(*shape):
            return (torch.randn(*shape, generator=g, device="cuda")
                    * shape[-1] ** -0.5).bfloat16()

        def empty(*shape, dtype=torch.bfloat16):
            return torch.empty(*shape, device="cuda", dtype=dtype)

        # weights to 8 bits, a scale per row: once, where the program starts
        self.wg, self.wu, self.w2 = (
            dpar.quantize(normal(p, part, width)),
            dpar.quantize(normal(p, part, width)),
            dpar.quantize(normal(p, width, part)))

        def expert_matrices(rows, cols):
            q, s = dpar.quantize(normal(experts * rows, cols))
            return q.view(p, own, rows, cols), s.view(p, own, rows)

        self.eg, self.eu = (expert_matrices(inner, width) for _ in range(2))
        self.ed = expert_matrices(width, inner)
        self.router = normal(experts, width)

        f32, i8 = torch.float32, torch.int8
        self.x = empty(tokens, width)
        self.x32, self.out = empty(tokens, width, dtype=f32), \
            empty(p, tokens, width, dtype=f32)
        self.xq, self.xs = empty(tokens, width, dtype=i8), \
            empty(tokens, dtype=f32)
        self.h = empty(p, tokens, part)
        self.hq, self.hs = empty(p, tokens, part, dtype=i8), \
            empty(p, tokens, dtype=f32)
        self.partial, self.y = (empty(p, tokens, width, dtype=f32)
                                for _ in range(2))
        self.y16 = empty(tokens, width)
        self.logits = empty(1, tokens, experts, dtype=f32)
        self.index = empty(tokens, top, dtype=torch.int32)
        self.weight = empty(tokens, top, dtype=f32)

        self.gated = dpar.product_options(tokens, width, part, "int8",
                                          "bfloat16", "silu")
        self.second = dpar.product_options(tokens, part, width, "int8",
                                           "float32")
        self.route = dpar.product_options(tokens, width, experts, "bfloat16",
                                          "float32")
        self.moe = dpar.moe_options(tokens, width, inner, own, top, "bfloat16",
                                    "int8", "float32")
        sizes = [dpar.dpar_product_workspace("gated", p, self.gated),
                 dpar.dpar_product_workspace("linear", p, self.second),
                 dpar.dpar_product_workspace("linear", 1, self.route),
                 dpar.dpar_moe_workspace(p, self.moe)]
        # (the calls follow one another on one stream and share a workspace)
        self.ws = empty(max(sizes), dtype=torch.uint8)
        self.ws_bytes = self.ws.numel()

    def step(self):
        """One pass: x to out, every rank's the same."""
        d, p, s = dpar, self.p, torch.cuda.current_stream()

        def every(t):
            return d.pointers([t.data_ptr()] * p)

        def first(t):                   # rank 0 only
            return d.pointers([t.data_ptr()] + [0] * (p - 1))

        def at(pair):
            return [d.rows(t) for t in pair]

        work = (self.ws, self.ws_bytes, s)
        n = self.tokens * self.width
        self.x32.copy_(self.x)
        d.dpar_quantize([self.x], [self.xq], [self.xs], 1,
                        d.quantize_options(*self.x.shape, "bfloat16"), s)
        d.dpar_gated_int8(every(self.xq), every(self.xs), *at(self.wg),
                          *at(self.wu), None, None, d.rows(self.h), p,
                          self.gated, *work)
        d.dpar_quantize(d.rows(self.h), d.rows(self.hq), d.rows(self.hs), p,
                        d.quantize_options(*self.h.shape[1:], "bfloat16"), s)
        d.dpar_linear_int8(d.rows(self.hq), d.rows(self.hs), *at(self.w2),
                           None, first(self.x32), d.rows(self.partial), p,
                           self.second, *work)
        d.dpar_allreduce(d.rows(self.partial), d.rows(self.y), p, n,
                         "float32", "sum", 0, s)
        self.y16.copy_(self.y[0])
        d.dpar_linear([self.y16], [self.router], None, None,
                      d.rows(self.logits), None, 1, self.route, *work)
        (eg, sg), (eu, su), (ed, sd) = (at(t) for t in (self.eg, self.eu,
                                                        self.ed))
        d.dpar_moe(every(self.y16), every(self.logits), eg, eu, ed, sg, su, sd,
                   first(self.y[0]), d.rows(self.partial), first(self.index),
                   first(self.weight), p, self.moe, *work)
        d.dpar_allreduce(d.rows(self.partial), d.rows(self.out), p, n,
                         "float32", "sum", 0, s)

    def record(self):
        self.step()                     # stages the reduction's arrays
        torch.cuda.synchronize()
        self.graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(self.graph):
            self.step()
        return self.graph

    def reference(self):
        """The block in 64 bits from the 8-bit weights, x in its 16 bits, without
        the activations' way to 8 bits: (out, chosen experts)."""
        def whole(pair):
            q, s = pair
            return q.double() * s.double()[..., None]

        act = torch.nn.functional.silu
        x = self.x.double()
        wg, wu, w2 = (whole(t) for t in (self.wg, self.wu, self.w2))
        y = x + sum(act(x @ a.t()) * (x @ b.t()) @ c.t()
                    for a, b, c in zip(wg, wu, w2))
        eg, eu, ed = (whole(t).flatten(0, 1) for t in (self.eg, self.eu,
                                                       self.ed))
        out = y.clone()
        for t in range(self.tokens):    # the experts that were chosen
            for e, w in zip(self.index[t].tolist(), self.weight[t].double()):
                out[t] += w * (ed[e] @ (act(eg[e] @ y[t]) * (eu[e] @ y[t])))
        return out


def main(argv):
    p, tokens, width, hidden, experts, top = (
        [int(v) for v in argv] + [8, 16, 2048, 8192, 64, 4][len(argv):])
    block = ServedBlock(p, tokens, width, hidden, experts, 1024, top)
    block.x.normal_()
    graph = block.record()
    for _ in range(5):
        graph.replay()
    a, b = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    a.record()
    for _ in range(50):
        graph.replay()
    b.record()
    torch.cuda.synchronize()
    want = block.reference()
    off = ((block.out[0].double() - want).norm() / want.norm()).item()
    print(f"{p} ranks, {tokens} tokens, {width} wide, {hidden} hidden, {top} of "
          f"{experts} experts of 1024: {a.elapsed_time(b) * 20:.1f} us a "
          f"step, {off:.2%} off the same block with 64-bit activations")
    del block, graph
    dpar.dpar_finalize()       # what a recorded reduction holds


if __name__ == "__main__":
    main(sys.argv[1:])
