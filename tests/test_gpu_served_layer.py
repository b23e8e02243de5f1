"""The 8-bit products, the mixture-of-experts layer and the reduction together,
as a served block calls them (examples/served_layer.py): each step against the
definition in 64 bits of what the step before it gave, and a recorded block
against eager ones."""

import os
import sys

import numpy as np
import pytest
import torch

from oracle import products as ref
from tests._gpu import lib, need_gpu
from tests.test_gpu_int8 import close, np64

pytestmark = pytest.mark.gpu
EXAMPLES = os.path.join(os.path.dirname(os.path.dirname(
    os.path.abspath(__file__))), "examples")


@pytest.fixture(autouse=True)
def release():
    """A recorded reduction keeps its table of addresses until dpar_finalize, of
    which there are few: later tests record too."""
    need_gpu()
    yield
    torch.cuda.synchronize()
    lib().dpar_finalize()


def block(*args):
    need_gpu()
    sys.path.insert(0, EXAMPLES)
    try:
        import served_layer
    finally:
        sys.path.remove(EXAMPLES)
    return served_layer.ServedBlock(*args)


@pytest.mark.parametrize("args", [(4, 6, 128, 256, 8, 64, 3),
                                  (3, 1, 200, 105, 6, 51, 2),
                                  (2, 40, 256, 512, 4, 96, 1)])
def test_steps(args):
    b = block(*args)
    p, tokens = b.p, b.tokens
    b.x.normal_()
    b.step()
    q, s = ref.quantize(np64(b.x))
    np.testing.assert_array_equal(np64(b.xq), q)
    np.testing.assert_array_equal(b.xs.cpu().numpy(), s)
    parts = np.zeros((tokens, b.width))
    slack = np.zeros_like(parts)
    for i in range(p):
        close(b.h[i], ref.gated_int8(
            q, s.astype(np.float64), *(np64(t[i]) for t in (*b.wg, *b.wu)),
            None, None, "silu", "bfloat16"), f"h of rank {i}")
        hq, hs = ref.quantize(np64(b.h[i]))
        np.testing.assert_array_equal(np64(b.hq[i]), hq)
        np.testing.assert_array_equal(b.hs[i].cpu().numpy(), hs)
        v, e = ref.linear_int8(hq, hs.astype(np.float64),
                               *(np64(t[i]) for t in b.w2), None,
                               np64(b.x) if i == 0 else None, "none",
                               "float32")
        parts += v
        # the reduction's additions, each rounded once
        slack += e + p * 2.0 ** -24 * np.abs(v)
    for i in range(p):
        close(b.y[i], (parts, slack), f"y of rank {i}")
        assert torch.equal(b.out[i], b.out[0])
    assert torch.equal(b.y16, b.y[0].bfloat16())
    close(b.logits[0], ref.linear(np64(b.y16), np64(b.router), None, None,
                                  "none", "bfloat16", "float32")["y"],
          "logits")
    index, weight = ref.choice(np64(b.logits[0]), args[-1], "softmax", True)
    np.testing.assert_array_equal(b.index.cpu().numpy(), index)
    np.testing.assert_allclose(np64(b.weight), weight, rtol=2.0 ** -20)
    out, slack = np.zeros_like(parts), np.zeros_like(parts)
    own = b.eg[0].shape[1]
    for i in range(p):
        v, e = ref.moe(np64(b.y16), index, weight, np64(b.eg[0][i]),
                       np64(b.eu[0][i]), np64(b.ed[0][i]),
                       [np64(t[1][i]) for t in (b.eg, b.eu, b.ed)],
                       np64(b.y[0]) if i == 0 else None, "silu", "bfloat16",
                       "float32", i * own)
        out += v
        slack += e + p * 2.0 ** -24 * np.abs(v)
    close(b.out[0], (out, slack), "out")


def test_recorded_block():
    b = block(4, 9, 128, 256, 8, 64, 3)
    g = torch.Generator("cuda").manual_seed(1)
    graph = b.record()
    for _ in range(4):
        b.x.normal_(generator=g)
        graph.replay()
        got, index = b.out.clone(), b.index.clone()
        b.out.zero_()
        b.step()
        assert torch.equal(b.out, got) and torch.equal(b.index, index)


def test_example_runs(capsys):
    need_gpu()
    sys.path.insert(0, EXAMPLES)
    try:
        import served_layer
    finally:
        sys.path.remove(EXAMPLES)
    served_layer.main(["2", "3", "256", "512", "4", "2"])
    assert "a step" in capsys.readouterr().out
