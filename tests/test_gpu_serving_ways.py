"""Every kernel of the 8-bit products and of the mixture-of-experts layer, against
64 bits (tests/test_serving_cases.py compares the calls with what the library
holds): each call takes the kernels that the plan without a device names.  Every
rank of an expert layer has an x, and is given arrays for the choice, of its own."""

import os
import shutil
import subprocess

import numpy as np
import pytest
import torch

from oracle import products as ref
from tests._gpu import _Env, lib, need_gpu
from tests._serving_cases import INT8, MOE
from tests.test_gpu_int8 import Ranks, close, np64, run_int8
from tests.test_gpu_moe import Layer
from tests.test_serving_cases import line_of
from tests.test_serving_plans import CSRC, ROOT

pytestmark = pytest.mark.gpu
ACTS = ["silu", "gelu", "relu", "gelu_tanh", "none"]
OUTS = ["bfloat16", "float16", "float32"]


@pytest.fixture(scope="module")
def planned(tmp_path_factory):
    """What DPAR_LOG prints of a call's kernels, by case."""
    gxx = shutil.which("g++")
    if gxx is None:
        pytest.skip("g++ not available")
    rocm = os.environ.get("ROCM_PATH", "/opt/rocm")
    exe = str(tmp_path_factory.mktemp("serving") / "plans")
    subprocess.run(
        [gxx, "-O1", "-std=c++17", "-D__HIP_PLATFORM_AMD__",
         "-I", os.path.join(ROOT, "include"), "-I", CSRC,
         "-I", os.path.join(rocm, "include"),
         os.path.join(ROOT, "tests", "cpp", "serving_plans.cpp")]
        + [os.path.join(CSRC, f) for f in ("int8_api.cpp", "moe_api.cpp",
                                           "products_api.cpp")]
        + ["-o", exe], check=True)
    cases = [*INT8, *MOE]
    lines = subprocess.run([exe], input="\n".join(map(line_of, cases)),
                           text=True, check=True, capture_output=True,
                           env={**os.environ, "DPAR_LOG": "1"}
                           ).stderr.splitlines()
    assert len(lines) == len(cases)
    return dict(zip(cases, lines))


def check_plan(case, planned, capfd, call):
    need_gpu()
    if torch.cuda.get_device_properties(0).multi_processor_count != 256:
        pytest.skip("the rules count CUs")
    lib()
    capfd.readouterr()
    with _Env("DPAR_LOG", 1):
        result = call()
    assert [ln for ln in capfd.readouterr().err.splitlines()
            if ln.startswith("dpar: ")] == [planned[case]]
    return result


@pytest.mark.parametrize("k", range(len(INT8)),
                         ids=["-".join(map(str, c)) for c in INT8])
def test_8_bit_product(k, planned, capfd):
    call, p, rows, n_in, n_out, far, ws = INT8[k]
    check_plan(INT8[k], planned, capfd, lambda: run_int8(
        call, p, rows, n_in, n_out, OUTS[k % 3], ACTS[k % 5], far=far,
        split=bool(ws), seed=k))


class Apart(Layer):
    """x, the arrays of the choice and, where `own`, the logits of each rank
    lie apart."""

    def __init__(self, own, p, tokens, n_in, hidden, experts, top, *args,
                 **kw):
        super().__init__(p, tokens, n_in, hidden, experts, top, *args, **kw)
        far = self.x.ld - n_in
        self.x = Ranks(p, tokens, n_in, self.dtype, far).normal(self.g)
        if own:
            self.logits = Ranks(p, tokens, p * experts, "float32",
                                far).normal(self.g, 2.0)
        self.index = torch.full((p, tokens, top), 99, dtype=torch.int32,
                                device="cuda")
        self.weight = torch.full((p, tokens, top), 99.0, device="cuda")

    def run(self, given=False, stream=None):
        d, p = lib(), self.p
        logits = self.logits.at if self.logits.t.shape[0] == p \
            else d.pointers([self.logits.t.data_ptr()] * p)
        d.dpar_moe(self.x.at, None if given else logits, self.wg.ranks,
                   self.wu.ranks, self.wd.ranks,
                   *([t.at for t in self.s] if self.s else [None] * 3),
                   self.r.at if self.r else None, self.y.at,
                   d.rows(self.index), d.rows(self.weight), p, self.opt,
                   self.ws, self.ws.numel(),
                   stream or torch.cuda.current_stream())

    def check(self, given=False):
        n, each = self.experts, {}
        for i in range(self.p):
            if given:
                chosen = self.index[i].cpu().numpy(), np64(self.weight[i])
            else:
                k = i if len(self.logits.t) > 1 else 0
                if k not in each:
                    each[k] = ref.choice(np64(self.logits.t[k]), self.top,
                                         self.route, self.normalize,
                                         self.scale)
                chosen = each[k]
                np.testing.assert_array_equal(self.index[i].cpu().numpy(),
                                              chosen[0])
                np.testing.assert_allclose(np64(self.weight[i]), chosen[1],
                                           rtol=2.0 ** -20, atol=2.0 ** -126)
            part = slice(i * n, (i + 1) * n)
            want = ref.moe(
                np64(self.x.t[i]), *chosen, np64(self.wg.m[part]),
                np64(self.wu.m[part]), np64(self.wd.m[part]),
                [np64(t.t[i]) for t in self.s] if self.s else None,
                np64(self.r.t[i]) if self.r else None, self.act, self.dtype,
                self.out, i * n, not given)
            close(self.y.t[i], want, f"rank {i}")
        assert self.y.gaps_untouched()


@pytest.mark.parametrize("k", range(len(MOE)),
                         ids=["-".join(map(str, c)) for c in MOE])
def test_expert_layer(k, planned, capfd):
    need_gpu()
    *sizes, dtype, weights, out, far, own = MOE[k]
    layer = Apart(bool(own), *sizes, dtype, weights, out, act=ACTS[k % 5],
                  route=["softmax", "sigmoid"][k % 2], normalize=k % 3 > 0,
                  far=far, residual=k % 2 == 0, seed=k)
    check_plan(MOE[k], planned, capfd, layer.run)
    layer.check()


# tokens, experts: the choice in the projections, by a launch, by every expert
@pytest.mark.parametrize("p,tokens,experts,top", [
    (2, 1, 4, 3), (5, 7, 6, 2), (3, 12, 24, 2), (2, 40, 5, 3), (35, 40, 1, 3),
    (40, 30, 16, 2)])
@pytest.mark.parametrize("own", [False, True])
@pytest.mark.parametrize("given", [False, True])
@pytest.mark.parametrize("n_in,hidden", [(96, 64), (51, 33)])
def test_ranks_with_rows_of_their_own(p, tokens, experts, top, own, given,
                                      n_in, hidden):
    """One choice for all ranks or one for each, read from or written to arrays
    of each rank's own."""
    need_gpu()
    layer = Apart(own, p, tokens, n_in, hidden, experts, top, "float16",
                  seed=tokens)
    if given:
        layer.index.copy_(torch.randint(-1, p * experts, layer.index.shape,
                                        generator=layer.g, device="cuda",
                                        dtype=torch.int32))
        layer.weight.normal_(generator=layer.g)
        if not own:
            layer.index[1:] = layer.index[0]
            layer.weight[1:] = layer.weight[0]
        held = layer.index.clone(), layer.weight.clone()
    layer.run(given)
    layer.check(given)
    if given:
        assert torch.equal(layer.index, held[0])
        assert torch.equal(layer.weight, held[1])
