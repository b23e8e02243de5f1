"""Every kernel of the layer products in every way that the rules reach, against
64 bits (tests/test_product_plans.py compares the cases with the rules' range):
all products of a call take the kernels that the plan without a device names."""

import pytest
import torch

from tests import _plans
from tests._gpu import _Env, lib, need_gpu
from tests._product_cases import CASES
from tests.test_gpu_products import RUNS

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def planned(tmp_path_factory):
    exe = _plans.build(tmp_path_factory.mktemp("plans"))
    lines = [_plans.line(op, p, rows, n_in, n_out, dtype, act, far,
                         workspace=bool(ws), bias=bool(bias))
             for op, p, rows, n_in, n_out, dtype, act, far, ws, bias in CASES]
    return [plans for plans, _ in _plans.ask(exe, lines)]


@pytest.mark.parametrize("k", range(len(CASES)),
                         ids=["-".join(map(str, c)) for c in CASES])
def test_way(k, planned, capfd):
    need_gpu()
    if torch.cuda.get_device_properties(0).multi_processor_count != 256:
        pytest.skip("the rules count CUs")
    lib()
    op, p, rows, n_in, n_out, dtype, act, far, ws, bias = CASES[k]
    capfd.readouterr()
    with _Env("DPAR_LOG", 1):
        RUNS[op](p, rows, n_in, n_out, dtype, act=act, far=far, seed=k,
                 split=bool(ws), bias=bool(bias))
    log = [ln for ln in capfd.readouterr().err.splitlines()
           if "product=" in ln]
    assert log == planned[k]
