"""Every kernel of the layer products: sizes that its rule gives it (the plan
line says so), against 64 bits."""

import pytest
import torch

from tests._gpu import _Env, lib, need_gpu
from tests.test_gpu_products import RUNS

pytestmark = pytest.mark.gpu

# call, ranks, rows, in, out, type, distance between rows; what the plan says
# of the call's first product
CASES = [
    ("linear", 1, 3, 200, 48, "bfloat16", 0,
     "operands=aligned kernel=few sets=1 waves=1"),
    ("linear", 1, 16, 2048, 512, "float16", 0,
     "operands=aligned kernel=few sets=1 waves=8"),
    ("linear", 1, 9, 1001, 512, "float16", 0,
     "operands=unaligned kernel=few sets=1 waves=2"),
    ("linear", 8, 16, 264, 2048, "bfloat16", 0,
     "operands=aligned kernel=few sets=2 waves=1"),
    ("linear", 8, 5, 1024, 1024, "bfloat16", 0,
     "operands=aligned kernel=few sets=2 waves=4"),
    ("linear", 1, 24, 512, 264, "float32", 0,
     "operands=aligned kernel=few sets=2 waves=4"),
    ("linear", 8, 24, 264, 2048, "bfloat16", 0,
     "operands=aligned kernel=few sets=4 waves=1"),
    ("linear", 8, 40, 520, 2064, "float16", 0,
     "operands=aligned kernel=few sets=4 waves=2"),
    ("linear", 8, 60, 1032, 2048, "bfloat16", 0,
     "operands=aligned kernel=few sets=4 waves=4"),
    ("gated", 1, 1, 1024, 72, "bfloat16", 0,
     "operands=aligned kernel=few sets=2 waves=4"),
    ("gated", 8, 7, 600, 1024, "bfloat16", 0,
     "operands=aligned kernel=few sets=4 waves=2"),
    ("gated", 8, 50, 600, 1024, "float16", 5,
     "operands=unaligned kernel=few sets=4 waves=2"),
    ("linear", 1, 300, 200, 200, "bfloat16", 0,
     "kernel=64x64x4 splits=1"),
    ("linear", 8, 300, 72, 520, "bfloat16", 0,
     "kernel=64x64 splits=1"),
    ("linear", 1, 70, 4104, 264, "float16", 0,
     "kernel=64x64x4 splits="),
    ("linear", 8, 300, 300, 500, "float32", 0,
     "operands=aligned kernel=64x64 splits=1"),
    ("linear", 8, 250, 200, 4096, "float32", 0,
     "kernel=128x128 splits=1"),
    ("linear", 7, 875, 1001, 400, "float16", 0,
     "operands=unaligned kernel=64x64 "),
    ("linear", 8, 256, 201, 4095, "float32", 0,
     "operands=unaligned kernel=128x128 "),
    ("linear", 1, 2000, 136, 2056, "bfloat16", 0,
     "kernel=256x128 splits=1"),
    ("gated", 1, 1000, 520, 4096, "float16", 0,
     "kernel=256x128 splits=1"),
    ("linear", 8, 1000, 136, 2000, "bfloat16", 0,
     "kernel=256x256 splits=1"),
    ("linear", 8, 1024, 72, 2040, "float16", 0,
     "kernel=256x256 splits=1"),
    ("gated", 8, 1000, 200, 1000, "bfloat16", 0,
     "kernel=256x256 splits=1"),
    ("linear_backward", 8, 1000, 2040, 136, "bfloat16", 0,
     "kernel=256x256 splits=1"),
    ("gated_backward", 8, 1000, 2040, 136, "float16", 0,
     "kernel=256x256 splits=1"),
    ("linear_backward", 1, 1301, 1303, 1305, "bfloat16", 0,
     "operands=copied kernel="),
    ("gated_backward", 1, 1301, 1303, 1305, "float16", 0,
     "operands=copied kernel="),
    ("linear", 1, 2001, 2001, 2001, "bfloat16", 0,
     "operands=copied kernel=128x128"),
    ("gated", 1, 1500, 1501, 1500, "float16", 0,
     "operands=copied kernel=256x128"),
]


@pytest.mark.parametrize("op,p,rows,n_in,n_out,dtype,far,plan", CASES)
def test_kernel_of_a_size(op, p, rows, n_in, n_out, dtype, far, plan, capfd):
    need_gpu()
    if torch.cuda.get_device_properties(0).multi_processor_count != 256:
        pytest.skip("the rules count CUs")
    lib()
    capfd.readouterr()
    with _Env("DPAR_LOG", 1):
        RUNS[op](p, rows, n_in, n_out, dtype, act="silu", far=far, seed=21)
    first = capfd.readouterr().err.splitlines()[0]
    assert plan in first, first
