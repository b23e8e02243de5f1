"""Which kernels the layer products' rules reach: all that the library holds,
and none that it does not.  CPU only."""

import glob
import itertools
import os
import random
import re
import shutil
import subprocess

import pytest

from paper_2109_12626_amd import dpar
from tests import _plans
from tests._product_cases import CASES

# tile -> BM, BN, tiles in LDS (0: 256-wide halves in turns)
TILES = {0: (64, 64, 2), 1: (64, 64, 4), 2: (128, 128, 2), 3: (256, 128, 0),
         4: (256, 256, 0)}


def _kernels_in_the_library():
    nm = shutil.which("nm")
    if nm is None:
        pytest.skip("nm not available")
    libs = glob.glob(os.path.join(os.path.dirname(dpar.LIB_PATH),
                                  "libdpar_products*.so"))
    assert len(libs) == 1, libs
    out = subprocess.run([nm, "-C", libs[0]], check=True, text=True,
                         capture_output=True).stdout
    out = out.replace("(dpar::products::Type)", "") \
        .replace("(dpar::products::Form)", "")
    return {(k, tuple(a.split(", "))) for k, a in re.findall(
        r"__device_stub__(k_few|k_tiled|k_pingpong)<(.*?)>", out)}


def kernel_of(launch):
    form, dtype, fast, waves, sets, tile, _, rows, sums = launch
    b = ["false", "true"]
    head = (str(dtype), str(form))
    if waves:
        return "k_few", head + (b[fast], str(-(-rows // 16)), str(sets),
                                str(waves))
    bm, bn, ring = TILES[tile]
    if not ring:
        return "k_pingpong", head + (b[sums], str(bn))
    return "k_tiled", head + (b[sums], b[fast], str(bm), str(bn),
                              str(bm // 2), str(bn // 2), str(ring))


def _lines():
    few = itertools.product(
        ["linear", "gated"], [1, 8], [1, 16, 17, 32, 33, 48, 49, 64],
        [64, 256, 512, 1024, 2048, 4096, 16384],
        [8, 64, 512, 1024, 2048, 4096, 8192, 16384],
        ["bfloat16", "float16", "float32"], [0, 1])
    for call, p, rows, n_in, n_out, dtype, far in few:
        yield _plans.line(call, p, rows, n_in, n_out, dtype, "none", far)
    tiles = itertools.product(
        _plans.CALLS, [1, 8], [65, 300, 1000, 4096], [64, 1000, 4096],
        [64, 1000, 4096], ["bfloat16", "float16", "float32"], ["none", "silu"],
        [0, 1], [False, True])
    for call, p, rows, n_in, n_out, dtype, act, far, bias in tiles:
        yield _plans.line(call, p, rows, n_in, n_out, dtype, act, far,
                          workspace=False, bias=bias)


def test_every_kernel_is_reached_and_there(tmp_path):
    asked = _plans.ask(_plans.build(tmp_path), list(_lines()))
    reached = {kernel_of(ln) for _, launches in asked for ln in launches}
    there = _kernels_in_the_library()
    assert reached - there == set()
    assert there - reached == set()


def _random_lines(n):
    rng = random.Random(7)

    def size(lo, hi):
        return round(lo * (hi / lo) ** rng.random())

    for _ in range(n):
        call = rng.choice(_plans.CALLS)
        forward = not call.endswith("backward")
        rows = size(1, 64 if forward and rng.random() < 0.4 else 6000)
        n_in, n_out = size(1, 12000), size(1, 6000)
        if rng.random() < 0.6:
            n_in, n_out = -(-n_in // 8) * 8, -(-n_out // 8) * 8
        yield _plans.line(
            call, rng.choice([1, 1, 1, 2, 3, 4, 8, 16, 36, 60]), rows, n_in,
            n_out, rng.choice(["bfloat16", "float32"]),
            rng.choice(["none", "silu"]) if call == "linear_backward"
            else "silu", rng.choice([0, 0, 8, 5]),
            workspace=rng.random() < 0.7, bias=forward or rng.random() < 0.7)


def test_every_way_has_a_case(tmp_path):
    """What the rules reach over their range is among the ways of the cases
    that run on the GPU against 64 bits."""
    exe = _plans.build(tmp_path)
    cases = [_plans.line(op, p, rows, n_in, n_out, dtype, act, far,
                         workspace=bool(ws), bias=bool(bias))
             for op, p, rows, n_in, n_out, dtype, act, far, ws, bias in CASES]
    tested = {w for a in _plans.ask(exe, cases) for w in _plans.ways(*a)}
    reached = {w for a in _plans.ask(exe, list(_random_lines(100000)))
               for w in _plans.ways(*a)}
    assert len(reached) > 250
    assert reached - tested == set()
