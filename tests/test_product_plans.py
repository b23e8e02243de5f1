"""Which kernels the layer products' rules reach: all that the library holds,
and none that it does not.  CPU only."""

import glob
import itertools
import os
import re
import shutil
import subprocess

import pytest

from paper_2109_12626_amd import dpar
from tests import _plans

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
