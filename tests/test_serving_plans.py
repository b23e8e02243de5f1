"""Which kernels the rules of the 8-bit products and of the mixture-of-experts
layer reach: all that the library holds, and none that it does not.  CPU only:
tests/cpp/serving_plans.cpp, compiled with the library's own entry points, answers
what they launch."""

import glob
import itertools
import os
import re
import shutil
import subprocess

import pytest

from paper_2109_12626_amd import dpar

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2109_12626_amd", "csrc")
TILES = {0: (64, 64, 2), 1: (64, 64, 4), 2: (128, 128, 2), 3: (256, 128, 0),
         4: (256, 256, 0)}
TYPES = {"float32": 1, "bfloat16": 3, "float16": 4, "int8": 5}
BOOL = ["false", "true"]


@pytest.fixture(scope="module")
def ask(tmp_path_factory):
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

    def run(lines):
        out = subprocess.run([exe], input="\n".join(lines), text=True,
                             check=True, capture_output=True).stdout
        got, launches = [], []
        for ln in out.splitlines():
            if ln.startswith("rc"):
                assert re.fullmatch(r"rc 0 ?", ln), ln
                got.append(launches)
                launches = []
            else:
                name, *values = ln.split()
                launches.append((name, *map(int, values)))
        assert len(got) == len(lines)
        return got
    return run


def _there(pattern):
    nm = shutil.which("nm")
    if nm is None:
        pytest.skip("nm not available")
    lib, = glob.glob(os.path.join(os.path.dirname(dpar.LIB_PATH),
                                  "libdpar_products*.so"))
    out = subprocess.run([nm, "-C", lib], check=True, text=True,
                         capture_output=True).stdout
    out = re.sub(r"\(dpar::(products|moe)::(Type|Form|Mode)\)", "", out)
    return {(k, tuple(a.split(", "))) for k, a in re.findall(
        rf"__device_stub__({pattern})<(.*?)>", out)}


def _int8_kernel(launch):
    _, form, fast, waves, sets, tile, _, rows = launch
    if waves:
        return "k_int8_few", (str(form), BOOL[fast], str(-(-rows // 16)),
                              str(sets), str(waves))
    bm, bn, ring = TILES[tile]
    if not ring:
        return "k_int8_pingpong", (str(form), str(bn))
    return "k_int8_tiled", (str(form), BOOL[fast], str(bm), str(bn),
                            str(bm // 2), str(bn // 2), str(ring))


def test_every_kernel_of_the_8_bit_products(ask):
    few = itertools.product(
        [0, 1], [1, 8], [1, 16, 17, 32, 33, 48, 49, 64],
        [64, 512, 1024, 2048, 4096, 16384],
        [8, 64, 512, 1024, 2048, 4096, 8192, 16384], [0, 1], [0])
    tiles = itertools.product(
        [0, 1], [1, 8], [65, 300, 1000, 4096], [64, 1000, 4096],
        [64, 1000, 4096], [0, 1, 16], [0, 1])
    lines = [f"int8 {g} {p} {rows} {n_in} {n_out} 3 {far} 0 {ws}"
             for g, p, rows, n_in, n_out, far, ws in
             itertools.chain(few, tiles)]
    reached = {_int8_kernel(ln) for launches in ask(lines)
               for ln in launches}
    assert reached == _there("k_int8_few|k_int8_tiled|k_int8_pingpong")


def _columns(eight, fused, shift, tiles):
    if fused:
        return 1
    n = tiles if not eight else 2 * tiles if tiles < 4 else 2
    return min(n, 2) if shift else n


def _moe_kernels(launch):
    (_, x, eight, mode, fast0, tiles0, waves0, small, fast1, tiles1, waves1,
     sets, planes) = launch
    w = 5 if eight else x
    head = (str(w), str(x))
    parts = str(1 if x == 1 else planes)
    columns = _columns(eight, mode == 1, not fast0, tiles0)
    yield "k_moe_up", head + (BOOL[not fast0], str(mode), str(tiles0),
                              str(columns), str(waves0))
    if small:
        yield "k_moe_down_small", head + (BOOL[not fast1], parts)
    else:
        yield "k_moe_down", head + (BOOL[not fast1], parts, str(tiles1),
                                    str(sets), str(waves1))


def test_every_kernel_of_the_mixture_of_experts(ask):
    lines = []
    for (p, tokens, n_in, hidden, experts, top, types, far) in \
            itertools.product(
                [1, 4], [1, 2, 8, 16, 17, 40, 128],
                [64, 512, 2048, 4096, 16384], [32, 512, 1024, 16384],
                [1, 2, 8, 64], [1, 4],
                [("float32", "float32", "float32"),
                 ("bfloat16", "bfloat16", "bfloat16"),
                 ("bfloat16", "bfloat16", "float32"),
                 ("float16", "float16", "float16"),
                 ("float16", "float16", "float32"),
                 ("bfloat16", "int8", "bfloat16"),
                 ("bfloat16", "int8", "float32"),
                 ("float16", "int8", "float16"),
                 ("float16", "int8", "float32")], [0, 1]):
        if top <= p * experts:
            dtype, weights, out = (TYPES[t] for t in types)
            lines.append(f"moe {p} {tokens} {n_in} {hidden} {experts} {top} "
                         f"{dtype} {weights} {out} {far} {far}")
    reached = {k for launches in ask(lines) for ln in launches
               if ln[0] == "moe" for k in _moe_kernels(ln)}
    there = _there("k_moe_up|k_moe_down|k_moe_down_small")
    assert reached - there == set()
    assert there - reached == set()


def test_the_choice_has_a_launch_unless_up_makes_it(ask):
    for line, mode in (("moe 1 1 2048 1024 64 8 3 3 3 0 0", 1),
                       ("moe 1 8 2048 1024 64 8 3 3 3 0 0", 0),
                       ("moe 1 1 2048 1024 512 8 3 3 3 0 0", 0),
                       ("moe 1 24 2048 1024 64 8 3 3 3 0 0", 2),
                       ("moe 1 23 2048 1024 64 8 3 3 3 0 0", 0),
                       ("moe 4 24 2048 1024 16 8 3 3 3 0 1", 2)):
        launches, = ask([line])
        assert [n for n, *_ in launches] == ["route"] * (mode == 0) + ["moe"]
        assert launches[-1][3] == mode


def test_ranks_take_turns(ask):
    launches, = ask(["moe 40 9 64 64 2 4 3 3 3 0 0"])
    assert [n for n, *_ in launches] == ["route", "moe"] * 2
