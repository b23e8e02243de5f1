"""Plans of the layer products' calls without a device: tests/cpp/
product_plans.cpp, compiled with the library's own entry points, answers which
kernels they launch."""

import os
import re
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CALLS = ["linear", "linear_backward", "gated", "gated_backward"]
DTYPES = {"float32": 1, "bfloat16": 3, "float16": 4}
ACTS = {"none": 0, "relu": 1, "gelu": 2, "gelu_tanh": 3, "silu": 4}


def build(where):
    gxx = shutil.which("g++")
    if gxx is None:
        pytest.skip("g++ not available")
    rocm = os.environ.get("ROCM_PATH", "/opt/rocm")
    csrc = os.path.join(ROOT, "paper_2109_12626_amd", "csrc")
    exe = os.path.join(str(where), "product_plans")
    subprocess.run([gxx, "-O1", "-std=c++17", "-D__HIP_PLATFORM_AMD__",
                    "-I", os.path.join(ROOT, "include"), "-I", csrc,
                    "-I", os.path.join(rocm, "include"),
                    os.path.join(ROOT, "tests", "cpp", "product_plans.cpp"),
                    os.path.join(csrc, "products_api.cpp"), "-o", exe],
                   check=True)
    return exe


def line(call, p, rows, n_in, n_out, dtype, act="silu", far=0, shift=0,
         workspace=True, out=None, bias=True):
    return " ".join(map(str, (
        CALLS.index(call), p, rows, n_in, n_out, DTYPES[dtype],
        DTYPES[out or dtype], ACTS[act], far, shift, int(workspace),
        int(bias))))


def ask(exe, lines):
    """Of each line: the plan lines of its products, and its launches as
    (form, type, fast, waves, sets, tile, splits, rows, sums)."""
    out = subprocess.run([exe], input="\n".join(lines), text=True, check=True,
                         capture_output=True).stdout
    got, plans, launches = [], [], []
    for ln in out.splitlines():
        if ln.startswith("dpar:"):
            plans.append(ln)
        elif ln.startswith("launch"):
            launches.append(tuple(map(int, ln.split()[1:])))
        else:
            assert re.fullmatch(r"rc 0 ?", ln), ln
            got.append((plans, launches))
            plans, launches = [], []
    assert len(got) == len(lines)
    return got


def ways(plans, launches):
    """What each product of a call takes: form, 16 or 32 bits, operands and
    kernel."""
    # (a call of many ranks launches each product several times)
    each = launches[::max(1, len(launches) // max(1, len(plans)))]
    out = []
    for plan, launch in zip(plans, each):
        form, dtype, operands, kernel, rest = re.match(
            r"dpar: product=(\w+) (\w+) .* operands=(\w+) kernel=(\S+) (.*)",
            plan).groups()
        bits = 32 if dtype == "float32" else 16
        if kernel == "few":
            rest += f" tiles={-(-launch[7] // 16)}"
        else:
            rest = "whole" if rest == "splits=1" else "split"
            rest += " sums" * launch[8]
        out.append((form, bits, operands, kernel, rest))
    return out
