"""Builds libdpar.so and libdpar_products-*.so (the layer products' kernels) in
place: HIP kernels for gfx950 with hipcc, host C++ with g++, linked by hipcc.
``python -m paper_2109_12626_amd.build``."""

import concurrent.futures
import glob
import hashlib
import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
BUILD = os.path.join(ROOT, "_build")
LIB = os.path.join(HERE, "libdpar.so")
ROCM = os.environ.get("ROCM_PATH", "/opt/rocm")
ARCH = "gfx950"

HIP_FLAGS = [
    "-O3", "-fPIC", "-std=c++17", f"--offload-arch={ARCH}",
    "-fno-fast-math", "-ffp-contract=off",
    # keep fp32 arithmetic on the scalar (non-packed) VALU instructions
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall", "-Wno-unused-result",
]
PRODUCT_SOURCES = ["products_bf16.hip", "products_f16.hip",
                   "products_f32.hip", "products_int8.hip",
                   "moe_route.hip", "moe_bf16.hip", "moe_f16.hip",
                   "moe_f32.hip"]
HOST_FLAGS = ["-O2", "-fPIC", "-std=c++17", "-Wall", "-Wextra",
              "-Wno-unused-parameter", "-D__HIP_PLATFORM_AMD__"]


def _run(cmd):
    print(" ".join(cmd), flush=True)
    subprocess.run(cmd, check=True)


def _run_all(cmds):
    """The commands side by side, as many as the machine is meant to run."""
    jobs = int(os.environ.get("MAX_JOBS") or min(8, os.cpu_count() or 1))
    with concurrent.futures.ThreadPoolExecutor(max(1, jobs)) as pool:
        for done in [pool.submit(_run, c) for c in cmds]:
            done.result()


def _link(hipcc, lib, objs, flags, libs, soname):
    tmp = lib + ".tmp"
    _run([hipcc, "-shared", "-fPIC", f"--offload-arch={ARCH}"] + flags
         + ["-o", tmp] + objs + libs + [f"-Wl,-soname,{soname}"])
    os.replace(tmp, lib)


def products_name(lib, objs):
    """File of the products' kernels that belongs to a build: after the
    library's own name and the kernels' contents, so that neither builds in one
    directory nor builds loaded into one process take each other's."""
    h = hashlib.sha256()
    for obj in objs:
        with open(obj, "rb") as f:
            h.update(f.read())
    return f"{_products_stem(lib)}{h.hexdigest()[:12]}.so"


def _products_stem(lib):
    return os.path.splitext(os.path.basename(lib))[0] + "_products-"


def drop_old_products(lib, keep):
    """Removes what earlier builds of this library left beside it."""
    where = os.path.dirname(os.path.abspath(lib))
    stem = os.path.join(glob.escape(where), glob.escape(_products_stem(lib)))
    for old in glob.glob(stem + "[0-9a-f]" * 12 + ".so"):
        if os.path.basename(old) != keep:
            os.remove(old)


def build(verbose=True, out=None, defines=(), host_sanitize=False):
    """Compiles libdpar.so (or ``out``); ``defines`` are extra -D flags for
    kernel experiments.  ``host_sanitize``: the host C++ (plan.cpp, api.cpp
    and the host side of the launches) built with AddressSanitizer and
    UndefinedBehaviorSanitizer, for CPU runs of the no-device entry points
    (needs ``out``; load it with libasan and libubsan preloaded)."""
    if host_sanitize and out is None:
        raise ValueError("a sanitized build needs its own output path")
    build_dir = BUILD if out is None else os.path.dirname(out) + "/_obj"
    os.makedirs(build_dir, exist_ok=True)
    inc = ["-I", os.path.join(ROOT, "include"), "-I", CSRC,
           "-I", os.path.join(ROCM, "include")]
    hipcc = os.path.join(ROCM, "bin", "hipcc")
    objs = []
    san = ["-fsanitize=address,undefined", "-g"] if host_sanitize else []
    for src in ("plan.cpp", "api.cpp", "products_api.cpp", "int8_api.cpp",
                "moe_api.cpp"):
        obj = os.path.join(build_dir, src + ".o")
        _run(["g++"] + HOST_FLAGS + san + inc +
             ["-c", os.path.join(CSRC, src), "-o", obj])
        objs.append(obj)
    cmds, products = [], []
    for src in ["kernels.hip"] + PRODUCT_SOURCES:
        obj = os.path.join(build_dir, src + ".o")
        cmds.append([hipcc] + HIP_FLAGS + [f"-D{d}" for d in defines] + inc
                    + ["-c", os.path.join(CSRC, src), "-o", obj])
        (products if src in PRODUCT_SOURCES else objs).append(obj)
    _run_all(cmds)
    lib = LIB if out is None else out
    link_san = (["-Xarch_host", "-fsanitize=address",
                 "-Xarch_host", "-fsanitize=undefined"] if host_sanitize else [])
    # the layer products' kernels are a library of their own beside it
    where = os.path.dirname(os.path.abspath(lib))
    name = products_name(lib, products)
    _link(hipcc, os.path.join(where, name), products, link_san, [], name)
    _link(hipcc, lib, objs, link_san,
          [os.path.join(where, name), "-Wl,-rpath,$ORIGIN"], "libdpar.so")
    drop_old_products(lib, name)
    return lib


if __name__ == "__main__":
    build()
    sys.exit(0)
