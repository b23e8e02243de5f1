"""The library of the layer products' kernels belongs to one build: builds in
one directory, and builds loaded into one process, keep their own."""

import os
import re
import shutil
import subprocess

import pytest

from paper_2109_12626_amd import build, dpar


def _needed(lib):
    readelf = shutil.which("readelf")
    if readelf is None:
        pytest.skip("readelf not available")
    out = subprocess.run([readelf, "-d", lib], check=True,
                         capture_output=True, text=True).stdout
    return re.findall(r"NEEDED.*\[(.*)\]", out), \
        re.findall(r"SONAME.*\[(.*)\]", out)


def test_library_needs_the_kernels_of_its_own_build():
    """By a name with the kernels' contents: the loader takes a library of
    that name that it has already loaded."""
    needed = [n for n in _needed(dpar.LIB_PATH)[0] if "dpar" in n]
    assert len(needed) == 1
    assert re.fullmatch(r"libdpar_products-[0-9a-f]{12}\.so", needed[0])
    kernels = os.path.join(os.path.dirname(dpar.LIB_PATH), needed[0])
    assert _needed(kernels)[1] == needed


def test_names_follow_the_library_and_the_contents(tmp_path):
    a, b = tmp_path / "a.o", tmp_path / "b.o"
    a.write_bytes(b"one")
    b.write_bytes(b"two")
    names = {build.products_name(lib, objs)
             for lib in ("x/libdpar.so", "x/libtrial.so")
             for objs in ([a], [b], [a, b])}
    assert len(names) == 6
    assert build.products_name("x/libdpar.so", [a]) == \
        build.products_name("y/libdpar.so", [a])


def test_a_build_drops_its_own_older_kernels_only(tmp_path):
    (tmp_path / "o").write_bytes(b"kernels")
    lib = str(tmp_path / "libdpar.so")
    name = build.products_name(lib, [tmp_path / "o"])
    keep = [name, "libtrial_products-0123456789ab.so", "libdpar.so",
            "libdpar_products-notes.so"]
    for f in keep + ["libdpar_products-0123456789ab.so"]:
        (tmp_path / f).touch()
    build.drop_old_products(lib, name)
    assert sorted(os.listdir(tmp_path)) == sorted(keep + ["o"])
