"""Barriers of the layer products' kernels, as written: the builtins order no
access that the compiler may move, so they stand only where nothing moves
across them, and where lanes exchange values through LDS one stands between
the stores and the loads.  CPU only: reads the source."""

import os
import re

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _source():
    path = os.path.join(ROOT, "paper_2109_12626_amd", "csrc",
                        "products_kernels.hpp")
    with open(path) as f:
        return re.sub(r"//[^\n]*", "", f.read())


def test_barriers_order_the_compiler_too():
    text = _source()
    for name in ("__builtin_amdgcn_s_barrier", "__builtin_amdgcn_wave_barrier"):
        fenced = re.findall(r'asm volatile\("" ::: "memory"\);\s*' + name
                            + r'\(\);\s*asm volatile\("" ::: "memory"\);',
                            text)
        assert len(fenced) == 1 and text.count(name) == 1, name


def test_results_that_change_lanes_are_fenced():
    """Results::store: each part's stores, a fence, its loads, a fence."""
    text = _source()
    body = text[text.index("struct Results"):]
    body = body[:body.index("struct Tiled")]
    loop = body[body.index("for (int mh"):]
    write = loop.index("*(LDS f32x4*)(mine")
    first = loop.index("in_order();")
    read = loop.index("*(LDS f32x4*)(at")
    second = loop.index("in_order();", first + 1)
    assert write < first < read < second
    assert "meet();" in body[:body.index("for (int mh")]
