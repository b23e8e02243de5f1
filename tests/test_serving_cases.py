"""The calls of tests/_serving_cases.py, which the GPU tests run
(tests/test_gpu_serving_ways.py), take every kernel of the 8-bit products and of
the mixture-of-experts layer that the library holds.  CPU only."""

from tests._serving_cases import INT8, MOE
from tests.test_serving_plans import (TYPES, _int8_kernel, _moe_kernels,
                                      _there, ask)  # noqa: F401

CALLS = ["linear", "gated"]


def line_of(case):
    """As tests/cpp/serving_plans.cpp reads it."""
    if case[0] in CALLS:
        call, p, rows, n_in, n_out, far, ws = case
        return (f"int8 {CALLS.index(call)} {p} {rows} {n_in} {n_out} "
                f"{TYPES['bfloat16']} {far} 0 {ws}")
    return " ".join(["moe", *map(str, case[:6]),
                     *(str(TYPES[t]) for t in case[6:9]),
                     *map(str, case[9:])])


def test_8_bit_products(ask):  # noqa: F811
    ran = [(c, ln) for c, launches in zip(INT8, ask([*map(line_of, INT8)]))
           for ln in launches]
    assert {_int8_kernel(ln) for _, ln in ran} == _there(
        "k_int8_few|k_int8_tiled|k_int8_pingpong")
    # (form, sum in parts, operands copied) of the tiles
    assert {(ln[1], ln[6] > 1, bool(ln[2]) and (c[3] + c[5]) % 16 != 0)
            for c, ln in ran if not ln[3]} == {
        (form, split, copied) for form in (0, 1)
        for split in (False, True) for copied in (False, True)}


def test_mixture_of_experts(ask):  # noqa: F811
    ran = [(c, ln) for c, launches in zip(MOE, ask([*map(line_of, MOE)]))
           for ln in launches if ln[0] == "moe"]
    assert {k for _, ln in ran for k in _moe_kernels(ln)} == _there(
        "k_moe_up|k_moe_down|k_moe_down_small")
    # the choice by a launch, in the projections, by every expert: one rank,
    # ranks that choose alike and apart; more ranks than a launch has
    for mode in range(3):
        assert {min(c[0], 2) * (1 + c[10]) for c, ln in ran
                if ln[3] == mode} >= {1, 2, 4}
    assert {(ln[3], c[10]) for c, ln in ran if c[0] > 32} >= {
        (mode, apart) for mode in (0, 2) for apart in (0, 1)}
