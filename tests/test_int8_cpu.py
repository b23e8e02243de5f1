"""Entry points of the 8-bit layer products without a GPU: what they refuse,
with which code, the workspace query and the oracle's rounding.  Argument checks
run before any device work; the addresses here are never read."""

import ctypes
import os

import numpy as np
import pytest

from oracle import products as ref
from paper_2109_12626_amd import dpar

A = 1 << 30          # fake device addresses, 1 MiB apart
STEP = 1 << 20
needs_no_gpu = pytest.mark.skipif(
    os.path.exists("/dev/kfd"),
    reason="would launch on fake addresses with a GPU present")
INVALID, UNSUPPORTED, ALIAS, HIP = (dpar.DPAR_ERR_INVALID_ARG,
                                    dpar.DPAR_ERR_UNSUPPORTED,
                                    dpar.DPAR_ERR_ALIAS, dpar.DPAR_ERR_HIP)


def _at(k, p=2):
    return [A + (k * p + i) * STEP for i in range(p)]


def _code(fn, *args):
    try:
        fn(*args)
        return 0
    except dpar.DparError as e:
        assert str(e).split(": ", 1)[1]          # every refusal has a text
        return e.code


def _opt(**kw):
    v = dict(rows=5, n_in=32, n_out=24, dtype="int8", out_dtype="bfloat16",
             act="none")
    v.update(kw)
    return dpar.product_options(**v)


def _linear(opt=None, p=2, **kw):
    a = dict(x=_at(0), sx=_at(1), w=_at(2), sw=_at(3), bias=_at(4),
             residual=_at(5), y=_at(6))
    a.update(kw)
    return _code(dpar.dpar_linear_int8, *a.values(), p, opt or _opt())


def _gated(opt=None, p=2, **kw):
    a = dict(x=_at(0), sx=_at(1), wg=_at(2), sg=_at(3), wu=_at(4), su=_at(5),
             bg=_at(6), bu=_at(7), h=_at(8))
    a.update(kw)
    return _code(dpar.dpar_gated_int8, *a.values(), p, opt or _opt())


def _quantize(p=2, rows=5, cols=24, dtype="float16", ldx=0, ldq=0, **kw):
    a = dict(x=_at(0), q=_at(1), scale=_at(2))
    a.update(kw)
    return _code(dpar.dpar_quantize, *a.values(), p,
                 dpar.quantize_options(rows, cols, dtype, ldx, ldq))


CALLS = [_linear, _gated]


@needs_no_gpu
def test_valid_calls_reach_the_device():
    for out in ("bfloat16", "float16", "float32"):
        for call in CALLS:
            assert call(_opt(out_dtype=out)) == HIP
    for dtype in ("bfloat16", "float16", "float32"):
        assert _quantize(dtype=dtype) == HIP
    assert _linear(bias=None, residual=None) == HIP
    assert _linear(bias=[0, A + 60 * STEP], residual=[A + 61 * STEP, 0]) == HIP
    assert _gated(bg=None, bu=None) == HIP
    assert _linear(y=_at(5)) == HIP                # the residual's place
    one = [A] * 2
    assert _linear(x=one, w=one, sx=_at(1)) == HIP
    assert _linear(_opt(n_in=131071)) == HIP


@pytest.mark.parametrize("call", CALLS)
def test_options(call):
    assert call(p=0) == INVALID
    for dtype in ("bfloat16", "float16", "float32", "int32"):
        assert call(_opt(dtype=dtype)) == UNSUPPORTED
    for out in ("int8", "int32", "u32mat2x2"):
        assert call(_opt(out_dtype=out)) == UNSUPPORTED
    assert call(_opt(n_in=131072)) == UNSUPPORTED      # sums past 32 bits
    assert call(_opt(act=5)) == INVALID
    assert call(_opt(rows=1 << 31)) == UNSUPPORTED
    assert call(_opt(ldx=31)) == INVALID
    assert call(_opt(ldw=31)) == INVALID
    assert call(_opt(ldx=(1 << 38) + 1)) == UNSUPPORTED


@pytest.mark.parametrize("call,needed,four", [
    (_linear, ["x", "sx", "w", "sw", "y"], ["sx", "sw"]),
    (_gated, ["x", "sx", "wg", "sg", "wu", "su", "h"], ["sx", "sg", "su"]),
    (_quantize, ["x", "q", "scale"], ["scale"])])
def test_null_arrays_and_entries(call, needed, four):
    for k in needed:
        if call is not _quantize:        # (its arrays are read by the binding)
            assert call(**{k: None}) == INVALID, k
        assert call(**{k: [A + 50 * STEP, 0]}) == INVALID, k
        assert call(**{k: [A + 50 * STEP, 1 << 48]}) == UNSUPPORTED, k
    for k in four:
        assert call(**{k: [A + 50 * STEP, A + 51 * STEP + 2]}) == INVALID, k


def test_overlap_is_refused():
    assert _linear(y=_at(0)) == ALIAS
    assert _linear(y=_at(1)) == ALIAS                  # the scales
    assert _linear(y=_at(3)) == ALIAS
    assert _linear(y=_at(5)[::-1]) == ALIAS            # another rank's
    assert _linear(y=[A + 50 * STEP] * 2) == ALIAS
    assert _gated(h=_at(5)) == ALIAS
    assert _gated(h=_at(6)) == ALIAS
    assert _quantize(q=_at(0)) == ALIAS                # not in place
    assert _quantize(scale=_at(1)) == ALIAS
    assert _quantize(q=[A + 50 * STEP] * 2) == ALIAS


def test_quantisation_options():
    assert _quantize(p=0) == INVALID
    for dtype in ("int8", "int32", "u32mat2x2"):
        assert _quantize(dtype=dtype) == UNSUPPORTED
    assert _quantize(rows=1 << 31) == UNSUPPORTED
    assert _quantize(cols=1 << 31) == UNSUPPORTED
    assert _quantize(ldx=23) == INVALID
    assert _quantize(ldq=23) == INVALID
    assert _quantize(ldq=(1 << 38) + 1) == UNSUPPORTED
    assert _quantize(rows=(1 << 31) - 1, ldx=1 << 38) == UNSUPPORTED
    f = dpar.lib().dpar_quantize
    assert f(None, None, None, 1, None, None) == INVALID


def test_nothing_to_do():
    assert _linear(_opt(rows=0), x=[0, 0], sx=[0, 0], residual=[0, 0],
                   y=[0, 0]) == 0
    assert _gated(_opt(n_out=0), bg=None, bu=None, h=[0, 0]) == 0
    assert _quantize(rows=0, x=[0, 0], q=[0, 0], scale=[0, 0]) == 0


def test_workspace():
    big = _opt(rows=128, n_in=65536, n_out=512)
    n = dpar.dpar_product_workspace("linear", 2, big)
    assert n > 0
    args = (_at(0), _at(1), [A + 200 * STEP, A + 300 * STEP], _at(3), None,
            None, _at(6), 2, big)
    f = dpar.dpar_linear_int8
    assert _code(f, *args, A + 500 * STEP, n - 1) == INVALID
    assert _code(f, *args, A + 500 * STEP + 8, n) == INVALID
    assert _code(f, *args, _at(1)[0] - n + 16, n) == ALIAS   # sx
    assert dpar.dpar_product_workspace(
        "gated", 8, _opt(rows=4096, n_in=4096, n_out=4096)) == 0
    for call in ("linear_backward", "gated_backward"):
        assert _code(dpar.dpar_product_workspace, call, 1, big) == UNSUPPORTED
    assert _code(dpar.dpar_product_workspace, 4, 1, big) == INVALID
    assert dpar.lib().dpar_product_workspace(0, 1, ctypes.byref(big),
                                             None) == INVALID


def test_the_other_products_refuse_8_bits():
    opt = _opt(out_dtype="int8")
    assert _code(dpar.dpar_linear, _at(0), _at(1), None, None, _at(4), None,
                 2, opt) == UNSUPPORTED
    assert _code(dpar.dpar_gated, _at(0), _at(1), _at(2), None, None, _at(4),
                 None, None, 2, opt) == UNSUPPORTED
    assert _code(dpar.dpar_allreduce, _at(0), _at(3), 2, 100, "int8", "sum",
                 1) == UNSUPPORTED
    assert _code(dpar.dpar_schedule_info, 2, 100, "int8") == UNSUPPORTED


def test_tensor_front_ends_check_their_tensors():
    import torch
    i8, f32 = torch.int8, torch.float32
    x, w = torch.zeros(3, 16, dtype=i8), torch.zeros(8, 16, dtype=i8)
    sx, sw = torch.zeros(3), torch.zeros(8)
    for bad in [(x.float(), sx, w, sw), (x, sx.half(), w, sw),
                (x, sx, w.float(), sw), (x, sx, w, sw.double()),
                (x, sx[:2], w, sw), (x, sx, w, sw[:7]),
                (x, torch.zeros(6)[::2], w, sw), (x[:, :15], sx, w, sw)]:
        with pytest.raises(ValueError):
            dpar.linear_int8(*bad)
        with pytest.raises(ValueError):
            dpar.gated_int8(*bad, w, sw)
    with pytest.raises(ValueError):
        dpar.linear_int8(x, sx, w, sw, out_dtype=torch.int32)
    with pytest.raises(ValueError):
        dpar.linear_int8(x, sx, w, sw, bias=torch.zeros(8, dtype=f32))
    with pytest.raises(ValueError):
        dpar.linear(x, w)
    for bad in [torch.zeros(3, 4, dtype=i8), torch.zeros(4),
                torch.zeros(4, 3).t(), torch.zeros(1, 4).expand(3, 4),
                torch.zeros(3, 4, requires_grad=True)]:
        with pytest.raises(ValueError):
            dpar.quantize(bad)


def test_oracle_quantises_as_written():
    q, s = ref.quantize(np.array([[127.0, 0.5, 1.5, -2.5, 126.5],
                                  [0, 0, 0, 0, 0], [1, np.inf, 0, 0, 0],
                                  [1, np.nan, 0, 0, 0]]))
    assert s[0] == 1 and s[1] == 0 and np.isnan(s[2:]).all()
    assert q.tolist() == [[127, 0, 2, -2, 126]] + [[0] * 5] * 3
