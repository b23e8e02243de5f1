"""Entry points of the layer products without a GPU: what they refuse, with
which code, and the workspace query.  Argument checks run before any device
work; the addresses here are never read."""

import ctypes
import os

import pytest

from paper_2109_12626_amd import dpar

A = 1 << 30          # fake device addresses, 1 MiB apart
STEP = 1 << 20
needs_no_gpu = pytest.mark.skipif(
    os.path.exists("/dev/kfd"),
    reason="would launch on fake addresses with a GPU present")


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
    v = dict(rows=5, n_in=16, n_out=24, dtype="bfloat16", act="none")
    v.update(kw)
    return dpar.product_options(**v)


def _linear(opt=None, p=2, **kw):
    a = dict(x=_at(0), w=_at(1), bias=_at(2), residual=_at(3), y=_at(4),
             z=_at(5))
    a.update(kw)
    return _code(dpar.dpar_linear, *a.values(), p, opt or _opt())


def _linear_backward(opt=None, p=2, **kw):
    a = dict(dy=_at(0), x=_at(1), w=_at(2), z=_at(3), dx=_at(4), dw=_at(5),
             dbias=_at(6), dz=_at(7))
    a.update(kw)
    return _code(dpar.dpar_linear_backward, *a.values(), p,
                 opt or _opt(act="silu"))


def _gated(opt=None, p=2, **kw):
    a = dict(x=_at(0), wg=_at(1), wu=_at(2), bg=_at(3), bu=_at(4), h=_at(5),
             g=_at(6), u=_at(7))
    a.update(kw)
    return _code(dpar.dpar_gated, *a.values(), p, opt or _opt(act="silu"))


def _gated_backward(opt=None, p=2, **kw):
    a = dict(dh=_at(0), x=_at(1), wg=_at(2), wu=_at(3), g=_at(4), u=_at(5),
             dx=_at(6), dwg=_at(7), dwu=_at(8), dbg=_at(9), dbu=_at(10),
             dg=_at(11), du=_at(12))
    a.update(kw)
    return _code(dpar.dpar_gated_backward, *a.values(), p,
                 opt or _opt(act="silu"))


CALLS = [_linear, _linear_backward, _gated, _gated_backward]
INVALID, UNSUPPORTED, ALIAS, HIP = (dpar.DPAR_ERR_INVALID_ARG,
                                    dpar.DPAR_ERR_UNSUPPORTED,
                                    dpar.DPAR_ERR_ALIAS, dpar.DPAR_ERR_HIP)


@needs_no_gpu
@pytest.mark.parametrize("call", CALLS)
def test_valid_calls_reach_the_device(call):
    assert call() == HIP


@pytest.mark.parametrize("call", CALLS)
def test_options(call):
    assert call(p=0) == INVALID
    assert call(_opt(dtype="int32")) == UNSUPPORTED
    assert call(_opt(dtype="u32mat2x2")) == UNSUPPORTED
    assert call(_opt(dtype="float32", out_dtype="bfloat16")) == UNSUPPORTED
    assert call(_opt(dtype="bfloat16", out_dtype="float16")) == UNSUPPORTED
    assert call(_opt(act=5)) == INVALID
    assert call(_opt(act=-1)) == INVALID
    assert call(_opt(rows=1 << 31)) == UNSUPPORTED
    assert call(_opt(n_in=1 << 40)) == UNSUPPORTED
    assert call(_opt(ldx=(1 << 38) + 1)) == UNSUPPORTED
    assert call(_opt(ldx=15)) == INVALID         # rows of x would overlap
    assert call(_opt(ldw=15)) == INVALID


def test_null_options():
    f = dpar.lib().dpar_linear
    assert f(None, None, None, None, None, None, 1, None, None, 0,
             None) == INVALID


@pytest.mark.parametrize("call,needed", [
    (_linear, ["x", "w", "y"]),
    (_linear_backward, ["dy", "x", "w", "z", "dz"]),
    (_gated, ["x", "wg", "wu", "h"]),
    (_gated_backward, ["dh", "x", "wg", "wu", "g", "u", "dg", "du"])])
def test_null_arrays_and_entries(call, needed):
    for k in needed:
        assert call(**{k: None}) == INVALID, k
        assert call(**{k: [A + 50 * STEP, 0]}) == INVALID, k
        assert call(**{k: [A + 50 * STEP, A + 51 * STEP + 1]}) == INVALID, k
        assert call(**{k: [A + 50 * STEP, 1 << 48]}) == UNSUPPORTED, k


def test_results_that_belong_together():
    assert _gated(g=None) == INVALID and _gated(u=None) == INVALID
    assert _gated_backward(dwg=None, dbg=None) == INVALID
    assert _gated_backward(dwu=None) == INVALID
    assert _gated_backward(dbu=None) == INVALID
    # bias gradients come with the weights'
    assert _linear_backward(dw=None) == UNSUPPORTED
    assert _gated_backward(dwg=None, dwu=None) == UNSUPPORTED


@needs_no_gpu
def test_optional_arguments_may_be_missing():
    assert _linear(bias=None, residual=None, z=None) == HIP
    assert _linear(bias=[0, A + 60 * STEP], residual=[A + 61 * STEP, 0]) == HIP
    assert _linear_backward(dbias=None) == HIP
    assert _linear_backward(dx=None, w=None) == HIP
    assert _linear_backward(dw=None, dbias=None, x=None) == HIP
    assert _linear_backward(_opt(), z=None, dz=None) == HIP
    assert _gated(bg=None, bu=None, g=None, u=None) == HIP
    assert _gated_backward(dbg=None, dbu=None) == HIP
    assert _gated_backward(dx=None, wg=None, wu=None) == HIP


def test_overlap_is_refused():
    x = _at(0)
    assert _linear(y=[x[1], A + 50 * STEP]) == ALIAS         # another rank's
    assert _linear(y=x) == ALIAS
    assert _linear(y=[v + 8 for v in _at(1)]) == ALIAS
    assert _linear(y=[A + 50 * STEP] * 2) == ALIAS           # each other
    assert _linear(y=_at(5)) == ALIAS                        # y is z
    assert _linear(y=[A + 50 * STEP, A + 50 * STEP + 4 * 24 * 2 + 2]) == ALIAS
    assert _linear_backward(dx=_at(1)) == ALIAS
    assert _gated_backward(du=_at(11)) == ALIAS              # dg is du
    # in place, but with another rank's values, or values others read too
    z = _at(3)
    assert _linear_backward(dz=z[::-1]) == ALIAS
    assert _linear_backward(z=[z[0]] * 2, dz=[z[0], A + 60 * STEP]) == ALIAS
    dy = _at(0)
    assert _linear_backward(dy=[dy[0]] * 2, dz=[dy[0], A + 60 * STEP]) == ALIAS
    # the result's row distance is not the input's
    assert _linear_backward(_opt(act="silu", ldy=48), dz=_at(0)) == ALIAS


@needs_no_gpu
def test_overlap_that_is_allowed():
    one = [A] * 2
    assert _linear(x=one) == HIP                             # a shared input
    assert _linear(x=one, w=one) == HIP
    assert _linear_backward(dz=_at(3)) == HIP                # in place of z
    assert _linear_backward(dz=_at(0)) == HIP                # in place of dy
    assert _gated_backward(dg=_at(4), du=_at(5)) == HIP
    assert _gated_backward(dg=_at(0), du=_at(5)) == HIP
    # g beside u in rows of 48, results of 24 columns side by side
    side = _at(6)
    assert _gated(_opt(act="silu", ldz=48), g=side,
                  u=[v + 24 * 2 for v in side]) == HIP
    assert _gated(_opt(act="silu", ldz=48), g=side,
                  u=[v + 22 * 2 for v in side]) == ALIAS
    # rows that end where the next matrix begins
    assert _linear(y=[A + 50 * STEP, A + 50 * STEP + 5 * 24 * 2]) == HIP


def test_nothing_to_do():
    # no result element: a success that touches nothing, null entries and all
    assert _linear(_opt(rows=0), x=[0, 0], y=[0, 0], z=[0, 0],
                   residual=[0, 0]) == 0
    assert _linear(_opt(n_out=0), w=[0, 0], y=[0, 0], z=None, bias=None) == 0
    assert _gated(_opt(rows=0, act="silu")) == 0
    assert _linear_backward(_opt(n_out=0, rows=0, act="relu")) == 0


def test_workspace_query_and_check():
    big = _opt(rows=128, n_in=16384, n_out=512, dtype="float16")
    n = dpar.dpar_product_workspace("linear", 2, big)
    assert n > 0 and n % 4 == 0
    f = dpar.dpar_linear
    args = (_at(0), [A + 200 * STEP, A + 300 * STEP], None, None, _at(4), None,
            2, big)
    assert _code(f, *args, A + 500 * STEP, n - 1) == INVALID
    assert _code(f, *args, A + 500 * STEP + 8, n) == INVALID
    # full of tiles: nothing to split
    for call in dpar.PRODUCTS:
        assert dpar.dpar_product_workspace(
            call, 8, _opt(rows=4096, n_in=4096, n_out=4096, act="silu")) == 0
    for call in (-1, 4):
        assert _code(dpar.dpar_product_workspace, call, 1, _opt()) == INVALID
    assert _code(dpar.dpar_product_workspace, "linear", 0, _opt()) == INVALID
    assert dpar.lib().dpar_product_workspace(0, 1, ctypes.byref(_opt()),
                                             None) == INVALID


def test_reduction_still_refuses_16_bit_types():
    ys = [A + (20 + i) * STEP for i in range(2)]
    for dtype in ("bfloat16", "float16"):
        assert _code(dpar.dpar_allreduce, _at(0), ys, 2, 100, dtype,
                     "sum", 1) == UNSUPPORTED
        assert _code(dpar.dpar_schedule_info, 2, 100, dtype) == UNSUPPORTED


def test_tensor_front_ends_check_their_tensors():
    import torch
    x, w = torch.zeros(3, 16), torch.zeros(8, 16)
    with pytest.raises(ValueError):
        dpar.linear(x, w, act="silu", out_dtype=torch.int32)
    with pytest.raises(ValueError):
        dpar.linear(x.bfloat16(), w)
    with pytest.raises(ValueError):
        dpar.linear(torch.zeros(3, 15), w)
    with pytest.raises(ValueError):
        dpar.linear(torch.zeros(16, 3).t(), w)
    with pytest.raises(ValueError):
        dpar.linear(x, w, bias=torch.zeros(9))
    with pytest.raises(ValueError):
        dpar.linear(x, torch.zeros(2, 8, 16), bias=torch.zeros(8))
    with pytest.raises(ValueError):
        dpar.gated(x, w, torch.zeros(8, 32)[:, ::2])
    with pytest.raises(ValueError):
        dpar.linear_backward(torch.zeros(3, 8), x, w, act="gelu")
    with pytest.raises(KeyError):
        dpar.linear(x, w, act="tanh")


@pytest.mark.parametrize("name", ["x", "w", "dy", "residual"])
@pytest.mark.parametrize("ranks", [(), (2,)])
@pytest.mark.parametrize("view", ["expand", "window"])
def test_front_ends_refuse_overlapping_rows(name, ranks, view):
    # a distance of 0 would mean packed rows to the library
    import torch

    def repeated(t):
        first = t[..., :1, :]
        if view == "expand":
            return first.expand(t.shape)
        long = torch.zeros(ranks + (t.shape[-1] + t.shape[-2] - 1,))
        return long.unfold(-1, t.shape[-1], 1)

    t = {"x": torch.zeros(ranks + (3, 8)), "w": torch.zeros(ranks + (5, 8)),
         "dy": torch.zeros(ranks + (3, 5)),
         "residual": torch.zeros(ranks + (3, 5))}
    assert t[name].shape == repeated(t[name]).shape
    t[name] = repeated(t[name])
    with pytest.raises(ValueError, match=f"{name}: rows .* overlap"):
        if name == "dy":
            dpar.linear_backward(t["dy"], t["x"], t["w"])
        else:
            dpar.linear(t["x"], t["w"], residual=t["residual"])


@needs_no_gpu
def test_matrices_past_the_address_space_are_refused():
    # 2^25 rows 2^38 values apart: 2^64 bytes in 16 bits, 0 in a 64-bit size
    big = dict(rows=(1 << 25) + 1, ldx=1 << 38)
    for call in CALLS:
        act = "none" if call is _linear else "silu"
        assert call(_opt(act=act, **big)) == UNSUPPORTED
        assert call(_opt(act=act, rows=(1 << 31) - 1, ldy=1 << 38)) \
            == UNSUPPORTED
        assert call(_opt(act=act, n_in=(1 << 31) - 1,
                         n_out=(1 << 31) - 1)) == UNSUPPORTED
