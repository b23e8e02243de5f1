"""Argument checks of the layer products: the workspace beside the operands and
results.  No device work: the addresses are never read."""

import os

import pytest

from paper_2109_12626_amd import dpar

A = 1 << 40
STEP = 1 << 36
needs_no_gpu = pytest.mark.skipif(
    os.path.exists("/dev/kfd"),
    reason="would launch on fake addresses with a GPU present")
INVALID, ALIAS, HIP = (dpar.DPAR_ERR_INVALID_ARG, dpar.DPAR_ERR_ALIAS,
                       dpar.DPAR_ERR_HIP)

# every array of each call, in order
ARRAYS = {"linear": "x w bias residual y z",
          "linear_backward": "dy x w z dx dw dbias dz",
          "gated": "x wg wu bg bu h g u",
          "gated_backward": "dh x wg wu g u dx dwg dwu dbg dbu dg du"}


def _code(call, p, opt, at, ws, n):
    try:
        getattr(dpar, "dpar_" + call)(
            *[[at[k] + i * (STEP // 4) for i in range(p)]
              for k in ARRAYS[call].split()], p, opt, ws, n)
        return 0
    except dpar.DparError as e:
        assert str(e).split(": ", 1)[1]
        return e.code


# rows, in, out of calls that take a workspace
SIZES = {"linear": (128, 16001, 515), "linear_backward": (2000, 2001, 2003),
         "gated": (2000, 2001, 2003), "gated_backward": (2000, 2001, 2003)}


def _setup(call, **far):
    opt = dpar.product_options(*SIZES[call], "bfloat16", act="silu", **far)
    n = dpar.dpar_product_workspace(call, 2, opt)
    assert n > 0
    at = {k: A + i * STEP for i, k in enumerate(ARRAYS[call].split())}
    return opt, n, at


@pytest.mark.parametrize("call,name", [(c, k) for c, v in ARRAYS.items()
                                       for k in v.split()])
def test_workspace_over_an_array_is_refused(call, name):
    opt, n, at = _setup(call)
    n_rows, n_in, n_out = SIZES[call]
    if name in ("x", "dx"):
        rows, cols = n_rows, n_in
    elif name.lstrip("d").startswith("w"):
        rows, cols = n_out, n_in
    elif name.lstrip("d").startswith("b"):
        rows, cols = 1, n_out
    else:
        rows, cols = n_rows, n_out
    first = at[name] + STEP // 4           # rank 1's
    end = first + rows * cols * 2
    for ws in (first // 16 * 16, (end - 1) // 16 * 16,
               (first - n + 16) // 16 * 16):
        assert _code(call, 2, opt, at, ws, n) == ALIAS, (call, name)


@needs_no_gpu
@pytest.mark.parametrize("call", ARRAYS)
def test_workspace_beside_arrays(call):
    opt, n, at = _setup(call)
    for k in at:
        # ends where the first rank's matrix begins
        assert _code(call, 2, opt, at, at[k] - (n + 15) // 16 * 16, n) == HIP
    # the bytes given beyond those asked for are not used
    k = ARRAYS[call].split()[0]
    assert _code(call, 2, opt, at, at[k] - (n + 15) // 16 * 16, 2 * n) == HIP


@needs_no_gpu
def test_workspace_between_rows():
    """Rows far apart leave room for it; a byte over either row does not."""
    far = 1 << 25                    # values: 64 MB between rows' starts
    opt, n, at = _setup("linear", ldx=far)
    assert n < 2 * far - 16001 * 2 - 64
    row = at["x"] + 5 * far * 2
    begin = row + 16001 * 2
    assert _code("linear", 2, opt, at, -(-begin // 16) * 16, n) == HIP
    assert _code("linear", 2, opt, at, begin // 16 * 16 - 16, n) == ALIAS
    end = row + far * 2
    ws = (end - n) // 16 * 16
    assert _code("linear", 2, opt, at, ws, n) == HIP
    assert _code("linear", 2, opt, at, ws + 16, n) == ALIAS


def test_no_workspace_asked_for_is_none_used():
    opt = dpar.product_options(0, 16, 24, "bfloat16", act="silu")
    assert dpar.dpar_product_workspace("linear", 2, opt) == 0
    at = {k: A + i * STEP for i, k in enumerate(ARRAYS["linear"].split())}
    assert _code("linear", 2, opt, at, at["w"], 0) == 0


@pytest.mark.parametrize("call,name", [
    ("linear", "x"), ("linear", "w"), ("linear", "bias"),
    ("linear", "residual"), ("linear_backward", "dy"),
    ("linear_backward", "z"), ("gated", "wu"), ("gated", "bg"),
    ("gated_backward", "dh"), ("gated_backward", "g")])
def test_front_ends_refuse_gradients_they_would_drop(call, name):
    import torch
    x, w, y, b = (torch.zeros(*s) for s in ((3, 16), (8, 16), (3, 8), (8,)))
    args = {"linear": dict(x=x, w=w, bias=b, residual=y),
            "linear_backward": dict(dy=y, x=x, w=w, z=y, act="silu"),
            "gated": dict(x=x, wg=w, wu=w, bg=b, bu=b),
            "gated_backward": dict(dh=y, x=x, wg=w, wu=w, g=y, u=y)}[call]
    args[name] = args[name].clone().requires_grad_()
    with pytest.raises(ValueError, match=f"{name} requires a gradient"):
        getattr(dpar, call)(**args)
    if not torch.cuda.is_available():
        # past the check where none is recorded: then the device is missing
        with torch.no_grad(), pytest.raises(Exception) as e:
            getattr(dpar, call)(**args)
        assert "gradient" not in str(e.value)


@needs_no_gpu
def test_a_single_row_has_no_distance():
    """In place with any distance, and with distances below its length."""
    at = {k: A + i * STEP for i, k in
          enumerate(ARRAYS["linear_backward"].split())}
    at["dz"] = at["dy"]
    for rows, want in ((1, HIP), (2, ALIAS)):
        opt = dpar.product_options(rows, 16, 24, "bfloat16", act="silu",
                                   ldy=48)
        assert _code("linear_backward", 2, opt, at, None, 0) == want
    at = {k: A + i * STEP for i, k in enumerate(ARRAYS["linear"].split())}
    for rows, out, far in ((1, 24, {"ldx": 1}), (2, 1, {"ldw": 3})):
        opt = dpar.product_options(rows, 16, out, "bfloat16", **far)
        assert _code("linear", 2, opt, at, None, 0) == HIP


@needs_no_gpu
def test_a_result_may_be_its_residual():
    """The update of a residual stream in place; not another rank's, another
    distance's or one that a second rank reads too."""
    at = {k: A + i * STEP for i, k in enumerate(ARRAYS["linear"].split())}
    at["residual"] = at["y"]
    opt = dpar.product_options(5, 16, 24, "bfloat16")
    assert _code("linear", 2, opt, at, None, 0) == HIP
    far = dpar.product_options(5, 16, 24, "bfloat16", ldr=48)
    assert _code("linear", 2, far, at, None, 0) == ALIAS
    y = [A, A + STEP]
    rest = [[A + (2 + i) * STEP, A + (4 + i) * STEP] for i in range(2)]

    def code(residual):
        with pytest.raises(dpar.DparError) as e:
            dpar.dpar_linear(*rest, None, residual, y, None, 2, opt)
        return e.value.code

    assert code(y) == HIP
    assert code([y[0], 0]) == HIP
    assert code(y[::-1]) == ALIAS
    assert code([y[0], y[0]]) == ALIAS
