"""Entry points of the mixture-of-experts layer without a GPU: what they refuse,
with which code, and the workspace query.  Argument checks run before any device
work; the addresses here are never read."""

import ctypes
import os

import numpy as np
import pytest

from oracle import products as ref
from paper_2109_12626_amd import dpar

A = 1 << 30          # fake device addresses, 1 MiB apart
STEP = 1 << 20
WORK, WORK_BYTES = 1 << 40, 1 << 30
needs_no_gpu = pytest.mark.skipif(
    os.path.exists("/dev/kfd"),
    reason="would launch on fake addresses with a GPU present")
INVALID, UNSUPPORTED, ALIAS, HIP = (dpar.DPAR_ERR_INVALID_ARG,
                                    dpar.DPAR_ERR_UNSUPPORTED,
                                    dpar.DPAR_ERR_ALIAS, dpar.DPAR_ERR_HIP)
NAMES = ["x", "logits", "wg", "wu", "wd", "sg", "su", "sd", "residual", "y",
         "index", "weight"]


def _at(k, p=2):
    return [A + (k * p + i) * STEP for i in range(p)]


def _opt(**kw):
    v = dict(tokens=5, n_in=32, hidden=24, experts=4, top=3, dtype="bfloat16")
    v.update(kw)
    return dpar.moe_options(**v)


def _moe(opt=None, p=2, ws=WORK, n=WORK_BYTES, eight=False, **kw):
    a = {k: _at(i) for i, k in enumerate(NAMES)}
    if not eight:
        a.update(sg=None, su=None, sd=None)
    a.update(kw)
    opt = opt or _opt(weight_dtype="int8" if eight else None)
    try:
        dpar.dpar_moe(*a.values(), p, opt, ws, n)
        return 0
    except dpar.DparError as e:
        assert str(e).split(": ", 1)[1]
        return e.code


@needs_no_gpu
def test_valid_calls_reach_the_device():
    assert _moe() == HIP
    assert _moe(eight=True) == HIP
    assert _moe(residual=None, index=None, weight=None) == HIP
    assert _moe(residual=[0, A + 90 * STEP], index=[0, A + 91 * STEP],
                weight=[A + 92 * STEP, 0]) == HIP
    assert _moe(logits=None) == HIP
    assert _moe(logits=None, index=[A] * 2, weight=[A + STEP] * 2) == HIP
    assert _moe(y=_at(8)) == HIP                   # the residual's place
    for dtype in ("float16", "float32"):
        assert _moe(_opt(dtype=dtype)) == HIP
    assert _moe(_opt(out_dtype="float32", act="none",
                     route="sigmoid")) == HIP
    assert _moe(_opt(tokens=128, top=8)) == HIP


def test_options():
    assert _moe(p=0) == INVALID
    for dtype in ("int8", "int32", "u32mat2x2"):
        assert _moe(_opt(dtype=dtype)) == UNSUPPORTED
    assert _moe(_opt(weight_dtype="float32")) == UNSUPPORTED
    assert _moe(_opt(dtype="float32", weight_dtype="int8")) == UNSUPPORTED
    assert _moe(_opt(dtype="float32", out_dtype="bfloat16")) == UNSUPPORTED
    assert _moe(_opt(out_dtype="float16")) == UNSUPPORTED
    assert _moe(_opt(act=5)) == INVALID
    assert _moe(_opt(route=2)) == INVALID
    assert _moe(_opt(top=0)) == INVALID
    assert _moe(_opt(top=9)) == INVALID            # of 8 experts
    assert _moe(_opt(experts=0)) == INVALID
    assert _moe(_opt(tokens=129)) == UNSUPPORTED
    assert _moe(_opt(experts=64, top=17)) == UNSUPPORTED
    assert _moe(_opt(experts=513)) == UNSUPPORTED
    assert _moe(_opt(experts=1 << 62)) == UNSUPPORTED
    assert _moe(_opt(n_in=1 << 31)) == UNSUPPORTED
    assert _moe(_opt(ldw=1 << 23)) == UNSUPPORTED
    assert _moe(_opt(ldd=1 << 23)) == UNSUPPORTED
    assert _moe(_opt(n_in=1 << 23, hidden=1)) == UNSUPPORTED
    assert _moe(_opt(hidden=(1 << 31) - 1, n_in=(1 << 31) - 1)) == UNSUPPORTED
    assert _moe(_opt(ldx=31)) == INVALID
    assert _moe(_opt(ldl=7)) == INVALID
    assert _moe(_opt(ldw=31)) == INVALID
    assert _moe(_opt(ldd=23)) == INVALID
    assert _moe(_opt(xw=24 * 32 - 1)) == INVALID   # matrices overlap
    assert _moe(_opt(xd=24 * 32 - 1)) == INVALID
    assert _moe(_opt(ldy=31)) == INVALID
    assert _moe(_opt(xw=(1 << 38) + 1)) == UNSUPPORTED
    f = dpar.lib().dpar_moe
    assert f(*[None] * 12, 1, None, None, 0, None) == INVALID


def test_null_arrays_and_entries():
    for k in ("x", "logits", "wg", "wu", "wd", "y"):
        if k != "logits":
            assert _moe(**{k: None}) == INVALID, k
        assert _moe(**{k: [A + 90 * STEP, 0]}) == INVALID, k
        assert _moe(**{k: [A + 90 * STEP, A + 91 * STEP + 1]}) == INVALID, k
        assert _moe(**{k: [A + 90 * STEP, 1 << 48]}) == UNSUPPORTED, k
    for k in ("sg", "su", "sd"):
        assert _moe(eight=True, **{k: None}) == INVALID
        assert _moe(**{k: _at(5)}) == INVALID      # scales of 16-bit weights
        assert _moe(eight=True, **{k: [A + 90 * STEP, 0]}) == INVALID
    # the choice as an input: all of it
    for k in ("index", "weight"):
        assert _moe(logits=None, **{k: None}) == INVALID
        assert _moe(logits=None, **{k: [A + 90 * STEP, 0]}) == INVALID


def test_overlap_is_refused():
    for k in range(8):
        if k not in (5, 6, 7):
            assert _moe(y=_at(k)) == ALIAS
    assert _moe(eight=True, y=_at(6)) == ALIAS
    assert _moe(y=_at(8)[::-1]) == ALIAS
    assert _moe(y=[A + 90 * STEP] * 2) == ALIAS
    assert _moe(index=_at(1)) == ALIAS
    assert _moe(weight=_at(10)) == ALIAS
    assert _moe(logits=None, y=_at(10)) == ALIAS


def test_workspace():
    n = dpar.dpar_moe_workspace(2, _opt())
    assert n > 0
    assert _moe(ws=None, n=0) == INVALID
    assert _moe(n=n - 1) == INVALID
    assert _moe(ws=WORK + 8) == INVALID
    assert _moe(ws=(1 << 48) - 128) == UNSUPPORTED
    for k in (0, 1, 4, 8, 9, 10, 11):
        assert _moe(ws=_at(k)[1] - n + 16, n=n) == ALIAS
    assert dpar.dpar_moe_workspace(1, _opt(tokens=0)) == 0
    # two 16-bit parts of every hidden value, three where y has 32 bits
    for out, parts in (("bfloat16", 2), ("float32", 3)):
        one, two = (dpar.dpar_moe_workspace(1, _opt(hidden=h, out_dtype=out))
                    for h in (1024, 2048))
        assert two - one == 15 * 1024 * 2 * parts
    f = dpar.lib().dpar_moe_workspace
    assert f(1, ctypes.byref(_opt()), None) == INVALID
    assert f(1, None, None) == INVALID


def test_nothing_to_do():
    null = [0, 0]
    assert _moe(_opt(tokens=0), ws=None, n=0, x=null, logits=null,
                residual=null, y=null, index=null, weight=null) == 0


def test_tensor_front_end_checks_its_tensors():
    import torch
    x, l = torch.zeros(3, 16), torch.zeros(3, 4)
    w, wd = torch.zeros(4, 8, 16), torch.zeros(4, 16, 8)
    i = torch.zeros(3, 2, dtype=torch.int32)
    c = torch.zeros(3, 2)
    for args, kw in [
            ((x, l, w, w, wd), {}),                       # no top
            ((x, None, w, w, wd, 2), {}),                 # no choice
            ((x, l, w, w, wd, 2), dict(index=i, weight=c)),
            ((x, None, w, w, wd), dict(index=i.long(), weight=c)),
            ((x, None, w, w, wd), dict(index=i[:2], weight=c)),
            ((x, l.bfloat16(), w, w, wd, 2), {}),
            ((x, l[:, :3], w, w, wd, 2), {}),
            ((x.half(), l, w, w, wd, 2), {}),
            ((x, l, w, w[:, :7], wd, 2), {}),
            ((x, l, w, w, w, 2), {}),
            ((x[:, :15], l, w, w, wd, 2), {}),
            ((x, l, w, w, wd, 2), dict(sg=torch.zeros(4, 8))),
            ((x.half(), l, w.char(), w.char(), wd.char(), 2), {}),
            ((x, l, w.transpose(1, 2), w.transpose(1, 2), wd, 2), {}),
            ((x, l, w, w, wd[:1].expand(4, 16, 8), 2), {}),
            ((x, l, w, w, wd, 2), dict(residual=torch.zeros(3, 15))),
            ((x, l, w, w, wd, 2), dict(out_dtype=torch.int8)),
            ((x.clone().requires_grad_(), l, w, w, wd, 2), {})]:
        with pytest.raises(ValueError):
            dpar.moe(*args, **kw)


def test_oracle_chooses_as_written():
    v = np.array([[1.0, 3.0, 3.0, -np.inf], [-np.inf] * 4,
                  [np.nan, 5.0, np.inf, np.nan]])
    index, weight = ref.choice(v, 3, "softmax", True)
    assert index.tolist() == [[1, 2, 0], [-1, -1, -1], [0, 3, 2]]
    assert weight[0, 0] == weight[0, 1] and abs(weight[0].sum() - 1) < 1e-15
    assert (weight[1] == 0).all() and np.isnan(weight[2]).all()


def test_work_runs_on_the_tensors_device(monkeypatch):
    """The front ends make the tensors' device the current one."""
    import contextlib
    import torch
    from paper_2109_12626_amd import dpar
    asked = []

    @contextlib.contextmanager
    def device(d):
        asked.append(d)
        yield

    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(torch.cuda, "device", device)
    for index, want in ((0, []), (1, [torch.device("cuda", 1)])):
        asked.clear()
        with dpar._on(torch.device("cuda", index)):
            pass
        assert asked == want
