"""The tensor front ends beside forward-mode differentiation: they compute no
tangents, and refuse a tensor that carries one, as they refuse one that requires
a gradient.  CPU only: every refusal comes before the first launch."""

import pytest
import torch
from torch.autograd import forward_ad

from paper_2109_12626_amd import dpar

I8, F32 = torch.int8, torch.float32
MATCH = "tangent"


def operands():
    """Front end, its arguments by name."""
    x, w, wd = torch.zeros(3, 16), torch.zeros(8, 16), torch.zeros(4, 16, 8)
    q, v = torch.zeros(3, 16, dtype=I8), torch.zeros(8, 16, dtype=I8)
    sx, sw, b, r = torch.ones(3), torch.ones(8), torch.ones(8), \
        torch.ones(3, 8)
    e = torch.zeros(4, 8, 16)
    eight = dict(wg=e.to(I8), wu=e.to(I8), wd=wd.to(I8), sg=torch.ones(4, 8),
                 su=torch.ones(4, 8), sd=torch.ones(4, 16))
    return {
        "quantize": (dpar.quantize, dict(x=x)),
        "linear": (dpar.linear, dict(x=x, w=w, bias=b, residual=r)),
        "gated": (dpar.gated, dict(x=x, wg=w, wu=w.clone(), bg=b,
                                   bu=b.clone())),
        "linear_backward": (dpar.linear_backward,
                            dict(dy=torch.ones(3, 8), x=x, w=w)),
        "linear_int8": (dpar.linear_int8,
                        dict(x=q, sx=sx, w=v, sw=sw, bias=b, residual=r,
                             out_dtype=F32)),
        "gated_int8": (dpar.gated_int8,
                       dict(x=q, sx=sx, wg=v, sg=sw, wu=v, su=sw.clone(),
                            bg=b, bu=b.clone(), out_dtype=F32)),
        "moe": (dpar.moe, dict(x=x, logits=torch.zeros(3, 4), wg=e,
                               wu=e.clone(), wd=wd, top=2,
                               residual=torch.zeros(3, 16))),
        "moe_given": (dpar.moe, dict(x=x, logits=None, wg=e, wu=e.clone(),
                                     wd=wd,
                                     index=torch.zeros(3, 2,
                                                       dtype=torch.int32),
                                     weight=torch.ones(3, 2))),
        "moe_int8": (dpar.moe, dict(x=x.half(), logits=torch.zeros(3, 4),
                                    top=2, **eight)),
    }


CASES = [(call, name) for call, (_, kw) in operands().items()
         for name, t in kw.items()
         if torch.is_tensor(t) and t.is_floating_point()]


@pytest.mark.parametrize("call,name", CASES)
def test_a_tangent_is_refused(call, name):
    fn, kw = operands()[call]
    with forward_ad.dual_level():
        kw[name] = forward_ad.make_dual(kw[name], torch.ones_like(kw[name]))
        with pytest.raises(ValueError, match=MATCH):
            fn(**kw)
        with torch.no_grad():           # which leaves forward mode on
            with pytest.raises(ValueError, match=MATCH):
                fn(**kw)


@pytest.mark.parametrize("call", operands())
def test_tensors_without_one_pass_the_check(call):
    """(to the device, which is none here)"""
    fn, kw = operands()[call]
    with forward_ad.dual_level():
        forward_ad.make_dual(torch.zeros(2), torch.ones(2))
        for level in (False, True):
            with pytest.raises(Exception) as e:
                if level:
                    with forward_ad._set_fwd_grad_enabled(False):
                        name = next(k for k, t in kw.items()
                                    if torch.is_tensor(t)
                                    and t.is_floating_point())
                        kw[name] = forward_ad.make_dual(
                            kw[name], torch.ones_like(kw[name]))
                        fn(**kw)
                else:
                    fn(**kw)
            assert MATCH not in str(e.value)


@pytest.mark.parametrize("call,name", CASES)
def test_no_silent_result_under_jvp(call, name):
    fn, kw = operands()[call]
    with pytest.raises((ValueError, RuntimeError)):
        torch.func.jvp(lambda t: fn(**{**kw, name: t}), (kw[name],),
                       (torch.ones_like(kw[name]),))
