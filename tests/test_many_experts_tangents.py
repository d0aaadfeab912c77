"""Routing, rows and 4-bit weights carry no tangents: dual tensors of forward-mode differentiation are refused, and taken where there is nothing to carry on."""
import pytest
import torch
from torch.autograd import forward_ad

import paper_2401_08383_amd as exf
from paper_2401_08383_amd import binding as B

BF, F32, I32, U8 = torch.bfloat16, torch.float32, torch.int32, torch.uint8


def _arguments(k):
    z = lambda *s, t=BF: torch.zeros(s, dtype=t)  # noqa: E731
    return dict(logits=z(4, 8), idx=z(4, k, t=I32), w=z(4, k, t=F32), ds=z(8, t=F32), y=z(4 * k, 64), pos=z(4 * k, t=I32), dout=z(4, 64), off=z(4, t=I32), q=z(3, 64, 32, t=U8),
                scale=z(3, 64, 2), b=z(3, 64), x=z(4, 64))


CALLS = {
    "moe_route": ("logits", lambda a: exf.moe_route(a["logits"], 3)),
    "moe_route_backward": ("logits w ds", lambda a: exf.moe_route_backward(a["w"], a["logits"], a["idx"], dscores=a["ds"])),
    "moe_dispatch": ("x", lambda a: exf.moe_dispatch(a["x"], a["idx"], 8)),
    "moe_dispatch_backward": ("y", lambda a: exf.moe_dispatch_backward(a["y"], a["pos"], a["idx"].shape[1])),
    "moe_combine": ("y w", lambda a: exf.moe_combine(a["y"], a["pos"], a["w"])),
    "moe_combine_backward": ("dout y w", lambda a: exf.moe_combine_backward(a["dout"], a["y"], a["pos"], a["w"])),
    "q4_quantize": ("x", lambda a: exf.q4_quantize(a["x"], 32)),
    "q4_dequantize": ("scale", lambda a: exf.q4_dequantize(exf.Q4(a["q"], a["scale"]))),
    "moe_grouped_product_q4": ("x b scale", lambda a: exf.moe_grouped_product_q4(a["x"], a["off"], exf.Q4(a["q"], a["scale"]), a["b"])),
}


@pytest.mark.parametrize("k", [1, 2, 3])
@pytest.mark.parametrize("name", list(CALLS))
def test_tangents_are_not_lost_without_a_word(name, k):
    names, run = CALLS[name]
    for which in names.split():
        a = _arguments(k)
        with forward_ad.dual_level():
            plain = dict(a)
            a[which] = forward_ad.make_dual(a[which], torch.ones_like(a[which]))
            for mode in (torch.enable_grad, torch.no_grad):
                with mode(), pytest.raises(exf.ExflowError, match=f"{name} .*dual") as caught:
                    run(a)
                assert caught.value.code == B.EXF_ERR_NOT_IMPLEMENTED
            with pytest.raises(exf.ExflowError, match="on the host"):  # (as far as tensors on the host get)
                run(plain)
            with pytest.raises(exf.ExflowError, match="on the host"):
                run({**a, which: a[which].detach()})


def test_a_function_with_a_jvp():
    """... sees its arguments without their tangents."""
    a = _arguments(2)

    class Combine(torch.autograd.Function):
        @staticmethod
        def forward(ctx, y, w):
            with pytest.raises(exf.ExflowError, match="on the host"):
                exf.moe_combine(y, a["pos"], w)
            return y.sum() * w.sum()

        @staticmethod
        def jvp(ctx, dy, dw):
            return torch.ones((), dtype=F32)

    with forward_ad.dual_level():
        got = Combine.apply(forward_ad.make_dual(a["y"], torch.ones_like(a["y"])), a["w"])
        assert forward_ad.unpack_dual(got).tangent is not None
