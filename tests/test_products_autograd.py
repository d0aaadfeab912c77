"""The experts' products record no autograd history: arguments that require gradients are refused in grad mode, and taken where nothing is recorded."""
import pytest
import torch

import paper_2401_08383_amd as exf
from paper_2401_08383_amd import binding as B

BF = torch.bfloat16


def _calls(dev):
    """name -> (arguments that may require a gradient, the call of them)"""
    def normal(seed, *shape):
        return (torch.randn(shape, generator=torch.Generator().manual_seed(seed)) * 0.25).to(BF).to(dev)

    off = torch.tensor([0, 20, 20, 50], dtype=torch.int32, device=dev)
    x, dy, w, b = normal(1, 50, 64), normal(2, 50, 96), normal(3, 3, 96, 64), normal(4, 3, 96)
    codes = torch.arange(3 * 96 * 32, device=dev).view(3, 96, 32).to(torch.uint8)
    held = exf.Mx4(codes, torch.full((1, 288, 8), 120, dtype=torch.uint8, device=dev))
    return {"product": ([x, w, b], lambda x, w, b: exf.moe_grouped_product(x, off, w, b)), "dx": ([dy, w], lambda dy, w: exf.moe_grouped_product_dx(dy, off, w)),
            "dw": ([dy, x], lambda dy, x: exf.moe_grouped_product_dw(dy, x, off)[0]), "mx4": ([x, b], lambda x, b: exf.moe_grouped_product_mx4(x, off, held, b))}


@pytest.mark.parametrize("call", ["product", "dx", "dw", "mx4"])
def test_gradients_are_not_lost_without_a_word(call):
    args, run = _calls("cpu")[call]
    for i in range(len(args)):
        given = [a.clone().requires_grad_() if i == j else a for j, a in enumerate(args)]
        with pytest.raises(exf.ExflowError, match="autograd") as caught:
            run(*given)
        assert caught.value.code == B.EXF_ERR_NOT_IMPLEMENTED
        with torch.no_grad(), pytest.raises(exf.ExflowError, match="on the host"):  # (as far as tensors on the host get)
            run(*given)


@pytest.mark.gpu
@pytest.mark.parametrize("call", ["product", "dx", "dw", "mx4"])
def test_parameters_where_nothing_is_recorded(call):
    args, run = _calls("cuda:0")[call]
    want = run(*args)
    given = [torch.nn.Parameter(a) for a in args]
    with torch.no_grad():
        assert torch.equal(run(*given), want)
    with pytest.raises(exf.ExflowError, match="autograd"):
        run(*given)


class Product(torch.autograd.Function):
    """moe_grouped_product with its gradients, as a program that uses autograd has it."""

    @staticmethod
    def forward(ctx, x, offsets, w, b):
        ctx.save_for_backward(x, offsets, w)
        return exf.moe_grouped_product(x, offsets, w, b)

    @staticmethod
    def backward(ctx, dy):
        x, offsets, w = ctx.saved_tensors
        dy = dy.contiguous()
        return exf.moe_grouped_product_dx(dy, offsets, w), None, *exf.moe_grouped_product_dw(dy, x, offsets, want_bias=True)


@pytest.mark.gpu
def test_in_a_function_of_autograd():
    args, _ = _calls("cuda:0")["product"]
    off = torch.tensor([0, 20, 20, 50], dtype=torch.int32, device="cuda:0")
    x, w, b = (a.float().requires_grad_() for a in args)
    c = torch.randn(50, 96, generator=torch.Generator().manual_seed(9)).to("cuda:0")
    (Product.apply(x, off, w, b) * c).sum().backward()
    assert torch.equal(x.grad, exf.moe_grouped_product_dx(c, off, w.detach()))
    dw, db = exf.moe_grouped_product_dw(c, x.detach(), off, want_bias=True)
    assert torch.equal(w.grad, dw) and torch.equal(b.grad, db) and float(dw.abs().sum()) > 0
