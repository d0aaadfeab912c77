"""Rows to 4-bit integers and back record no autograd history: what requires a gradient is refused in grad mode."""
import pytest
import torch

import paper_2401_08383_amd as exf
from paper_2401_08383_amd import binding as B

BF, U8 = torch.bfloat16, torch.uint8


def _held(dev, dt=BF):
    g = torch.Generator().manual_seed(1)
    return exf.Q4(torch.randint(0, 256, (6, 32), generator=g).to(U8).to(dev), torch.rand(6, 2, generator=g).to(dt).to(dev), torch.randint(0, 16, (6, 2), generator=g).to(U8).to(dev))


@pytest.mark.parametrize("symmetric", [False, True])
def test_gradients_are_not_lost_without_a_word(symmetric):
    x, m = torch.zeros(6, 64, dtype=BF, requires_grad=True), _held("cpu")
    m.scale.requires_grad_()
    for name, run in (("q4_quantize", lambda: exf.q4_quantize(x, 32, symmetric)), ("q4_dequantize", lambda: exf.q4_dequantize(m))):
        with pytest.raises(exf.ExflowError, match=name) as caught:
            run()
        assert caught.value.code == B.EXF_ERR_NOT_IMPLEMENTED and "autograd" in str(caught.value)
        with torch.no_grad(), pytest.raises(exf.ExflowError, match="on the host"):  # (as far as tensors on the host get)
            run()


@pytest.mark.gpu
def test_parameters_where_nothing_is_recorded():
    x, m = torch.randn(6, 64, generator=torch.Generator().manual_seed(2)).to(BF).to("cuda:0"), _held("cuda:0")
    want, values = exf.q4_quantize(x, 32), exf.q4_dequantize(m)
    weight, scale = torch.nn.Parameter(x), torch.nn.Parameter(m.scale)
    with torch.no_grad():
        got = exf.q4_quantize(weight, 32)
        assert torch.equal(got.q, want.q) and torch.equal(got.scale, want.scale) and torch.equal(got.zero, want.zero)
        assert torch.equal(exf.q4_dequantize(exf.Q4(m.q, scale, m.zero)), values)
    assert torch.equal(exf.q4_quantize(weight.detach(), 32).q, want.q)
    with pytest.raises(exf.ExflowError, match="autograd"):
        exf.q4_quantize(weight, 32)
    with pytest.raises(exf.ExflowError, match="autograd"):
        exf.q4_dequantize(exf.Q4(m.q, scale, m.zero))
