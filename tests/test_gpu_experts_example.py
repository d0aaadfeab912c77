"""The example that trains experts and serves them in 4 bits: all of the experts' products together, against autograd in fp32."""
import importlib.util
import os

import pytest
import torch

from helpers import DEV

pytestmark = pytest.mark.gpu

PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "train_and_serve_experts.py")
spec = importlib.util.spec_from_file_location("train_and_serve_experts", PATH)
example = importlib.util.module_from_spec(spec)
spec.loader.exec_module(example)


def test_training_and_serving():
    out = example.run(tokens=700, d=128, f=320, experts=5, steps=30, say=lambda s: print(f"[case] {s}", flush=True))
    assert out["losses"][-1] < 0.5 * out["losses"][0]
    assert out["size"] == pytest.approx((0.5 + 1 / 32) / 2, rel=0.25)  # (k = 320: scale tiles of 256, padded)
    # each of two products rounds both operands to 4 bits: relative steps of at most 1/4, of uniform error 1/4 / sqrt(12) and less, four times
    assert 0.01 < out["away"] < 0.3


def test_gradients_against_autograd():
    """The example's gradients on bf16 values, against autograd on the same values in fp32: both round intermediate rows to bf16 or not at
    all, 2^-8 each, on a chain of three."""
    g = torch.Generator(device=DEV)
    g.manual_seed(3)
    normal = lambda *s: torch.empty(s, device=DEV).normal_(0.0, 1.0, generator=g)  # noqa: E731
    sizes, d, f = [60, 0, 130, 9], 64, 136
    E, A = len(sizes), sum(sizes)
    offsets = torch.tensor([0, 60, 60, 190, 199], dtype=torch.int32, device=DEV)
    x, dy = normal(A, d).bfloat16(), normal(A, d).bfloat16()
    w = [(normal(E, f, d) * d ** -0.5).bfloat16(), normal(E, f).bfloat16(), (normal(E, d, f) * f ** -0.5).bfloat16(), normal(E, d).bfloat16()]
    z, h, y = example.forward(x, offsets, *w)
    got = example.gradients(x, offsets, w[2], z, h, dy)
    ref = [t.float().requires_grad_() for t in w]
    rows = []
    for e in range(E):
        part = x[offsets[e]:offsets[e + 1]].float()
        rows.append(torch.nn.functional.gelu(part @ ref[0][e].t() + ref[1][e]) @ ref[2][e].t() + ref[3][e])
    torch.cat(rows).backward(dy.float())
    for name, a, b in zip(("dw1", "db1", "dw2", "db2"), got, ref):
        assert a.dtype == torch.float32
        assert float((a - b.grad).norm() / b.grad.norm()) < 3 * 2.0 ** -8, name
    assert float((y.float() - torch.cat(rows).detach()).norm() / y.float().norm()) < 3 * 2.0 ** -8
    assert (got[0][1] == 0).all() and (got[1][1] == 0).all()
