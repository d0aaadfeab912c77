#!/usr/bin/env python3
"""The experts' products as they are used together: the experts of one MoE layer are trained for a few steps, their weights are
quantised, and the layer is served in 4 bits.

    python examples/train_and_serve_experts.py

Tokens are routed and sorted once (moe_gate_topk, moe_dispatch).  A training step is

    z = x_sorted W1_e^T + b1_e       moe_grouped_product
    y = GELU(z) W2_e^T + b2_e        moe_grouped_product
    L = mean |y - target|^2 / 2
    dh = dy W2_e, dW2, db2           moe_grouped_product_dx, moe_grouped_product_dw
    dW1, db1                         moe_grouped_product_dw

with weights in bf16, gradients in fp32 and fp32 copies of the weights that Adam takes its steps on.  Targets are the outputs of experts
of the same shape with other weights.  Serving calls moe_grouped_product_mx4, which quantises the rows on the way.
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2401_08383_amd as exf  # noqa: E402

DEV = "cuda"


def forward(x, offsets, w1, b1, w2, b2):
    """(pre-activations, hidden activations, outputs) of the experts on their rows."""
    z = exf.moe_grouped_product(x, offsets, w1, b1)
    h = torch.nn.functional.gelu(z)
    return z, h, exf.moe_grouped_product(h, offsets, w2, b2)


def gradients(x, offsets, w2, z, h, dy):
    """Gradients of W1, b1, W2, b2, in fp32."""
    dw2, db2 = exf.moe_grouped_product_dw(dy, h, offsets, want_bias=True, grad_dtype=torch.float32)
    dh = exf.moe_grouped_product_dx(dy, offsets, w2)
    dz = torch.ops.aten.gelu_backward(dh, z)
    dw1, db1 = exf.moe_grouped_product_dw(dz, x, offsets, want_bias=True, grad_dtype=torch.float32)
    return dw1, db1, dw2, db2


def serve(x, offsets, w1, b1, w2, b2):
    """The outputs with weights held in 4 bits."""
    h = torch.nn.functional.gelu(exf.moe_grouped_product_mx4(x, offsets, w1, b1))
    return exf.moe_grouped_product_mx4(h, offsets, w2, b2)


def run(tokens=2048, d=256, f=1024, experts=8, steps=30, rate=3e-3, seed=0, say=print):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    normal = lambda *shape, std=1.0: torch.empty(shape, device=DEV).normal_(0.0, std, generator=g)  # noqa: E731
    shapes = ((experts, f, d), (experts, f), (experts, d, f), (experts, d))
    stds = (d ** -0.5, 0.1, f ** -0.5, 0.1)
    teacher = [normal(*shape, std=s).bfloat16() for shape, s in zip(shapes, stds)]
    master = [t.float() + normal(*t.shape, std=0.3 * s) for t, s in zip(teacher, stds)]
    adam = torch.optim.Adam(master, lr=rate)

    x = normal(tokens, d).bfloat16()
    idx, _, _ = exf.moe_gate_topk(x, normal(experts, d, std=d ** -0.5).bfloat16(), 1)
    sent = exf.moe_dispatch(x, idx, experts)
    rows, offsets = sent.x_sorted, sent.expert_offsets
    target = forward(rows, offsets, *teacher)[2]

    losses = []
    for step in range(steps):
        w = [m.bfloat16() for m in master]
        z, h, y = forward(rows, offsets, *w)
        off = y.float() - target.float()
        losses.append(0.5 * float(off.square().mean()))
        # (a row's share of its expert's mean: experts of many rows and of few take steps of one size)
        share = 1.0 / sent.expert_counts.clamp(min=1).float()
        dy = (off * torch.repeat_interleave(share, sent.expert_counts.long(), output_size=tokens)[:, None]).bfloat16()
        for m, grad in zip(master, gradients(rows, offsets, w[2], z, h, dy)):
            m.grad = grad
        adam.step()
        if step % 10 == 0 or step == steps - 1:
            say(f"step {step:3d}  loss {losses[-1]:.6f}")

    w = [m.bfloat16() for m in master]
    full = forward(rows, offsets, *w)[2].float()
    held = exf.mx4_quantize(w[0]), exf.mx4_quantize(w[2])
    small = serve(rows, offsets, held[0], w[1], held[1], w[3]).float()
    away = float((small - full).norm() / full.norm())
    size = sum(t.numel() for h in held for t in (h.q, h.scale)) / (2 * sum(t.numel() for t in (w[0], w[2])))
    say(f"served in 4 bits: weights {size:.3f} of their size in bf16, outputs {away:.3f} away (relative)")
    return dict(losses=losses, away=away, size=size)


if __name__ == "__main__":
    run()
