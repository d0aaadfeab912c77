"""Tensors that no kernel of the experts' products may be given: well-formed ones on the host, workspaces on the host, and what has no rows or experts to speak of."""
import pytest
import torch

import paper_2401_08383_amd as exf
from paper_2401_08383_amd import binding as B

BF, F32 = torch.bfloat16, torch.float32


class NothingIsLaunched:
    """Stands for the library: sizes of workspaces may be asked for, everything else fails the test."""

    def __getattr__(self, name):
        if name.endswith("_bytes"):
            return getattr(B._lib, name)
        pytest.fail(f"{name} was called with host addresses")


def _calls(dt):
    x, dy, w, off = torch.zeros(300, 64, dtype=dt), torch.zeros(300, 64, dtype=dt), torch.zeros(3, 64, 64, dtype=dt), torch.zeros(4, dtype=torch.int32)
    held = exf.Mx4(torch.zeros(3, 64, 32, dtype=torch.uint8), torch.zeros(1, 192, 8, dtype=torch.uint8))
    rows = exf.Mx4(torch.zeros(300, 32, dtype=torch.uint8), torch.zeros(1, 300, 8, dtype=torch.uint8))
    return {
        "product": lambda: exf.moe_grouped_product(x, off, w),
        "product with a bias": lambda: exf.moe_grouped_product(x, off, w, torch.zeros(3, 64, dtype=dt), out=torch.zeros(300, 64, dtype=dt)),
        "dx": lambda: exf.moe_grouped_product_dx(dy, off, w),
        "dw": lambda: exf.moe_grouped_product_dw(dy, x, off, want_bias=True),
        "dw with a workspace": lambda: exf.moe_grouped_product_dw(dy, x, off, workspace=torch.zeros(1 << 20, dtype=torch.uint8)),
        "quantise": lambda: exf.mx4_quantize(x),
        "quantise into": lambda: exf.mx4_quantize(x, out=rows),
        "dequantise": lambda: exf.mx4_dequantize(rows, dt),
        "mx4": lambda: exf.moe_grouped_product_mx4(x, off, held),
        "mx4 of few rows": lambda: exf.moe_grouped_product_mx4(x[:2], off, held),
        "mx4 of rows in 4 bits": lambda: exf.moe_grouped_product_mx4(rows, off, held, dtype=dt),
    }


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("call", list(_calls(BF)))
def test_host_tensors_are_refused(monkeypatch, call, dt):
    run = _calls(dt)[call]
    exf.lib()
    monkeypatch.setattr(B, "lib", NothingIsLaunched)
    monkeypatch.setattr(B, "_stream", lambda: None)
    with pytest.raises(exf.ExflowError, match="on the host"):
        run()


def test_what_has_no_axes_is_refused():
    """... by the binding's own error."""
    x, dy, off, nothing = torch.zeros(4, 64, dtype=BF), torch.zeros(4, 64, dtype=BF), torch.zeros(4, dtype=torch.int32), torch.zeros((), dtype=torch.uint8)
    held, flat = exf.Mx4(torch.zeros(3, 64, 32, dtype=torch.uint8), torch.zeros(1, 192, 8, dtype=torch.uint8)), exf.Mx4(nothing, torch.zeros(1, 1, 8, dtype=torch.uint8))
    bad = [lambda: exf.moe_grouped_product_dw(dy, x, off[:0]), lambda: exf.moe_grouped_product_dw(dy, x, off[:1]), lambda: exf.mx4_dequantize(flat),
           lambda: exf.mx4_quantize(nothing.to(BF)), lambda: exf.moe_grouped_product_mx4(flat, off, held), lambda: exf.moe_grouped_product_mx4(x, off, flat)]
    for i, call in enumerate(bad):
        with pytest.raises(exf.ExflowError) as caught:
            call()
        assert caught.value.code == B.EXF_ERR_BAD_SHAPE, i


def test_workspaces():
    some = torch.zeros(64, dtype=F32)
    assert B._bytes_of(some, -1) == (some.data_ptr(), 256)
    for bad, dev in ((some, 0), (torch.zeros(64, 2)[:, 0], -1)):
        with pytest.raises(exf.ExflowError, match="workspace"):
            B._bytes_of(bad, dev)


@pytest.mark.gpu
def test_workspaces_on_the_host_are_refused():
    dev = torch.device("cuda:0")
    x, off = torch.zeros(5000, 64, dtype=BF, device=dev), torch.tensor([0, 5000], dtype=torch.int32, device=dev)
    need = exf.lib().moe_grouped_product_dw_workspace_bytes(5000, 64, 64, 1, B.EXF_BF16)
    assert need > 0
    host = torch.zeros(need, dtype=torch.uint8)
    with pytest.raises(exf.ExflowError, match="workspace"):
        exf.moe_grouped_product_dw(x, x, off, workspace=host)
    held = exf.mx4_quantize(torch.zeros(1, 8192, 64, dtype=BF, device=dev))
    need = exf.lib().moe_grouped_product_mx4_workspace_bytes(5000, 8192, 64)
    assert need > 0
    with pytest.raises(exf.ExflowError, match="workspace"):
        exf.moe_grouped_product_mx4(x, off, held, workspace=torch.zeros(need, dtype=torch.uint8))
    # ... and one of another type is as long as it is
    ws = torch.empty((need + 3) // 4, dtype=F32, device=dev)
    assert exf.moe_grouped_product_mx4(x, off, held, workspace=ws).shape == (5000, 8192)
