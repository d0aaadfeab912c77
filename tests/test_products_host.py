"""What the experts' products refuse, without a GPU: bad arguments come back as errors before anything could be launched."""
import ctypes

import pytest
import torch

import paper_2401_08383_amd as exf
from paper_2401_08383_amd import binding as B


def _p(i):  # aligned dummies, far apart; never dereferenced on these paths
    return ctypes.c_void_p((i + 1) << 32)


ODD = ctypes.c_void_p((99 << 32) + 4)


def _product(x=_p(0), off=_p(1), w=_p(2), b=None, A=4, n=64, k=32, E=8, dt=B.EXF_BF16, y=_p(3)):
    return exf.lib().moe_grouped_product(x, off, w, b, A, n, k, E, dt, y, None)


def _dx(dy=_p(0), off=_p(1), w=_p(2), A=4, n=64, k=32, E=8, dt=B.EXF_BF16, dx=_p(3)):
    return exf.lib().moe_grouped_product_dx(dy, off, w, A, n, k, E, dt, dx, None)


def _dw(dy=_p(0), x=_p(1), off=_p(2), A=4, n=64, k=32, E=8, dt=B.EXF_BF16, grad=B.EXF_F32, dw=_p(3), db=None, ws=_p(4), size=1 << 31):
    return exf.lib().moe_grouped_product_dw(dy, x, off, A, n, k, E, dt, grad, dw, db, ws, size, None)


def _mx4(x=_p(0), xs=_p(1), off=_p(2), w=_p(3), ws=_p(4), b=None, A=4, n=64, k=32, E=8, dt=B.EXF_BF16, y=_p(5), work=None, size=0):
    return exf.lib().moe_grouped_product_mx4(x, xs, off, w, ws, b, A, n, k, E, dt, y, work, size, None)


def _quantise(x=_p(0), rows=4, k=64, dt=B.EXF_BF16, q=_p(1), s=_p(2)):
    return exf.lib().mx4_quantize(x, rows, k, dt, q, s, None)


def _dequantise(q=_p(1), s=_p(2), rows=4, k=64, dt=B.EXF_BF16, out=_p(0)):
    return exf.lib().mx4_dequantize(q, s, rows, k, dt, out, None)


SHAPES = [dict(A=-1), dict(A=1 << 31), dict(n=0), dict(n=-8), dict(n=60), dict(k=0), dict(k=36), dict(E=0), dict(E=65), dict(dt=B.EXF_F32, n=62), dict(n=(1 << 21) + 8), dict(k=(1 << 21) + 32)]


@pytest.mark.parametrize("call", [_product, _dx, _dw, _mx4])
@pytest.mark.parametrize("bad", SHAPES)
def test_shapes(call, bad):
    if call is _dw and bad.get("dt") == B.EXF_F32:
        bad = dict(bad, grad=B.EXF_F32)
    assert call(**bad) == B.EXF_ERR_BAD_SHAPE and B.last_error()


@pytest.mark.parametrize("call,bad", [(_product, dict(dt=2)), (_dx, dict(dt=-1)), (_dw, dict(dt=5)), (_mx4, dict(dt=2)), (_quantise, dict(dt=2)), (_dequantise, dict(dt=9)),
                                      (_dw, dict(grad=2)), (_dw, dict(dt=B.EXF_F32, grad=B.EXF_BF16))])
def test_types(call, bad):
    assert call(**bad) == B.EXF_ERR_BAD_DTYPE


@pytest.mark.parametrize("call,names", [(_product, "x off w y"), (_dx, "dy off w dx"), (_dw, "dy x off dw"), (_mx4, "x off w ws y"), (_quantise, "x q s"), (_dequantise, "q s out")])
def test_null_pointers(call, names):
    for name in names.split():
        assert call(**{name: None}) == B.EXF_ERR_NULL_PTR, name


@pytest.mark.parametrize("call,names", [(_product, "x w b y"), (_dx, "dy w dx"), (_dw, "dy x dw db"), (_mx4, "x xs w ws b y"), (_quantise, "x q s"), (_dequantise, "q s out")])
def test_misaligned_pointers(call, names):
    for name in names.split():
        assert call(**{name: ODD}) == B.EXF_ERR_MISALIGNED, name


def _near(i, by):
    return ctypes.c_void_p(((i + 1) << 32) + by)


@pytest.mark.parametrize("call,bad", [(_product, dict(y=_p(0))), (_product, dict(y=_near(2, 64))), (_product, dict(y=_p(7), b=_p(7))), (_dx, dict(dx=_p(0))), (_dx, dict(dx=_near(0, 256))),
                                      (_dw, dict(dw=_p(0))), (_dw, dict(dw=_near(1, 16))), (_dw, dict(db=_near(3, 64))), (_mx4, dict(y=_p(0))), (_mx4, dict(y=_near(3, 16))),
                                      (_quantise, dict(q=_p(0))), (_quantise, dict(s=_near(1, 16))), (_dequantise, dict(out=_p(1)))])
def test_arrays_that_overlap(call, bad):
    assert call(**bad) == B.EXF_ERR_BAD_SHAPE


def test_blocks():
    for k in (0, 16, 33, 48, -32):
        assert _quantise(k=k) == B.EXF_ERR_BAD_SHAPE and _dequantise(k=k) == B.EXF_ERR_BAD_SHAPE
    assert _quantise(rows=-1) == B.EXF_ERR_BAD_SHAPE
    assert _mx4(k=40) == B.EXF_ERR_BAD_SHAPE and _mx4(k=48) == B.EXF_ERR_BAD_SHAPE


def test_workspaces():
    lib = exf.lib()
    need = lib.moe_grouped_product_mx4_workspace_bytes(1000, 4096, 96)
    assert need >= 1000 * 48 + 1000 * 8
    big = dict(xs=None, A=1000, n=4096, k=96)
    assert _mx4(**big) == B.EXF_ERR_NULL_PTR
    assert _mx4(**big, work=_p(8), size=need - 1) == B.EXF_ERR_WORKSPACE_TOO_SMALL
    assert _mx4(**big, work=ODD, size=need) == B.EXF_ERR_MISALIGNED
    assert _mx4(**big, work=_p(0), size=need) == B.EXF_ERR_BAD_SHAPE  # over the rows
    assert lib.moe_grouped_product_mx4_workspace_bytes(-1, 64, 96) == 0
    assert lib.moe_grouped_product_mx4_workspace_bytes(B.EXF_MX4_INLINE_ROWS, 1 << 20, 1 << 14) == 0  # whatever the weights
    assert lib.moe_grouped_product_mx4_workspace_bytes(100, 64, 96) == 0
    for dt in (B.EXF_F32, B.EXF_BF16):
        need = lib.moe_grouped_product_dw_workspace_bytes(1 << 20, 64, 64, 1, dt)
        if need:
            assert _dw(A=1 << 20, k=64, E=1, dt=dt, size=need - 1) == B.EXF_ERR_WORKSPACE_TOO_SMALL
            assert _dw(A=1 << 20, k=64, E=1, dt=dt, ws=None) == B.EXF_ERR_NULL_PTR
    assert lib.mx4_scale_bytes(10, 257) == 2 * 10 * 8 and lib.mx4_scale_bytes(-1, 32) == 0


def test_no_rows_launch_nothing():
    assert _product(A=0, x=None, y=None) == B.EXF_OK and _dx(A=0, dy=None, dx=None) == B.EXF_OK
    assert _mx4(A=0, x=None, y=None) == B.EXF_OK
    assert _quantise(rows=0, x=None) == B.EXF_OK and _dequantise(rows=0, out=None) == B.EXF_OK


def test_the_binding_refuses_what_the_library_cannot_see():
    """Tensors whose shape, type, layout or number of rows does not fit the others."""
    bf, f32 = torch.bfloat16, torch.float32
    x, dy, w, off = torch.zeros(4, 32, dtype=bf), torch.zeros(4, 64, dtype=bf), torch.zeros(3, 64, 32, dtype=bf), torch.zeros(4, dtype=torch.int32)
    held = exf.Mx4(torch.zeros(3, 64, 16, dtype=torch.uint8), torch.zeros(1, 192, 8, dtype=torch.uint8))
    bad = [
        lambda: exf.moe_grouped_product(x[:, :16], off, w),
        lambda: exf.moe_grouped_product(x.t(), off, w),
        lambda: exf.moe_grouped_product(x, off[:3], w),
        lambda: exf.moe_grouped_product(x, off.long(), w),
        lambda: exf.moe_grouped_product(x, off, w.float()),
        lambda: exf.moe_grouped_product(x, off, w.transpose(1, 2)),
        lambda: exf.moe_grouped_product(x, off, w, torch.zeros(3, 32, dtype=bf)),
        lambda: exf.moe_grouped_product(x, off, w, out=torch.zeros(3, 64, dtype=bf)),
        lambda: exf.moe_grouped_product(x, off, w, out=torch.zeros(4, 64, dtype=f32)),
        lambda: exf.moe_grouped_product(x, off, w, out=torch.zeros(4, 128, dtype=bf)[:, ::2]),
        lambda: exf.moe_grouped_product(x.half(), off, w.half()),
        lambda: exf.moe_grouped_product(x, off, w[0]),
        lambda: exf.moe_grouped_product_dx(x, off, w),
        lambda: exf.moe_grouped_product_dx(dy, off, w, out=torch.zeros(4, 64, dtype=bf)),
        lambda: exf.moe_grouped_product_dw(dy[:3], x, off),
        lambda: exf.moe_grouped_product_dw(dy.float(), x, off),
        lambda: exf.moe_grouped_product_dw(dy, x, off, out=torch.zeros(3, 32, 64, dtype=bf)),
        lambda: exf.moe_grouped_product_dw(dy, x, off, grad_dtype=torch.float16),
        lambda: exf.moe_grouped_product_dw(dy, x, off, out_bias=torch.zeros(3, 64, dtype=f32)),
        lambda: exf.mx4_quantize(torch.zeros(4, 48, dtype=bf)),
        lambda: exf.mx4_quantize(torch.zeros(64, 4, dtype=bf).t()),
        lambda: exf.mx4_quantize(torch.zeros(4, 64, dtype=bf), out=held),
        lambda: exf.mx4_quantize(torch.zeros(4, 64, dtype=torch.float16)),
        lambda: exf.mx4_dequantize(exf.Mx4(held.q, held.scale[:, :191])),
        lambda: exf.mx4_dequantize(held, out=torch.zeros(3, 64, 16, dtype=bf)),
        lambda: exf.moe_grouped_product_mx4(dy, off, held),
        lambda: exf.moe_grouped_product_mx4(x, off, exf.Mx4(held.q, held.scale.int())),
        lambda: exf.moe_grouped_product_mx4(x, off, held, dtype=f32),
        lambda: exf.moe_grouped_product_mx4(x, off, held, torch.zeros(3, 64, dtype=f32)),
        lambda: exf.moe_grouped_product_mx4(exf.Mx4(held.q[0, :4], held.scale[:, :5]), off, held),
    ]
    for i, call in enumerate(bad):
        with pytest.raises(exf.ExflowError):
            call()
            pytest.fail(f"case {i} was taken")
