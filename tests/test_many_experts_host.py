"""What the calls of many experts and of 4-bit integers refuse, without a GPU, and the reference that their results are tested against."""
import ctypes
import itertools

import pytest
import torch

import many_experts_reference as R
import paper_2401_08383_amd as exf
from paper_2401_08383_amd import binding as B

BF, F32, I32, U8 = torch.bfloat16, torch.float32, torch.int32, torch.uint8


def _p(i):  # aligned dummies, far apart; never dereferenced on these paths
    return ctypes.c_void_p((i + 1) << 40)


ODD = ctypes.c_void_p((99 << 40) + 4)


def _route(logits=_p(0), bias=None, T=4, E=64, k=8, score=0, groups=1, top=1, best=1, renorm=1, scale=1.0, dt=B.EXF_F32, idx=_p(1), w=_p(2), scores=None):
    return exf.lib().moe_route(logits, bias, T, E, k, score, groups, top, best, renorm, scale, dt, idx, w, scores, None)


def _route_backward(dw=_p(0), logits=_p(1), idx=_p(2), ds=None, stride=0, T=4, E=64, k=8, score=0, renorm=1, scale=1.0, dt=B.EXF_F32, out=_p(3)):
    return exf.lib().moe_route_backward(dw, logits, idx, ds, stride, T, E, k, score, renorm, scale, dt, out, None)


def _dispatch(x=_p(0), idx=_p(1), T=4, d=64, k=8, E=128, E_local=64, dt=B.EXF_BF16, xs=_p(2), src=_p(3), pos=_p(4), counts=_p(5), off=_p(6), ws=_p(7), size=1 << 20):
    return exf.lib().moe_dispatch_topk(x, idx, None, T, d, k, E, E_local, dt, xs, src, pos, counts, off, ws, size, None)


def _combine(y=_p(0), pos=_p(1), w=_p(2), T=4, d=64, k=8, dt=B.EXF_BF16, out=_p(3)):
    return exf.lib().moe_combine_topk(y, pos, w, T, d, k, dt, out, None)


def _combine_backward(dout=_p(0), y=_p(1), pos=_p(2), w=_p(3), T=4, d=64, k=8, dt=B.EXF_BF16, dy=_p(4), dw=_p(5)):
    return exf.lib().moe_combine_backward(dout, y, pos, w, T, d, k, dt, dy, dw, None)


def _quantise(x=_p(0), rows=4, k=256, group=128, dt=B.EXF_BF16, q=_p(1), s=_p(2), z=None):
    return exf.lib().q4_quantize(x, rows, k, group, dt, q, s, z, None)


def _dequantise(q=_p(0), s=_p(1), z=None, rows=4, k=256, group=128, dt=B.EXF_BF16, out=_p(2)):
    return exf.lib().q4_dequantize(q, s, z, rows, k, group, dt, out, None)


def _product(x=_p(0), off=_p(1), w=_p(2), s=_p(3), z=None, b=None, A=4, n=64, k=256, group=128, E=8, dt=B.EXF_BF16, y=_p(4)):
    return exf.lib().moe_grouped_product_q4(x, off, w, s, z, b, A, n, k, group, E, dt, y, None)


SHAPES = [(_route, b) for b in (dict(T=-1), dict(T=1 << 28), dict(T=1 << 62), dict(E=0), dict(E=513), dict(k=0), dict(k=17), dict(E=7), dict(score=2), dict(score=-1), dict(groups=0),
                                dict(groups=3), dict(E=128, groups=128), dict(groups=8, top=0), dict(groups=8, top=9), dict(best=0), dict(best=3),
                                dict(groups=16, top=1), dict(scale=float("nan")), dict(scale=float("inf")))]
SHAPES += [(_route_backward, b) for b in (dict(T=-1), dict(T=1 << 28), dict(E=0), dict(E=513), dict(k=0), dict(k=17), dict(E=7), dict(score=2), dict(ds=_p(5), stride=63),
                                          dict(ds=_p(5), stride=-64), dict(scale=float("inf")))]
SHAPES += [(_dispatch, b) for b in (dict(T=-1), dict(T=1 << 28), dict(T=1 << 61), dict(k=0), dict(k=17), dict(E=0), dict(E_local=65), dict(E_local=0), dict(d=60))]
SHAPES += [(c, b) for c in (_combine, _combine_backward) for b in (dict(T=-1), dict(T=1 << 28), dict(T=1 << 62), dict(k=0), dict(k=17), dict(d=0), dict(d=60), dict(dt=B.EXF_F32, d=62), dict(d=(1 << 21) + 8))]
SHAPES += [(c, b) for c in (_quantise, _dequantise) for b in (dict(rows=-1), dict(rows=1 << 40), dict(k=0), dict(k=192), dict(group=16), dict(group=256), dict(group=0), dict(k=-128))]
SHAPES += [(_product, b) for b in (dict(A=-1), dict(A=1 << 31), dict(n=0), dict(n=60), dict(n=(1 << 21) + 8), dict(k=192), dict(group=16), dict(group=0), dict(E=0), dict(E=65), dict(dt=B.EXF_F32, n=62))]


@pytest.mark.parametrize("call,bad", SHAPES)
def test_shapes(call, bad):
    assert call(**bad) == B.EXF_ERR_BAD_SHAPE
    name = {_route: "moe_route", _route_backward: "moe_route_backward", _dispatch: "moe_dispatch_topk", _combine: "moe_combine_topk", _combine_backward: "moe_combine_backward",
            _quantise: "q4_quantize", _dequantise: "q4_dequantize", _product: "moe_grouped_product_q4"}[call]
    assert B.last_error().startswith(name + ":")


CALLS = [_route, _route_backward, _dispatch, _combine, _combine_backward, _quantise, _dequantise, _product]


@pytest.mark.parametrize("call", CALLS)
def test_types(call):
    assert call(dt=2) == B.EXF_ERR_BAD_DTYPE and call(dt=-1) == B.EXF_ERR_BAD_DTYPE


@pytest.mark.parametrize("call,names", zip(CALLS, ("logits idx w", "dw logits idx out", "x idx src pos counts off ws", "y pos out", "dout y pos w", "x q s", "q s out", "x off w s y")))
def test_null_pointers(call, names):
    for name in names.split():
        assert call(**{name: None}) == B.EXF_ERR_NULL_PTR, name


@pytest.mark.parametrize("call,names", zip(CALLS, ("logits scores", "logits ds out", "x xs", "y out", "dout y dy", "x q s z", "q s z out", "x w s z b y")))
def test_misaligned_pointers(call, names):
    for name in names.split():
        assert call(**{name: ODD}) == B.EXF_ERR_MISALIGNED, name


def _near(i, by=16):
    return ctypes.c_void_p(((i + 1) << 40) + by)


@pytest.mark.parametrize("call,bad", [(_route, dict(idx=_near(0))), (_route, dict(w=_near(0))), (_route, dict(scores=_near(0))), (_route, dict(w=_near(1))), (_route, dict(scores=_near(2))),
                                      (_route, dict(bias=_p(1))), (_route_backward, dict(out=_near(0))), (_route_backward, dict(out=_p(1))), (_route_backward, dict(out=_near(2))),
                                      (_route_backward, dict(ds=_near(3))), (_combine, dict(out=_near(0, 256))), (_combine, dict(out=_near(1))), (_combine, dict(out=_near(2))),
                                      (_combine_backward, dict(dy=_p(0))), (_combine_backward, dict(dy=_p(1))), (_combine_backward, dict(dw=_near(1))),
                                      (_combine_backward, dict(dw=_p(3))), (_combine_backward, dict(dw=_near(4))), (_quantise, dict(q=_p(0))), (_quantise, dict(s=_near(1))),
                                      (_quantise, dict(z=_p(2))), (_dequantise, dict(out=_near(0))), (_product, dict(y=_p(0))), (_product, dict(y=_near(2))), (_product, dict(y=_near(3))),
                                      (_product, dict(z=_p(4))), (_product, dict(b=_near(4)))])
def test_arrays_that_overlap(call, bad):
    assert call(**bad) == B.EXF_ERR_BAD_SHAPE


def test_no_rows_launch_nothing():
    assert _route(T=0, logits=None, idx=None, w=None) == B.EXF_OK and _route_backward(T=0, logits=None, out=None) == B.EXF_OK
    assert _combine(T=0, y=None, out=None) == B.EXF_OK and _combine_backward(T=0, dout=None) == B.EXF_OK
    assert _combine_backward(dy=None, dw=None) == B.EXF_OK  # nothing is wanted
    assert _quantise(rows=0, x=None) == B.EXF_OK and _dequantise(rows=0, out=None) == B.EXF_OK and _product(A=0, x=None, y=None) == B.EXF_OK


def test_dispatch_workspace():
    need = exf.lib().moe_dispatch_workspace_bytes(1000, 8, 64)
    assert _dispatch(T=1000, size=need - 1) == B.EXF_ERR_WORKSPACE_TOO_SMALL


def _arguments(dev="cpu", dt=BF):
    z = lambda *s, t=dt: torch.zeros(s, dtype=t, device=dev)  # noqa: E731
    return dict(logits=z(4, 8), idx=z(4, 3, t=I32), w=z(4, 3, t=F32), bias=z(8, t=F32), y=z(12, 64), pos=z(12, t=I32), dout=z(4, 64), off=z(4, t=I32),
                q=exf.Q4(z(3, 64, 32, t=U8), z(3, 64, 2), z(3, 64, 2, t=U8)), x=z(4, 64))


def _fine(a):
    return {
        "route": lambda: exf.moe_route(a["logits"], 3, a["bias"]),
        "route_backward": lambda: exf.moe_route_backward(a["w"], a["logits"], a["idx"], dscores=a["bias"]),
        "dispatch": lambda: exf.moe_dispatch(a["x"], a["idx"], 8),
        "dispatch_backward": lambda: exf.moe_dispatch_backward(a["y"], a["pos"], 3),
        "combine": lambda: exf.moe_combine(a["y"], a["pos"], a["w"]),
        "combine_backward": lambda: exf.moe_combine_backward(a["dout"], a["y"], a["pos"], a["w"]),
        "quantise": lambda: exf.q4_quantize(a["x"], 32),
        "dequantise": lambda: exf.q4_dequantize(a["q"]),
        "product": lambda: exf.moe_grouped_product_q4(a["x"], a["off"], a["q"]),
    }


class NothingIsLaunched:
    def __getattr__(self, name):
        if name.endswith("_bytes"):
            return getattr(B._lib, name)
        if name in ("moe_dispatch_topk", "moe_combine_topk", "moe_combine_backward", "moe_route", "moe_route_backward", "q4_quantize", "q4_dequantize", "moe_grouped_product_q4"):
            return lambda *arguments: pytest.fail(f"{name} was called")
        pytest.fail(f"{name} was called")


@pytest.fixture
def nothing_is_launched(monkeypatch):
    exf.lib()
    monkeypatch.setattr(B, "lib", NothingIsLaunched)
    monkeypatch.setattr(B, "_stream", lambda: None)


@pytest.mark.parametrize("call", list(_fine(_arguments())))
@pytest.mark.parametrize("dt", [BF, F32])
def test_host_tensors_are_refused(nothing_is_launched, call, dt):
    with pytest.raises(exf.ExflowError, match="on the host"):
        _fine(_arguments(dt=dt))[call]()


@pytest.mark.parametrize("call", list(_fine(_arguments())))
def test_tensors_of_a_device_that_is_not_the_current_one_are_refused(nothing_is_launched, monkeypatch, call):
    monkeypatch.setattr(torch.Tensor, "get_device", lambda t: 1)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    with pytest.raises(exf.ExflowError, match="on device 1, the current one is 0"):
        _fine(_arguments())[call]()


@pytest.mark.parametrize("call,names", [("route", "logits"), ("route_backward", "w logits bias"), ("dispatch", "x"), ("dispatch_backward", "y"), ("combine", "y w"),
                                        ("combine_backward", "dout y w"), ("product", "x")])
def test_gradients_are_not_lost_without_a_word(nothing_is_launched, call, names):
    for name in names.split():
        a = _arguments()
        a[name] = a[name].requires_grad_()
        with pytest.raises(exf.ExflowError, match="autograd") as caught:
            _fine(a)[call]()
        assert caught.value.code == B.EXF_ERR_NOT_IMPLEMENTED
        with torch.no_grad(), pytest.raises(exf.ExflowError, match="on the host"):
            _fine(a)[call]()


def test_the_binding_refuses_what_the_library_cannot_see(nothing_is_launched):
    a = _arguments()
    logits, idx, w, bias, y, pos, dout, off, q, x = (a[n] for n in ("logits", "idx", "w", "bias", "y", "pos", "dout", "off", "q", "x"))
    bad = [
        lambda: exf.moe_route(logits.half(), 3),
        lambda: exf.moe_route(logits.t(), 3),
        lambda: exf.moe_route(logits[0], 3),
        lambda: exf.moe_route(logits, 3, bias[:7]),
        lambda: exf.moe_route(logits, 3, bias.to(BF)),
        lambda: exf.moe_route_backward(w[:, :2], logits, idx),
        lambda: exf.moe_route_backward(w.to(BF), logits, idx),
        lambda: exf.moe_route_backward(w, logits, idx.long()),
        lambda: exf.moe_route_backward(w, logits, idx[:3]),
        lambda: exf.moe_route_backward(w, logits, idx, dscores=bias[:7]),
        lambda: exf.moe_route_backward(w, logits, idx, dscores=torch.zeros(3, 8)),
        lambda: exf.moe_route_backward(w, logits, idx, out=logits.float()),
        lambda: exf.moe_dispatch(x[:3], idx, 8),
        lambda: exf.moe_dispatch(x, idx, 8, expert_map=idx[0]),
        lambda: exf.moe_combine(y[:11], pos, w),
        lambda: exf.moe_combine(y, pos[:9], w),
        lambda: exf.moe_combine(y, pos.long(), w),
        lambda: exf.moe_combine(y, pos, w.to(BF)),
        lambda: exf.moe_combine(y, pos, w, out=y),
        lambda: exf.moe_dispatch_backward(y, pos, 5),
        lambda: exf.moe_dispatch_backward(y, pos, 0),
        lambda: exf.moe_dispatch_backward(y, pos.view(3, 4), 3),
        lambda: exf.moe_combine_backward(dout[:3], y, pos, w),
        lambda: exf.moe_combine_backward(dout.float(), y, pos, w),
        lambda: exf.moe_combine_backward(dout, y, pos, w, out=y[:11]),
        lambda: exf.moe_combine_backward(dout, y, pos, w.view(-1)),
        lambda: exf.q4_quantize(x, 48),
        lambda: exf.q4_quantize(x.half(), 32),
        lambda: exf.q4_quantize(x.t(), 4),
        lambda: exf.q4_quantize(x, 32, out=q),
        lambda: exf.q4_quantize(torch.zeros(3, 64, 64, dtype=BF), 32, symmetric=True, out=q),
        lambda: exf.q4_quantize(torch.zeros((), dtype=BF), 32),
        lambda: exf.q4_dequantize(exf.Q4(q.q, q.scale[:, :63], q.zero)),
        lambda: exf.q4_dequantize(exf.Q4(q.q, q.scale, q.zero[..., :1])),
        lambda: exf.q4_dequantize(exf.Q4(q.q, q.scale, q.zero.int())),
        lambda: exf.q4_dequantize(q, out=torch.zeros(3, 64, 64)),
        lambda: exf.moe_grouped_product_q4(x.float(), off, q),
        lambda: exf.moe_grouped_product_q4(x[:, :32], off, q),
        lambda: exf.moe_grouped_product_q4(x, off[:3], q),
        lambda: exf.moe_grouped_product_q4(x, off, exf.Q4(q.q[0], q.scale[0])),
        lambda: exf.moe_grouped_product_q4(x, off, q, torch.zeros(3, 32, dtype=BF)),
        lambda: exf.moe_grouped_product_q4(x, off, q, out=torch.zeros(4, 64)),
    ]
    for i, call in enumerate(bad):
        with pytest.raises(exf.ExflowError) as caught:
            call()
            pytest.fail(f"case {i} was taken")
        assert "on the host" not in str(caught.value), i


@pytest.mark.parametrize("score,renorm,k", [(s, r, k) for s, r, k in itertools.product((0, 1), (False, True), (1, 3)) if not (r and k == 1)])
def test_the_reference_gradient_against_differences(score, renorm, k):
    g = torch.Generator().manual_seed(3)
    l, dw, ds = torch.randn(5, 9, generator=g).double(), torch.randn(5, k, generator=g).double(), torch.randn(9, generator=g).double()
    idx = R.route(l, k)[0]
    idx[0, -1] = -1
    if k > 1:
        idx[1, 1] = idx[1, 0]  # the same expert twice

    def loss(l):
        return float((R.weights(l, idx, score, renorm, 1.7) * dw).sum() + (R.scores(l, score) * ds).sum())

    got, _ = R.route_gradient(l, idx, dw, score, renorm, 1.7, ds)
    for t, e in itertools.product(range(5), range(9)):
        h = torch.zeros_like(l)
        h[t, e] = 1e-5
        assert abs((loss(l + h) - loss(l - h)) / 2e-5 - float(got[t, e])) < 1e-9


@pytest.mark.parametrize("symmetric", [False, True])
def test_the_reference_quantisation(symmetric):
    """... is the nearest of the sixteen values of a group."""
    x = torch.randn(40, 64, generator=torch.Generator().manual_seed(5)).to(BF)
    code, scale, zero = R.q4_quantised(x, 32, symmetric)
    q = code[..., 0::2] + 16 * code[..., 1::2]
    v = R.q4_values(q, scale, zero)
    at = torch.full_like(scale.double(), 8.0) if zero is None else zero.double()
    all16 = (torch.arange(16).double() - at[..., None]) * scale.double()[..., None]
    off = (x.double().view(40, 2, 32, 1) - all16[:, :, None, :]).abs().amin(-1).view(40, 64)
    assert torch.allclose((v - x.double()).abs(), off, rtol=0, atol=1e-12)
