"""The rows of up to 16 experts a token: moe_dispatch, moe_combine and their gradients against their definitions in 64 bits."""
import pytest
import torch

import many_experts_reference as R
import paper_2401_08383_amd as exf
from paper_2401_08383_amd.binding import DispatchResult

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32
SIZES = [(1, 8, 1), (1, 2048, 8), (3, 16, 16), (17, 520, 3), (129, 1032, 6), (64, 64, 2), (1000, 256, 8), (333, 24, 5), (40, 4104, 10), (5, 20000, 9), (2100, 72, 16)]


def _d(d, dt):
    return d if dt == BF else d // 8 * 4 + 4


def _case(T, d, k, dt, kept, seed):
    g = torch.Generator().manual_seed(seed)
    position, src = R.assignments(T, k, 64, g, kept)
    normal = lambda *s: torch.randn(*s, generator=g).to(dt)  # noqa: E731
    return position, src, normal(T * k, d), normal(T, d), torch.rand(T, k, generator=g)


@pytest.mark.parametrize("T,d,k", SIZES)
@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("kept", [1.0, 0.3, 0.0])
def test_combine(T, d, k, dt, kept):
    d = _d(d, dt)
    print(f"[case] combine T={T} d={d} k={k} {dt} kept={kept}", flush=True)
    position, src, y, dout, w = _case(T, d, k, dt, kept, T + d)
    y[len(src):] = float("nan")  # rows behind the last kept one are not read
    for weights in (w, None):
        ref, mag = torch.zeros(T, d, dtype=torch.float64), torch.zeros(T, d, dtype=torch.float64)
        v = y[:len(src)].double() * (1.0 if weights is None else w.view(-1)[src].double()[:, None])
        ref.index_add_(0, src // k, v)
        mag.index_add_(0, src // k, v.abs())
        if weights is None:
            got = exf.moe_dispatch_backward(y.to(DEV), position.to(DEV), k)
        else:
            got = exf.moe_combine(y.to(DEV), position.to(DEV), w.to(DEV))
        if k > 2 or weights is None:
            R.assert_close(got.cpu(), ref, mag, k + 1, "combine")


@pytest.mark.parametrize("T,d,k", SIZES)
@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("kept", [1.0, 0.3, 0.0])
def test_gradients(T, d, k, dt, kept):
    d = _d(d, dt)
    print(f"[case] combine_backward T={T} d={d} k={k} {dt} kept={kept}", flush=True)
    position, src, y, dout, w = _case(T, d, k, dt, kept, T + d + 1)
    n = len(src)
    y[n:] = float("nan")
    wild = w.clone().view(-1)
    wild[position == -1] = float("nan")  # weights of assignments that are not kept do not count
    wild = wild.view(T, k).to(DEV)
    out = torch.full((T * k, d), 3.0, dtype=dt, device=DEV)
    dy, dw = exf.moe_combine_backward(dout.to(DEV), y.to(DEV), position.to(DEV), wild, out=out)
    assert dy is out and (dy[n:] == 3.0).all()
    rows = dout[src // k].double()
    R.assert_close(dy[:n].cpu(), rows * w.view(-1)[src].double()[:, None], (rows * w.view(-1)[src].double()[:, None]).abs(), 1, "rows")
    ref, mag = torch.zeros(T * k, dtype=torch.float64), torch.zeros(T * k, dtype=torch.float64)
    ref[src], mag[src] = (rows * y[:n].double()).sum(1), (rows * y[:n].double()).abs().sum(1)
    # a lane adds its pieces one after the other, lanes in six steps; four times that at most
    units = d // 64 + 8 + 8 + 6
    R.assert_close(dw.cpu(), ref.view(T, k), mag.view(T, k), 4 * units, "weights")
    assert (dw.view(-1)[(position == -1).to(DEV)] == 0).all()
    only, none = exf.moe_combine_backward(dout.to(DEV), y.to(DEV), position.to(DEV), w.to(DEV), want_weights=False)
    assert none is None and torch.equal(only[:n], dy[:n]) and not only[n:].any()
    none, only = exf.moe_combine_backward(dout.to(DEV), y.to(DEV), position.to(DEV), w.to(DEV), want_rows=False)
    assert none is None and torch.equal(only, dw)


@pytest.mark.parametrize("T,d,k,E_local,E,gather", [(1, 64, 8, 64, 64, True), (50, 64, 16, 16, 512, True), (700, 1032, 8, 64, 64, True), (5000, 64, 10, 64, 64, True), (3000, 8, 5, 7, 30, False),
                                                    (40000, 8, 16, 64, 64, False), (20000, 8, 16, 33, 64, True), (900, 2056, 5, 16, 300, True), (1400, 512, 3, 64, 64, True),
                                                    (4099, 520, 16, 64, 64, True), (0, 64, 8, 8, 8, True)])
def test_dispatch(T, d, k, E_local, E, gather):
    print(f"[case] dispatch T={T} d={d} k={k} E_local={E_local} E={E} gather={gather}", flush=True)
    g = torch.Generator().manual_seed(T + k)
    idx = torch.randint(-1, E + 1, (T, k), generator=g)  # (also what is no expert)
    emap = torch.randperm(E, generator=g)
    x = torch.randn(T, d, generator=g).to(BF)
    local = torch.where((idx >= 0) & (idx < E), emap[idx.clamp(0, E - 1)], E_local).view(-1).clamp(max=E_local)
    order = torch.argsort(local, stable=True)
    n = int((local < E_local).sum())
    counts = torch.bincount(local, minlength=E_local + 1)[:E_local]
    A = T * k
    out = DispatchResult(torch.full((A, d), 3.0, dtype=BF, device=DEV) if gather else None, *(torch.full((m,), -7, dtype=torch.int32, device=DEV) for m in (A, A, E_local, E_local + 1)))
    got = exf.moe_dispatch(x.to(DEV), idx.int().to(DEV), E, E_local=E_local, expert_map=emap.int().to(DEV), out=out, gather=gather)
    want = torch.full((A,), -1, dtype=torch.int64)
    want[order[:n]] = torch.arange(n)
    assert torch.equal(got.sorted_of_src.cpu().long(), want) and torch.equal(got.src_of_sorted[:n].cpu().long(), order[:n]) and (got.src_of_sorted[n:] == -7).all()
    assert torch.equal(got.expert_counts.cpu().long(), counts) and torch.equal(got.expert_offsets.cpu().long(), torch.cat((torch.zeros(1, dtype=torch.int64), counts.cumsum(0))))
    if gather:
        assert torch.equal(got.x_sorted[:n].cpu(), x[order[:n] // k]) and (got.x_sorted[n:] == 3.0).all()


def test_positions_that_are_none():
    """What moe_dispatch never writes is not followed."""
    T, k, d = 20, 4, 64
    position, _, y, dout, w = _case(T, d, k, F32, 1.0, 3)
    bad = position.clone()
    bad[::7] = torch.tensor([T * k, 1 << 30, -5, -(1 << 31)], dtype=torch.int32).repeat(3)
    dropped = torch.where((bad < 0) | (bad >= T * k), -1, position).int()
    args = (y.to(DEV), w.to(DEV), dout.to(DEV))
    assert torch.equal(exf.moe_combine(args[0], bad.to(DEV), args[1]), exf.moe_combine(args[0], dropped.to(DEV), args[1]))
    for a, b in zip(exf.moe_combine_backward(args[2], args[0], bad.to(DEV), args[1]), exf.moe_combine_backward(args[2], args[0], dropped.to(DEV), args[1])):
        assert torch.equal(a, b)


def test_rows_past_32_bits_of_bytes():
    """5.4 GB of sorted rows."""
    T, k, d = 82000, 16, 2048
    position = torch.arange(T * k, dtype=torch.int32, device=DEV).flip(0)
    y = torch.empty((T * k, d), dtype=BF, device=DEV).normal_(generator=torch.Generator(DEV).manual_seed(2))
    w = torch.rand((T, k), device=DEV, generator=torch.Generator(DEV).manual_seed(3))
    out = exf.moe_combine(y, position, w)
    for t in (0, T - 1, T // 2):
        rows = y[position[t * k:(t + 1) * k].long()].double() * w[t].double()[:, None]
        R.assert_close(out[t:t + 1].cpu(), rows.sum(0, keepdim=True).cpu(), rows.abs().sum(0, keepdim=True).cpu(), k + 1)
    dy, dw = exf.moe_combine_backward(out, y, position, w)
    for t in (0, T - 1, T // 2):
        at = position[t * k:(t + 1) * k].long()
        want = out[t].double() * w[t].double()[:, None]
        R.assert_close(dy[at].cpu(), want.cpu(), want.abs().cpu(), 1)
        want = y[at].double() * out[t].double()
        R.assert_close(dw[t].cpu(), want.sum(1).cpu(), want.abs().sum(1).cpu(), 4 * (d // 64 + 22))


def test_no_tokens():
    y, position, w = torch.empty((0, 64), dtype=BF, device=DEV), torch.empty(0, dtype=torch.int32, device=DEV), torch.empty((0, 5), device=DEV)
    assert exf.moe_combine(y, position, w).shape == (0, 64) and exf.moe_dispatch_backward(y, position, 5).shape == (0, 64)
    dy, dw = exf.moe_combine_backward(y, y, position, w)
    assert dy.shape == (0, 64) and dw.shape == (0, 5)
