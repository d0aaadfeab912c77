"""One and two assignments a token through the calls that take up to sixteen: the package sends these to moe_dispatch and moe_combine, a C program may not."""
import pytest
import torch

import many_experts_reference as R
import paper_2401_08383_amd as exf
from paper_2401_08383_amd import binding as B

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32


def _stream():
    return torch.cuda.current_stream().cuda_stream


@pytest.mark.parametrize("T,d", [(1, 8), (1, 2048), (17, 520), (64, 64), (333, 1032), (2047, 24), (4099, 1368), (8195, 688), (32775, 296), (9001, 72)])
@pytest.mark.parametrize("k", [1, 2])
@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("kept", [1.0, 0.3])
def test_weighted_rows(T, d, k, dt, kept):
    d = d if dt == BF else d // 2
    print(f"[case] combine_topk T={T} d={d} k={k} {dt} kept={kept}", flush=True)
    g = torch.Generator().manual_seed(T + d + k)
    position, src = R.assignments(T, k, 64, g, kept)
    y, w = torch.randn(T * k, d, generator=g).to(dt), torch.rand(T, k, generator=g)
    y[len(src):] = float("nan")  # rows behind the last kept one are not read
    ref, mag = torch.zeros(T, d, dtype=torch.float64), torch.zeros(T, d, dtype=torch.float64)
    v = y[:len(src)].double() * w.view(-1)[src].double()[:, None]
    ref.index_add_(0, src // k, v)
    mag.index_add_(0, src // k, v.abs())
    yd, pd, wd, out = y.to(DEV), position.to(DEV), w.to(DEV), torch.full((T, d), 7.0, dtype=dt, device=DEV)
    assert exf.lib().moe_combine_topk(yd.data_ptr(), pd.data_ptr(), wd.data_ptr(), T, d, k, B.dtype_code(yd), out.data_ptr(), _stream()) == B.EXF_OK
    # a product and an addition a slot
    R.assert_close(out.cpu(), ref, mag, k + 1, "moe_combine_topk")
    R.assert_close(exf.moe_combine(yd, pd, wd).cpu(), ref, mag, k + 1, "moe_combine")


@pytest.mark.parametrize("T,k", [(1, 1), (1, 2), (63, 2), (2047, 2), (2048, 2), (2049, 2), (4095, 1), (4097, 1), (20011, 1), (20011, 2), (70001, 2)])
@pytest.mark.parametrize("d,E_local,E,gather", [(72, 64, 64, True), (1032, 5, 70, True), (8, 64, 300, True), (64, 9, 9, False)])
def test_sorted_rows(T, k, d, E_local, E, gather):
    print(f"[case] dispatch_topk T={T} k={k} d={d} E_local={E_local} E={E} gather={gather}", flush=True)
    g = torch.Generator().manual_seed(T + k + d)
    idx = torch.randint(-1, E + 1, (T, k), generator=g)  # (also what is no expert)
    emap = torch.randperm(E, generator=g)
    x = torch.randn(T, d, generator=g).to(BF)
    local = torch.where((idx >= 0) & (idx < E), emap[idx.clamp(0, E - 1)], E_local).view(-1).clamp(max=E_local)
    order, n, A = torch.argsort(local, stable=True), int((local < E_local).sum()), T * k
    counts = torch.bincount(local, minlength=E_local + 1)[:E_local]
    want = torch.full((A,), -1, dtype=torch.int64)
    want[order[:n]] = torch.arange(n)
    xd, idx_d, map_d = x.to(DEV), idx.int().to(DEV), emap.int().to(DEV)
    size = exf.lib().moe_dispatch_workspace_bytes(T, k, E_local)
    for name in ("moe_dispatch_topk", "moe_dispatch"):
        rows = torch.full((A, d), 3.0, dtype=BF, device=DEV) if gather else None
        src, at, count, offsets = (torch.full((m,), -7, dtype=torch.int32, device=DEV) for m in (A, A, E_local, E_local + 1))
        workspace = torch.empty(size, dtype=torch.uint8, device=DEV)
        rc = getattr(exf.lib(), name)(xd.data_ptr(), idx_d.data_ptr(), map_d.data_ptr(), T, d, k, E, E_local, B.EXF_BF16, B._ptr(rows), src.data_ptr(), at.data_ptr(), count.data_ptr(),
                                      offsets.data_ptr(), workspace.data_ptr(), size, _stream())
        assert rc == B.EXF_OK, name
        assert torch.equal(at.cpu().long(), want) and torch.equal(src[:n].cpu().long(), order[:n]) and (src[n:] == -7).all(), name
        assert torch.equal(count.cpu().long(), counts) and torch.equal(offsets.cpu().long(), torch.cat((torch.zeros(1, dtype=torch.int64), counts.cumsum(0)))), name
        if gather:
            assert torch.equal(rows[:n].cpu(), x[order[:n] // k]) and (rows[n:] == 3.0).all(), name
