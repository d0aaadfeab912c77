"""moe_combine of one and two assignments a token where the last tokens and the rows' pieces do not come out even."""
import pytest
import torch

import paper_2401_08383_amd as exf

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("T,d", [(8195, 688), (8195, 1368), (16391, 296), (16389, 1640), (32771, 1368), (32775, 296), (32783, 144), (40007, 1464), (4097, 688), (2047, 8), (8195, 8), (32770, 4104)])
@pytest.mark.parametrize("k", [1, 2])
@pytest.mark.parametrize("dt", [BF, F32])
def test_every_element_of_the_last_tokens(T, d, k, dt):
    """Wholes up to 8 times quarters up to 1, of two assignments at most: all sums are exact in 16 bits."""
    d = d if dt == BF else d // 2
    print(f"[case] combine T={T} d={d} k={k} {dt}", flush=True)
    g = torch.Generator(DEV).manual_seed(T + d + k)
    y = torch.randint(-8, 9, (T * k, d), device=DEV, generator=g).to(dt)
    w = torch.randint(1, 5, (T, k), device=DEV, generator=g).float() / 4
    position = torch.randperm(T * k, device=DEV, generator=g).int()
    position[torch.randint(0, T * k, (T // 8,), device=DEV, generator=g)] = -1
    position[-k:] = T * k - 1
    want = torch.zeros(T, d, device=DEV)
    for j in range(k):
        at = position.view(T, k)[:, j].long()
        want += torch.where((at >= 0)[:, None], w[:, j, None] * y[at.clamp(min=0)].float(), 0.0)
    out = torch.full((T, d), 77.0, dtype=dt, device=DEV)
    got = exf.moe_combine(y, position, w, out=out)
    assert got is out
    wrong = torch.nonzero(got.float() != want)
    assert not len(wrong), (len(wrong), wrong[:3].tolist(), wrong[-1].tolist())
