"""Products with 4-bit weights of rows up to 2^113: a group's sums are formed in front of its scale and do not overflow."""
import pytest
import torch

import many_experts_reference as R
import paper_2401_08383_amd as exf

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
BF, F32, U8 = torch.bfloat16, torch.float32, torch.uint8


@pytest.mark.parametrize("rows,n,k", [(1, 64, 1024), (20, 72, 640), (3, 8192, 2048), (40, 8192, 256), (300, 8192, 256), (5, 20000, 384)])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("dt", [BF, F32])
def test_rows_of_the_largest_magnitude(rows, n, k, group, dt):
    """All elements of a row of one sign and +-2^113 or half of it, codes 0 or 15, zero points to 255, scales small enough for the result."""
    if dt == F32 and n > 8192:
        n = 8192
    print(f"[case] large rows {rows} x {n} x {k} group={group} {dt}", flush=True)
    g = torch.Generator(DEV).manual_seed(n + k + group)
    sign = torch.randint(0, 2, (rows, 1), device=DEV, generator=g).float() * 2 - 1
    x = (sign * 2.0 ** 113 / (1 + torch.randint(0, 2, (rows, k), device=DEV, generator=g).float())).to(dt)
    code = torch.randint(0, 2, (1, n, k // group, 1), device=DEV, generator=g).expand(1, n, k // group, group).reshape(1, n, k) * 15  # a group's all 0, or all 15
    q = (code[..., 0::2] + 16 * code[..., 1::2]).to(U8)
    zero = torch.tensor([0, 8, 15, 255], dtype=U8, device=DEV)[torch.randint(0, 4, (1, n, k // group), device=DEV, generator=g)]
    scale = torch.full((1, n, k // group), 2.0 ** -24, dtype=dt, device=DEV)
    off = torch.tensor([0, rows], dtype=torch.int32, device=DEV)
    for z in (zero, None):
        y = exf.moe_grouped_product_q4(x, off, exf.Q4(q, scale, z))
        ref = x.double() @ R.q4_values(q[0], scale[0], None if z is None else z[0]).t()
        at = 8.0 if z is None else z[0].double().repeat_interleave(group, 1)
        mag = x.double().abs() @ ((16 + code[0].double() + 16 + at) * 2.0 ** -24).t()
        # at most k sums and as many roundings of products, each by at most two units where the hardware chops; the scales' products and sums of groups
        R.assert_close(y, ref, mag, 4 * (min(k, 1024) / 16 + k / group + 8), "large rows")
