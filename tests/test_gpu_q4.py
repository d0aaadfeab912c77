"""4-bit integers with group scales: rows to them and back, and the experts' products with them, against their definitions in 64 bits."""
import pytest
import torch

import many_experts_reference as R
import paper_2401_08383_amd as exf
from product_reference import ranges, sizes_to_offsets

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
BF, F32, INF = torch.bfloat16, torch.float32, float("inf")


def _rows(shape, dt, seed):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * torch.exp2(torch.randint(-8, 8, (*shape[:-1], 1), generator=g))).to(dt)


def _codes(q):
    return torch.stack((q % 16, q // 16), -1).flatten(-2)


def _check_quantise(x, group, symmetric):
    print(f"[case] q4_quantize {tuple(x.shape)} {x.dtype} group={group} symmetric={symmetric}", flush=True)
    code, scale, zero = R.q4_quantised(x, group, symmetric)
    m = exf.q4_quantize(x.to(DEV), group, symmetric=symmetric)
    assert m.shape == x.shape and m.group == group and (m.zero is None) == symmetric
    assert torch.equal(m.scale.cpu().float().nan_to_num(-1.0), scale.float().nan_to_num(-1.0))
    if not symmetric:
        assert torch.equal(m.zero.cpu(), zero)
    assert torch.equal(_codes(m.q.cpu()), code), torch.nonzero(_codes(m.q.cpu()) != code)[:4]
    back = exf.q4_dequantize(m)
    want = R.q4_values(m.q.cpu(), m.scale.cpu(), None if zero is None else zero)
    # one rounding to fp32, one to the type, which make an infinity of what lies past its range (-8 steps of 2 max / 15 are 1.07 max)
    rounded = want.float().to(x.dtype)
    past = ~torch.isfinite(rounded)
    assert torch.equal(back.cpu()[past].float().nan_to_num(123.0), rounded[past].float().nan_to_num(123.0))
    R.assert_close(back.cpu()[~past], want[~past], want[~past].abs(), 1)
    return m


@pytest.mark.parametrize("shape", [(1, 128), (3, 384), (2, 5, 256), (77, 1024), (1000, 128), (1, 16384)])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("symmetric", [False, True])
def test_quantise(shape, group, dt, symmetric):
    _check_quantise(_rows(shape, dt, shape[-1]), group, symmetric)


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("symmetric", [False, True])
def test_quantise_what_lies_between_two_codes(dt, symmetric):
    """Quotients that are, and nearly are, halfway between two integers; zeros; one sign; the ends of the type's range; infinities and NaN."""
    g = torch.Generator().manual_seed(1)
    x = torch.randint(-15, 15, (64, 64), generator=g).float() / 2  # halves of a scale of 1, if the ends are there
    x[:, 0], x[:, 1] = (-7.0, 7.0) if symmetric else (-7.0, 8.0)
    x = torch.cat((x, x * 3.0, x * 0.7109375, x * 2.0 ** -120, x * 2.0 ** 120, x.abs(), -x.abs()))
    edge = torch.stack((torch.zeros(64), torch.full((64,), 2.0 ** -133), torch.full((64,), -(2.0 ** -130)), torch.full((64,), 3.0), torch.full((64,), -0.0),
                        torch.where(torch.arange(64) % 2 == 0, torch.finfo(dt).max, torch.finfo(dt).min), torch.where(torch.arange(64) == 40, float("nan"), 1.0),
                        torch.where(torch.arange(64) == 9, INF, 1.0), torch.where(torch.arange(64) == 63, -INF, 1.0), torch.where(torch.arange(64) == 5, 1.0, 2.0 ** -126)))
    x = torch.cat((x, edge)).to(dt)
    if dt == F32:  # a last place to either side of the middle
        bits = x.view(torch.int32)
        x = torch.cat((x, (bits[:448] + torch.randint(-1, 2, (448, 64), generator=g, dtype=torch.int32)).view(F32)))
        x[448 + 10:] = x[448 + 10:].nan_to_num(1.0, 1.0, 1.0)
    for group in (32, 64):
        _check_quantise(x, group, symmetric)


def test_no_rows():
    m = exf.q4_quantize(torch.empty((0, 128), dtype=BF, device=DEV))
    assert m.shape == (0, 128) and exf.q4_dequantize(m).shape == (0, 128)


def _weights(E, n, k, group, dt, zeros, seed):
    g = torch.Generator().manual_seed(seed)
    q = torch.randint(0, 256, (E, n, k // 2), generator=g, dtype=torch.int32).to(torch.uint8)
    scale = (0.01 + 0.05 * torch.rand((E, n, k // group), generator=g)).to(dt)
    scale = scale * torch.where(torch.rand(scale.shape, generator=g) < 0.1, -1, 1).to(dt)  # (a scale may have any sign)
    zero = torch.randint(0, 17, (E, n, k // group), generator=g, dtype=torch.int32).to(torch.uint8) if zeros else None
    return q, scale, zero


def _check_product(sizes, n, k, group, dt, zeros=True, bias=False, first=0, behind=0, seed=0):
    A, E = first + sum(sizes) + behind, len(sizes)
    print(f"[case] q4 product {sizes if E < 10 else E} n={n} k={k} group={group} {dt} zeros={zeros} bias={bias} first={first} behind={behind}", flush=True)
    g = torch.Generator().manual_seed(seed + 1)
    q, scale, zero = _weights(E, n, k, group, dt, zeros, seed)
    x, off = torch.randn(A, k, generator=g).to(dt), sizes_to_offsets(sizes, first)
    b = torch.randn(E, n, generator=g).to(dt) if bias else None
    out = torch.full((A, n), 3.0, dtype=dt, device=DEV)
    to = lambda t: None if t is None else t.to(DEV)  # noqa: E731
    m = exf.Q4(to(q), to(scale), to(zero))
    y = exf.moe_grouped_product_q4(to(x), to(off), m, to(b), out=out)
    assert y is out
    inside = torch.zeros(A, dtype=torch.bool)
    for e, (lo, hi) in enumerate(ranges(off, A)):
        if lo == hi:
            continue
        inside[lo:hi] = True
        w, rows = R.q4_values(q[e], scale[e], None if zero is None else zero[e]), x[lo:hi].double()
        ref = rows @ w.t()
        # the terms that are summed: codes and zero points as they stand (bf16: both with sixteen), by the scale's magnitude
        most = scale[e].double().abs().repeat_interleave(group, 1) * (16 + 15 + 16 + 17)
        mag = rows.abs() @ most.t()
        if b is not None:
            ref, mag = ref + b[e].double(), mag + b[e].double().abs()
        # at most k sums and as many roundings of products, each by at most two units where the hardware chops; the scales' products and sums of groups, a bias
        R.assert_close(y[lo:hi].cpu(), ref, mag, 4 * (min(k, 1024) / 16 + k / group + 8), f"expert {e}")
    assert (y[(~inside).to(DEV)] == 3.0).all()
    again = exf.moe_grouped_product_q4(to(x), to(off), m, to(b))
    assert torch.equal(again[inside.to(DEV)], y[inside.to(DEV)])


@pytest.mark.parametrize("sizes,n,k", [([1], 8, 128), ([1], 4096, 1024), ([0, 1, 0], 64, 256), ([5, 0, 16, 17, 1], 72, 640), ([16], 16, 128), ([33, 64, 100], 200, 384), ([3] * 64, 40, 256), ([700], 136, 512),
                                       ([2, 2], 24, 16384), ([0, 0], 8, 128)])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("dt", [BF, F32])
def test_product(sizes, n, k, group, dt):
    _check_product(sizes, n, k, group, dt, zeros=True, bias=False)
    _check_product(sizes, n, k, group, dt, zeros=False, bias=True, seed=5)


@pytest.mark.parametrize("k,group", [(32, 32), (64, 32), (96, 32), (160, 32), (64, 64), (192, 64), (1120, 32), (1216, 64)])
@pytest.mark.parametrize("dt", [BF, F32])
def test_product_of_steps_that_are_not_full(k, group, dt):
    _check_product([3, 20, 0, 1], 44 if dt == F32 else 48, k, group, dt, bias=True)


# (rows of the experts, n, k): many rows an expert; few columns for the chip, and still fewer with a long reduction; enough.  Of each, reductions that end with a line
# of a column, inside one with whole and with odd numbers of groups, and inside the first.
SPREADS = {"two tiles": ([64, 50, 0, 100, 64, 17, 130, 64], 4096, (128, 384, 32, 96, 160, 192, 256, 512, 288, 320)), "tall": ([64, 50, 0, 100, 64, 17, 130, 64], 12288, (128, 384, 32, 96, 160, 192)), "few": ([1, 0, 3, 1, 2, 1, 16, 1], 4104, (512, 384, 32, 288, 352, 320)),
           "tallest": ([64, 70, 1, 130, 0, 64, 100, 64], 16392, (128, 384, 32, 96, 160, 192)), "fewest": ([3, 2], 8192, (2048, 2176, 2080, 2112, 2272)), "wide": ([1, 4, 1, 0, 17, 1, 9, 1, 1, 1, 1, 1, 3], 4160, (256, 640, 64, 96, 288, 192))}


@pytest.mark.parametrize("spread,k,group", [(name, k, group) for name, (_, _, ks) in SPREADS.items() for k in ks for group in (32, 64, 128) if k % group == 0])
def test_product_of_many_columns(spread, k, group):
    sizes, n, _ = SPREADS[spread]
    _check_product(sizes, n, k, group, BF, zeros=True, bias=k % 3 == 0, first=2, behind=3)
    _check_product(sizes, n, k, group, BF, zeros=False, bias=k % 3 != 0, seed=7)


@pytest.mark.parametrize("k,group", [(k, group) for k in (512, 544, 576, 640) for group in (32, 64, 128) if k % group == 0])
@pytest.mark.parametrize("some", [(1, 2, 1, 2), (33, 1, 17, 25)])
def test_product_of_weights_that_no_cache_holds(k, group, some):
    """Rows of four of 64 experts, the last among them."""
    E, n, g = 64, 17000, torch.Generator(DEV).manual_seed(k + group)
    q = torch.empty((E, n, k // 2), dtype=torch.uint8, device=DEV).random_(generator=g)
    scale = torch.empty((E, n, k // group), dtype=BF, device=DEV).uniform_(0.01, 0.05, generator=g)
    zero = torch.empty((E, n, k // group), dtype=torch.uint8, device=DEV).random_(0, 17, generator=g)
    x = torch.randn((sum(some) if sum(some) < 64 else 1100, k), generator=torch.Generator().manual_seed(3)).to(BF).to(DEV)  # (rows behind the last expert's count as rows)
    sizes = [0] * E
    sizes[0], sizes[5], sizes[40], sizes[63] = some
    off = sizes_to_offsets(sizes)
    for z in (zero, None):
        y = exf.moe_grouped_product_q4(x, off.to(DEV), exf.Q4(q, scale, z))
        for e in (0, 5, 40, 63):
            lo, hi = int(off[e]), int(off[e + 1])
            rows = x[lo:hi].double()
            ref = rows @ R.q4_values(q[e], scale[e], None if z is None else z[e]).t()
            mag = rows.abs() @ (scale[e].double().repeat_interleave(group, 1) * (16 + 15 + 16 + 17)).t()
            R.assert_close(y[lo:hi].cpu(), ref.cpu(), mag.cpu(), 4 * (k / 16 + k / group + 8), f"expert {e}")


@pytest.mark.parametrize("spread,k", [("tall", 160), ("two tiles", 288), ("tallest", 96), ("few", 352), ("fewest", 2080), ("wide", 288), ("few", 512), ("tall", 128), ("two tiles", 512), ("tallest", 128)])
def test_what_is_no_number_stays_in_its_row_and_column(spread, k):
    """... also where a step reads past the end of one into the next."""
    sizes, n, _ = SPREADS[spread]
    q, scale, zero = _weights(len(sizes), n, k, 32, BF, True, 3)
    A, off = sum(sizes), sizes_to_offsets(sizes).to(DEV)
    x = torch.randn(A, k, generator=torch.Generator().manual_seed(1)).to(BF)
    rows = [1, A - 1]
    x_bad, scale_bad = x.clone(), scale.clone()
    x_bad[rows[0], :] = float("nan")
    x_bad[rows[1], 0] = INF
    bad = [e for e in range(len(sizes)) if sizes[e]][-1]
    scale_bad[bad, 9, 0], scale_bad[bad, 70, -1] = float("nan"), INF
    to = lambda t: t.to(DEV)  # noqa: E731
    want = exf.moe_grouped_product_q4(to(x), off, exf.Q4(to(q), to(scale), to(zero)))
    got = exf.moe_grouped_product_q4(to(x_bad), off, exf.Q4(to(q), to(scale_bad), to(zero)))
    same = torch.ones((A, n), dtype=torch.bool, device=DEV)
    same[rows] = False
    lo, hi = int(off[bad]), int(off[bad + 1])
    same[lo:hi, 9] = same[lo:hi, 70] = False
    assert torch.equal(got[same], want[same]) and not torch.isfinite(got[rows]).any() and not torch.isfinite(got[lo:hi, [9, 70]]).any()


@pytest.mark.parametrize("dt", [BF, F32])
def test_rows_outside_all_ranges_are_left_alone(dt):
    _check_product([4, 0, 30], 64, 256, 128, dt, first=3, behind=9)


def test_rows_that_are_not_a_numbers_stay_by_themselves():
    """An infinity or a NaN in one row, and a group whose scale is NaN."""
    q, scale, zero = _weights(1, 64, 512, 128, BF, True, 3)
    scale[0, 7, 2] = float("nan")
    x = torch.randn(20, 512, generator=torch.Generator().manual_seed(1)).to(BF)
    clean = x.clone()
    x[3, 100], x[9, 511] = float("nan"), INF
    off = torch.tensor([0, 20], dtype=torch.int32, device=DEV)
    m = exf.Q4(q.to(DEV), scale.to(DEV), zero.to(DEV))
    got, want = exf.moe_grouped_product_q4(x.to(DEV), off, m), exf.moe_grouped_product_q4(clean.to(DEV), off, m)
    rows = [r for r in range(20) if r not in (3, 9)]
    assert torch.equal(got[rows].nan_to_num(9.0), want[rows].nan_to_num(9.0)) and torch.isnan(got[3]).all() and not torch.isfinite(got[9]).any()
    assert torch.isnan(want[:, 7]).all() and torch.isfinite(want[:, :7]).all() and torch.isfinite(want[:, 8:]).all()


def test_quantised_and_multiplied():
    """The product of what q4_quantize holds is that of the values q4_dequantize gives back."""
    g = torch.Generator(DEV).manual_seed(4)
    w = torch.empty((4, 256, 512), dtype=BF, device=DEV).normal_(0, 0.05, generator=g)
    x = torch.empty((50, 512), dtype=BF, device=DEV).normal_(generator=g)
    off = torch.tensor([0, 10, 10, 49, 50], dtype=torch.int32, device=DEV)
    for group in (32, 128):
        m = exf.q4_quantize(w, group)
        y, full = exf.moe_grouped_product_q4(x, off, m).double(), exf.moe_grouped_product(x, off, exf.q4_dequantize(m)).double()
        assert float((y - full).norm() / full.norm()) < 2.0 ** -7  # (the values are rounded to bf16 on the way back)
        few = exf.Q4(m.q[2:3], m.scale[2:3], m.zero[2:3])
        assert torch.equal(exf.moe_grouped_product_q4(x[10:49], torch.tensor([0, 39], dtype=torch.int32, device=DEV), few).double(), y[10:49])


@pytest.mark.parametrize("symmetric", [False, True])
def test_rows_past_32_bits_of_elements(symmetric):
    """The last rows of 2.2 G values are held and given back as they are by themselves."""
    x = torch.empty((270000, 8192), dtype=BF, device=DEV).normal_(generator=torch.Generator(DEV).manual_seed(1))
    m = exf.q4_quantize(x, 128, symmetric=symmetric)
    end = slice(270000 - 40, 270000)
    few = exf.q4_quantize(x[end], 128, symmetric=symmetric)
    assert torch.equal(m.q[end], few.q) and torch.equal(m.scale[end], few.scale) and (symmetric or torch.equal(m.zero[end], few.zero))
    assert torch.equal(exf.q4_dequantize(m, out=x)[end], exf.q4_dequantize(few))


def test_weights_past_32_bits_of_bytes():
    """4.6 GB of codes: the last expert's product is that of the expert by itself."""
    E, n, k = 3, 1 << 17, 24576
    q = torch.empty((E, n, k // 2), dtype=torch.uint8, device=DEV).random_(generator=torch.Generator(DEV).manual_seed(1))
    scale = torch.empty((E, n, k // 128), dtype=BF, device=DEV).uniform_(0.01, 0.02, generator=torch.Generator(DEV).manual_seed(2))
    x = torch.randn((3, k), generator=torch.Generator().manual_seed(3)).to(BF).to(DEV)
    y = exf.moe_grouped_product_q4(x, torch.tensor([0, 1, 1, 3], dtype=torch.int32, device=DEV), exf.Q4(q, scale))
    part = slice(n - 64, n)
    w = R.q4_values(q[2, part], scale[2, part], None)
    ref, mag = x[1:].double() @ w.t(), x[1:].double().abs() @ (w.abs() + 63 * 0.02).t()
    R.assert_close(y[1:, part].cpu(), ref.cpu(), mag.cpu(), 4 * (64 + k / 128 + 8))
