"""Infinite and undefined operands of the contractions: a result is infinite or undefined where the definition says so, with the sign that it says,
and finite everywhere else, whatever the reduction's length leaves over of a step.  References are computed on the CPU."""
import pytest
import torch

import paper_2401_08383_amd as exf
import product_reference as R
from helpers import DEV

pytestmark = pytest.mark.gpu

TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
INF, NAN = float("inf"), float("nan")


def _normal(shape, std, dt, seed):
    g = torch.Generator()
    g.manual_seed(seed)
    return torch.empty(shape, dtype=torch.float32).normal_(0.0, std, generator=g).to(dt)


def _same(got, ref, mag, terms, what):
    got = got.cpu()
    g, finite = got.double(), torch.isfinite(ref)
    assert torch.equal(torch.isnan(g), torch.isnan(ref)), f"{what}: {int(torch.isnan(g).sum())} NaN, expected {int(torch.isnan(ref).sum())}"
    assert torch.equal(g[torch.isinf(ref)], ref[torch.isinf(ref)]), f"{what}: infinities"
    zero = torch.zeros((), dtype=torch.float64)
    R.assert_sums_close(torch.where(finite, got, torch.zeros((), dtype=got.dtype)), torch.where(finite, ref, zero), torch.where(finite, mag, zero), terms, what)


# Rows an expert on both sides of what chooses the kernel; reductions that end 4, 12, 20 or 28 elements into a step of 32; few tiles and many, one wavefront
# a tile and several.
PRODUCTS = [([5, 0, 9], 40, 36), ([40, 3], 72, 100), ([90, 30], 136, 44), ([12] * 8, 64, 1156), ([20, 3] * 8, 260, 1036), ([10] * 30, 516, 92), ([500, 9], 264, 140),
            ([100, 41], 64, 2068), ([20, 2] * 20, 1028, 60), ([18, 0, 23], 1040, 2052), ([20] * 30, 1040, 300), ([20] * 30, 1040, 1036)]


def _operands(sizes, n, k, dt, seed):
    """x, W, offsets: both ends of the reduction hold infinities of either sign in some rows of x and in some weights; one NaN in each."""
    A, E = sum(sizes), len(sizes)
    x, w = _normal((A, k), 1.0, dt, seed), _normal((E, n, k), 0.1, dt, seed + 1)
    w[0, 1, 0], w[0, 2, 3], w[0, 5, k - 1], w[E - 1, 7, 1], w[E - 1, n - 1, k - 2] = INF, -INF, INF, -INF, INF
    w[E - 1, 3, k // 2] = NAN
    x[1, k - 1], x[2, 2], x[A - 1, k // 2] = INF, -INF, NAN
    return x, w, R.sizes_to_offsets(sizes)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("sizes,n,k", PRODUCTS)
def test_products(dtype, sizes, n, k):
    if dtype == "bf16":
        n, k = (n + 7) // 8 * 8, (k + 7) // 8 * 8
    print(f"[case] product {dtype} sizes={sizes} n={n} k={k}", flush=True)
    x, w, off = _operands(sizes, n, k, TYPES[dtype], 3)
    _same(exf.moe_grouped_product(x.to(DEV), off.to(DEV), w.to(DEV)), *R.rows_product(x, off, w), "y")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("sizes,k,n", PRODUCTS)
def test_rows_gradients(dtype, sizes, k, n):
    if dtype == "bf16":
        n, k = (n + 7) // 8 * 8, (k + 7) // 8 * 8
    print(f"[case] dx {dtype} sizes={sizes} n={n} k={k}", flush=True)
    dy, w, off = _operands(sizes, k, n, TYPES[dtype], 5)
    w = w.transpose(1, 2).contiguous()
    _same(exf.moe_grouped_product_dx(dy.to(DEV), off.to(DEV), w.to(DEV)), *R.rows_product(dy, off, w, None, True), "dx")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("sizes,n,k", [([5, 0, 9], 40, 48), ([33, 1, 70], 136, 72), ([700], 64, 64), ([257, 300], 520, 264)])
def test_weight_gradients(dtype, sizes, n, k):
    print(f"[case] dw {dtype} sizes={sizes} n={n} k={k}", flush=True)
    A, off = sum(sizes), R.sizes_to_offsets(sizes)
    dy, x = _normal((A, n), 1.0, TYPES[dtype], 7), _normal((A, k), 1.0, TYPES[dtype], 8)
    dy[0, 3], dy[sizes[0] - 1, 5], x[A - 1, 2], x[min(sizes[0], A - 1), k - 1], dy[A - 2, n - 1] = INF, -INF, INF, -INF, NAN
    dw, db = exf.moe_grouped_product_dw(dy.to(DEV), x.to(DEV), off.to(DEV), want_bias=True)
    ref, mag, ref_b, mag_b, terms = R.weight_gradient(dy, x, off)
    _same(dw, ref, mag, terms, "dw")
    _same(db, ref_b, mag_b, terms, "db")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("sizes,n,k", [([5, 0, 9], 40, 96), ([40, 3], 72, 288), ([600, 41], 520, 1056), ([12] * 8, 2048, 4128)])
def test_blocks_of_4_bits(dtype, sizes, n, k):
    """A block that holds an infinity or a NaN stands for NaN."""
    print(f"[case] mx4 {dtype} sizes={sizes} n={n} k={k}", flush=True)
    x, w, off = _operands(sizes, n, k, TYPES[dtype], 9)
    held = exf.mx4_quantize(w.to(DEV))
    got = exf.moe_grouped_product_mx4(x.to(DEV), off.to(DEV), held)
    _same(got, *R.rows_product(R.quantised(x)[0], off, R.quantised(w)[0]), "y")


# both contractions in a launch each, of tiles of 16 x 16, 16 x 32, 64 x 64, long reductions, and both in one launch (from 1025 rows on)
@pytest.mark.parametrize("sizes,d,f", [([5, 0, 9], 36, 100), ([60, 30], 132, 396), ([12] * 8, 1036, 1156), ([400] * 9 + [124], 120, 444), ([1500, 13, 1504], 92, 188),
                                       ([300, 0, 700, 200], 516, 1044), ([1600, 0, 700, 500], 516, 1044)])
def test_expert_ffn_in_fp32(sizes, d, f):
    print(f"[case] ffn sizes={sizes} d={d} f={f}", flush=True)
    E, A, dt = len(sizes), sum(sizes), torch.float32
    x, w1, w2 = _normal((A, d), 1.0, dt, 11), _normal((E, f, d), 0.1, dt, 12), _normal((E, d, f), 0.1, dt, 13)
    x[:, 0], x[:, d - 1] = x[:, 0].abs() + 0.5, x[:, d - 1].abs() + 0.5
    w1[E - 1, [0, f - 1]] *= 0.2  # (their GELU is no zero, which would make a NaN of an infinity)
    w1[0, 1, 0], w1[0, 6, d - 1] = INF, INF     # hidden 1 and 6 of the first expert are +inf, so are its outputs, by w2's signs
    w2[0, :, 6] = w2[0, :, 6].abs() * w2[0, :, 1].sign()
    w2[E - 1, 2, 0], w2[E - 1, 4, f - 1] = -INF, INF  # outputs 2 and 4 of the last one
    off = R.sizes_to_offsets(sizes)
    got = exf.moe_expert_ffn(x.to(DEV), off.to(DEV), w1.to(DEV), w2.to(DEV)).cpu().double()
    lo = off.tolist()
    for e in (0, E - 1):
        h = torch.nn.functional.gelu(x[lo[e]:lo[e + 1]].double() @ w1[e].double().t())
        ref = h @ w2[e].double().t()
        part = got[lo[e]:lo[e + 1]]
        assert torch.isinf(ref).any() and not torch.isnan(ref).any()
        assert torch.equal(torch.isinf(part), torch.isinf(ref)) and torch.equal(part[torch.isinf(ref)], ref[torch.isinf(ref)]), f"expert {e}"
        finite = torch.isfinite(ref)
        assert torch.isfinite(part[finite]).all()
