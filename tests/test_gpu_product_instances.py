"""One case at least for every kernel that the experts' products choose by size: those whose sizes lie beyond what the other tests have, against 64 bits."""
import pytest
import torch

import paper_2401_08383_amd as exf
import product_reference as R
from helpers import DEV
from test_gpu_products import _dw_case, _mx4_case, _normal, _rows_case

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32


# Weight gradients as one stream of tiles: far more 128 x 128 tiles than the 512 workgroups, so that each has several, whole ones and ragged ones in turn,
# experts of one stage, of several and of none.  At most 128 rows an expert (stages of 32 rows) and more (of 64).
SHORT = [200, 0, 5, 33, 64, 65, 1, 128, 31, 32, 96, 300, 0, 17, 100, 2, 160, 129, 63, 40]
LONG = [700, 0, 5, 33, 64, 65, 1, 128, 400, 256, 96, 300, 0, 17, 511, 513, 160, 129, 63, 140]


@pytest.mark.parametrize("grad", ["bf16", "f32"])
@pytest.mark.parametrize("bias", [True, False])
@pytest.mark.parametrize("sizes,n,k", [(SHORT, 1000, 776), (SHORT, 768, 1024), ([3] * 64, 520, 640), (LONG, 1000, 776), (LONG, 1024, 768), ([150] * 20 + [0, 1], 648, 1032)])
def test_weight_gradients_in_a_stream(sizes, n, k, bias, grad):
    assert len(sizes) * ((n + 127) // 128) * ((k + 127) // 128) > 768
    assert len(sizes) * ((n + 255) // 256) * ((k + 255) // 256) < 512 or sum(sizes) < 256 * len(sizes)
    _dw_case(sizes, n, k, "bf16", grad, bias=bias, before=3, behind=2)


def _skewed(A, E, seed):
    g = torch.Generator()
    g.manual_seed(seed)
    loads = torch.rand(E, generator=g) ** 2 + 0.02
    loads[E // 2] = 0.0
    return torch.bincount(torch.multinomial(loads, A, replacement=True, generator=g), minlength=E).tolist()


# ... of long reductions, in 256 x 256 tiles: from 512 of these and 256 rows an expert on.
@pytest.mark.parametrize("grad", ["bf16", "f32"])
@pytest.mark.parametrize("bias", [True, False])
@pytest.mark.parametrize("A,E,n,k", [(9000, 32, 1032, 1032), (2600, 8, 2048, 2048)])
def test_weight_gradients_in_large_tiles(A, E, n, k, bias, grad):
    assert E * ((n + 255) // 256) * ((k + 255) // 256) >= 512 and A >= 256 * E
    _dw_case(_skewed(A, E, n), n, k, "bf16", grad, bias=bias, before=1, behind=4)


# ... in fp32, in 64 x 64 tiles through LDS: from 512 of them on.
@pytest.mark.parametrize("bias", [True, False])
@pytest.mark.parametrize("sizes,n,k", [([40, 0, 1, 33, 100, 31, 32, 64] * 2, 520, 264), ([500, 3], 1028, 1100)])
def test_weight_gradients_in_fp32_tiles(sizes, n, k, bias):
    assert len(sizes) * ((n + 63) // 64) * ((k + 63) // 64) >= 512
    _dw_case(sizes, n, k, "f32", "f32", bias=bias, before=2, behind=3)


# Products, gradients of rows and 4-bit products with 128 MiB of weights and more, whose single row tiles load them with the streaming hint: one row tile of
# every height, two and three, in launches of less than a round of tiles, which are cut into pieces, and of several.
HEIGHTS = [40, 0, 100, 250, 256, 257, 300, 500, 600, 700, 1, 33, 64, 65, 150, 200]


@pytest.mark.parametrize("kind", ["product", "dx"])
@pytest.mark.parametrize("sizes,n,k", [(HEIGHTS, 2048, 2048), ([30, 65, 0, 129, 161, 193, 225, 20] * 4, 2048, 1024), (HEIGHTS * 2, 4096, 512), ([45, 1, 90], 4096, 8192)])
def test_rows_with_streamed_weights(kind, sizes, n, k):
    assert len(sizes) * n * k * 2 >= 128 << 20 and 28 * len(sizes) < sum(sizes) <= 1024 * len(sizes)
    _rows_case(kind, sizes, n, k, "bf16", bias=kind == "product", before=1, behind=2)


@pytest.mark.parametrize("sizes,n,k", [(HEIGHTS, 8192, 2048), ([30, 65, 0, 129, 161, 193, 225, 20] * 4, 4096, 2048), ([3] * 16, 8192, 2048)])
def test_mx4_product_with_streamed_weights(sizes, n, k):
    assert len(sizes) * n * k // 2 >= 128 << 20 and sum(sizes) * k * (n // 16) > 1 << 24
    _mx4_case(sizes, n, k, "bf16", held=sum(sizes) > 1000, before=1, behind=2)


def test_mx4_product_of_many_fp32_rows():
    _mx4_case([300, 0, 65, 700], 1032, 1056, "f32", held=False)
    _mx4_case([300, 0, 65, 700], 520, 2080, "f32", held=True)


# Few rows an expert on the mean, but all of them with one: streams of weights in many row tiles of one expert.
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_products_whose_rows_meet_in_one_expert(dtype):
    _rows_case("product", [0] * 40 + [1400] + [0] * 23, 256, 320, dtype, bias=True)
    _rows_case("product", [1] * 10 + [700] + [0] * 21, 192, 1088, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_offsets_that_fall(dtype):
    """An expert whose end lies in front of its begin has no rows."""
    dt = {"bf16": BF, "f32": F32}[dtype]
    A, n, k = 100, 72, 64
    off = torch.tensor([10, 5, 40, 30, 400], dtype=torch.int32, device=DEV)  # none, 5 .. 39, none, 30 .. 99
    x, dy, w = _normal((A, k), 1.0, dt, 1), _normal((A, n), 1.0, dt, 2), _normal((4, n, k), 0.1, dt, 3)
    alone = [r for r in range(5, 100) if not 30 <= r < 40]  # (the others are two experts' rows: which result stays is not said)
    out = torch.full((A, n), 7.0, dtype=dt, device=DEV)
    exf.moe_grouped_product(x, off, w, out=out)
    ref, mag, terms = R.rows_product(x, off, w)
    R.assert_sums_close(out[alone], ref[alone], mag[alone], terms, "y")
    assert (out[:5] == 7.0).all()
    out = torch.full((A, k), 7.0, dtype=dt, device=DEV)
    exf.moe_grouped_product_dx(dy, off, w, out=out)
    ref, mag, terms = R.rows_product(dy, off, w, None, True)
    R.assert_sums_close(out[alone], ref[alone], mag[alone], terms, "dx")
    assert (out[:5] == 7.0).all()
    dw, db = exf.moe_grouped_product_dw(dy, x, off, want_bias=True, grad_dtype=F32)
    ref, mag, ref_b, mag_b, terms = R.weight_gradient(dy, x, off)
    R.assert_sums_close(dw, ref, mag, terms, "dw")
    R.assert_sums_close(db, ref_b, mag_b, terms, "db")
    w4 = exf.mx4_quantize(w)
    out = torch.full((A, n), 7.0, dtype=dt, device=DEV)
    exf.moe_grouped_product_mx4(x, off, w4, out=out)
    ref, mag, terms = R.rows_product(R.quantised(x)[0], off, R.held_values(w4.q.view(-1, k // 2), w4.scale).view(4, n, k))
    R.assert_sums_close(out[alone], ref[alone], mag[alone], terms, "mx4")
    assert (out[:5] == 7.0).all()


# ----------------------------------------------------------------------------- arrays beyond 4 GiB
def _wide(shape, dt, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return torch.empty(shape, dtype=dt, device=DEV).normal_(0.0, 0.25, generator=g)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_beyond_4_gib(dtype):
    """2^32 elements of x and more: sampled rows from both ends, and the gradient of a few weights from them."""
    dt, A, n, k = {"bf16": BF, "f32": F32}[dtype], 66000, 64, 65600
    print(f"[case] {A} rows of {k}, {dtype}", flush=True)
    assert A * k > 1 << 32
    x, w = _wide((A, k), dt, 1), _wide((2, n, k), dt, 2)
    off = torch.tensor([0, 100, A], dtype=torch.int32, device=DEV)
    pick = torch.tensor([0, 99, 100, 40000, 65500, 65999], device=DEV)  # (65499 is the last row below 2^32 elements)
    y = exf.moe_grouped_product(x, off, w)
    to = R.sizes_to_offsets([2, 4]).to(DEV)
    R.assert_sums_close(y[pick], *R.rows_product(x[pick].contiguous(), to, w), "y")
    dy = _wide((A, n), dt, 3)
    dx = exf.moe_grouped_product_dx(dy, off, w)
    R.assert_sums_close(dx[pick], *R.rows_product(dy[pick].contiguous(), to, w, None, True), "dx")
    del dx
    dw, _ = exf.moe_grouped_product_dw(dy, x, off, grad_dtype=F32)
    for cols in (slice(0, 8), slice(k - 8, k)):
        ref, mag, _, _, terms = R.weight_gradient(dy, x[:, cols].contiguous(), off)
        R.assert_sums_close(dw[:, :, cols].contiguous(), ref, mag, terms, "dw")
    held, w4 = exf.mx4_quantize(x), exf.mx4_quantize(w)
    assert torch.equal(exf.mx4_dequantize(held, F32)[pick].double(), R.quantised(x[pick].contiguous())[0])
    y4 = exf.moe_grouped_product_mx4(held, off, w4, dtype=dt)
    ref, mag, terms = R.rows_product(R.quantised(x[pick].contiguous())[0], to, R.quantised(w)[0])
    R.assert_sums_close(y4[pick], ref, mag, terms, "mx4")


@pytest.mark.parametrize("A", [3, 300])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_weights_beyond_4_gib(dtype, A):
    """2^32 elements of an expert's weights and more: sampled columns of results, and sampled gradients."""
    dt, n, k = {"bf16": BF, "f32": F32}[dtype], 65600, 66048
    print(f"[case] {A} rows, weights of {n} x {k}, {dtype}", flush=True)
    assert n * k > 1 << 32
    x, w, dy = _wide((A, k), dt, 1), _wide((2, n, k), dt, 2), _wide((A, n), dt, 3)
    off = torch.tensor([0, A // 3, A], dtype=torch.int32, device=DEV)
    y = exf.moe_grouped_product(x, off, w)
    for at in (0, 65024, n - 8):  # (row 65028 is the first one beyond 2^32 elements)
        R.assert_sums_close(y[:, at:at + 8].contiguous(), *R.rows_product(x, off, w[:, at:at + 8].contiguous()), "y")
    dx = exf.moe_grouped_product_dx(dy, off, w)
    for at in (0, k - 8):
        R.assert_sums_close(dx[:, at:at + 8].contiguous(), *R.rows_product(dy, off, w[:, :, at:at + 8].contiguous(), None, True), "dx")
    w4 = exf.mx4_quantize(w)
    del w
    y4 = exf.moe_grouped_product_mx4(x, off, w4)
    codes, scales = w4.q.view(2 * n, k // 2), w4.scale
    for at in (0, 65024, n - 8):
        rows = torch.cat([torch.arange(e * n + at, e * n + at + 8, device=DEV) for e in (0, 1)])
        w8 = R.held_values(codes[rows], scales[:, rows].contiguous()).view(2, 8, k)
        R.assert_sums_close(y4[:, at:at + 8].contiguous(), *R.rows_product(R.quantised(x)[0], off, w8), "mx4")
    del w4, codes, scales
    dw, _ = exf.moe_grouped_product_dw(dy, x, off)
    for at in (0, 65024, n - 8):
        ref, mag, _, _, terms = R.weight_gradient(dy[:, at:at + 8].contiguous(), x, off)
        R.assert_sums_close(dw[:, at:at + 8].contiguous(), ref, mag, terms, "dw")


def test_some_of_the_experts():
    """Experts 1 and 2 of four, cut out of the others' 4-bit weights as Mx4 says, and quantised by themselves."""
    n, k, off = 72, 544, torch.tensor([0, 30, 41], dtype=torch.int32, device=DEV)
    w, x = _normal((4, n, k), 0.1, BF, 1), _normal((41, k), 1.0, BF, 2)
    m = exf.mx4_quantize(w)
    cut, own = exf.Mx4(m.q[1:3], m.scale[:, n:3 * n].contiguous()), exf.mx4_quantize(w[1:3])
    assert torch.equal(cut.q, own.q) and torch.equal(cut.scale, own.scale)
    assert torch.equal(exf.moe_grouped_product_mx4(x, off, cut), exf.moe_grouped_product_mx4(x, off, own))
    with pytest.raises(exf.ExflowError):
        exf.moe_grouped_product_mx4(x, off, exf.Mx4(m.q[1:3], m.scale[:, n:3 * n]))
