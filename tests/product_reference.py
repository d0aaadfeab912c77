"""The experts' products in 64 bits, from their definitions, and how far a kernel that sums in fp32 may be from them."""
import torch

U32 = 2.0 ** -24  # unit roundoff of fp32
BLOCK = 32


def sizes_to_offsets(sizes, first=0):
    return torch.tensor([first, *(first + torch.cumsum(torch.tensor(sizes), 0)).tolist()], dtype=torch.int32)


def ranges(offsets, A):
    """Clamped row range of every expert."""
    out = []
    for lo, hi in zip(offsets[:-1].tolist(), offsets[1:].tolist()):
        lo = min(max(lo, 0), A)
        out.append((lo, min(max(hi, lo), A)))
    return out


def rows_product(rows, offsets, w, bias=None, gradient=False):
    """(result, sum of the terms' magnitudes, reduction length), rows outside all ranges NaN / 0."""
    A, E = rows.shape[0], w.shape[0]
    N = w.shape[2] if gradient else w.shape[1]
    ref = torch.full((A, N), float("nan"), dtype=torch.float64, device=rows.device)
    mag = torch.zeros((A, N), dtype=torch.float64, device=rows.device)
    for e, (lo, hi) in enumerate(ranges(offsets, A)):
        if lo == hi:
            continue
        x, m = rows[lo:hi].double(), w[e].double()
        m = m if gradient else m.t().contiguous()
        ref[lo:hi], mag[lo:hi] = x @ m, x.abs() @ m.abs()
        if bias is not None:
            ref[lo:hi] += bias[e].double()
            mag[lo:hi] += bias[e].double().abs()
    return ref, mag, rows.shape[1] + 1


def weight_gradient(dy, x, offsets):
    E = offsets.numel() - 1
    dev = x.device
    dw = torch.zeros((E, dy.shape[1], x.shape[1]), dtype=torch.float64, device=dev)
    db = torch.zeros((E, dy.shape[1]), dtype=torch.float64, device=dev)
    mw, mb, longest = torch.zeros_like(dw), torch.zeros_like(db), 1
    for e, (lo, hi) in enumerate(ranges(offsets, x.shape[0])):
        if lo == hi:
            continue
        a, b = dy[lo:hi].double(), x[lo:hi].double()
        at = a.t().contiguous()
        dw[e], mw[e] = at @ b, at.abs() @ b.abs()
        db[e], mb[e] = a.sum(0), a.abs().sum(0)
        longest = max(longest, hi - lo)
    return dw, mw, db, mb, longest


def assert_sums_close(got, ref, mag, terms, what=""):
    """A sum of `terms` fp32 products in any order is within terms * u * (sum of magnitudes) of the exact one; the products' own roundings and
    a hardware that chops instead of rounding cost a factor of two each at most; then one rounding to the type of `got`: half of the
    last place of 8 (bf16) or 24 (fp32) binary digits, 2^-8 or 2^-24 of the value."""
    g = got.double()
    half_ulp = 2.0 ** -8 if got.dtype == torch.bfloat16 else 2.0 ** -24
    tiny = 2.0 ** -133 if got.dtype == torch.bfloat16 else 2.0 ** -149
    err = (g - ref).abs()
    sums = 4 * (terms + 1) * U32 * mag
    lim = sums + half_ulp * 1.01 * (ref.abs() + sums) + tiny
    bad = ~(err <= lim)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} outside, worst excess {float((err - lim)[bad].max()):.3e} at {torch.nonzero(bad)[0].tolist()}"


def power_of_two(exponent):
    """2^exponent in 64 bits, exactly (the device's own exponential functions are not)."""
    return ((exponent.long() + 1023) << 52).view(torch.float64)


def quantised(x):
    """(values in 64 bits, scale bytes) of rows in blocks of 32: nearest of what four bits say, ties to the even code."""
    b = x.double().reshape(*x.shape[:-1], -1, BLOCK)
    most = b.abs().amax(-1, keepdim=True)
    broken = ~torch.isfinite(b).all(-1, keepdim=True)
    fraction, exponent = torch.frexp(torch.where(broken, 1.0, most))
    exponent = torch.where(fraction == 0, -127, exponent - 3).clamp(min=-127)
    t = torch.where(broken, 0.0, b) * power_of_two(-exponent)
    table = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64, device=x.device)
    halfway = (table[1:] + table[:-1]) / 2
    below, upto = torch.bucketize(t.abs(), halfway), torch.bucketize(t.abs(), halfway, right=True)
    code = torch.where(below % 2 == 0, below, upto)
    v = torch.copysign(table[code], t) * power_of_two(exponent)
    v = torch.where(broken, float("nan"), v).reshape(x.shape)
    byte = torch.where(broken, 255, exponent + 127).squeeze(-1)
    return v, byte.to(torch.uint8)


def scale_tiles(byte):
    """Scale bytes [rows, k/32] in the layout [ceil(k/256), rows, 8]."""
    rows, blocks = byte.shape
    tiles = (blocks + 7) // 8
    full = torch.zeros((rows, tiles * 8), dtype=torch.uint8, device=byte.device)
    full[:, :blocks] = byte
    return full.view(rows, tiles, 8).transpose(0, 1).contiguous()


def held_values(q, scale):
    """What packed codes [rows, k/2] and scale bytes [tiles, rows, 8] stand for, in 64 bits."""
    rows, half = q.shape
    code = torch.stack((q % 16, q // 16), -1).reshape(rows, 2 * half)
    table = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64, device=q.device)
    v = torch.where(code >= 8, -table[(code % 8).long()], table[(code % 8).long()])
    byte = scale.transpose(0, 1).reshape(rows, -1)[:, :2 * half // BLOCK].int()
    s = torch.where(byte == 255, float("nan"), power_of_two(byte - 127))
    return v * s.repeat_interleave(BLOCK, 1)
