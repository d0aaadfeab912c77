"""Routing to many experts, the rows of their assignments and 4-bit integers with group scales in 64 bits, from their definitions, and how far kernels that compute
in fp32 may be from them."""
import torch

U32 = 2.0 ** -24
SOFTMAX, SIGMOID = 0, 1
INF = float("inf")


def scores(logits, score):
    l = logits.double()
    if score == SIGMOID:
        return 1 / (1 + torch.exp(-l))
    top = l.amax(1, keepdim=True)
    e = torch.exp(l - torch.where(top == -INF, 0.0, top))
    total = e.sum(1, keepdim=True)
    return e / torch.where(total == 0, 1.0, total)


def _ranked(values):
    """Order of each row, largest first, the lowest index of equals first."""
    return torch.sort(values, dim=1, descending=True, stable=True)[1]


def route(logits, k, bias=None, score=SOFTMAX, renormalize=False, scale=1.0, groups=1, top_groups=None, group_best=1):
    """(ids [T,k], weights in 64 bits [T,k], scores [T,E]) of rows without NaN."""
    T, E = logits.shape
    s = scores(logits, score)
    out = torch.isnan(logits) | (logits == -INF)
    key = logits.double() if bias is None else s + bias.double()
    out |= torch.isnan(key) | (key == -INF)
    key = torch.where(out, -INF, key)
    top_groups = groups if top_groups is None else top_groups
    if groups > 1:
        by = torch.where(out, -INF, s) if bias is None and group_best == 2 else key
        high = torch.sort(by.view(T, groups, -1), dim=2, descending=True)[0][..., :group_best]
        value = torch.where(high[..., 0] == -INF, -INF, torch.where(high == -INF, 0.0, high).sum(-1))
        rank = torch.empty((T, groups), dtype=torch.int64, device=logits.device)
        rank.scatter_(1, _ranked(value), torch.arange(groups, device=logits.device).expand(T, groups))
        key = torch.where((rank < top_groups).repeat_interleave(E // groups, 1), key, -INF)
    idx = _ranked(key)[:, :k]
    idx = torch.where(torch.gather(key, 1, idx) == -INF, -1, idx)
    return idx, weights(logits, idx, score, renormalize, scale, s), s


def weights(logits, idx, score, renormalize, scale, s=None):
    """Weights of given ids; renormalised ones by shares of exp(log score), which do not underflow."""
    s = scores(logits, score) if s is None else s
    live = (idx >= 0) & (idx < logits.shape[1])
    at = idx.clamp(0, logits.shape[1] - 1).long()
    if renormalize and idx.shape[1] > 1:
        l = torch.gather(logits.double(), 1, at)
        log = torch.nn.functional.logsigmoid(l) if score == SIGMOID else l
        log = torch.where(live, log, -INF)
        top = log.amax(1, keepdim=True)
        u = torch.exp(log - torch.where(top == -INF, 0.0, top))
        u = torch.where(live, u, 0.0)
        total = u.sum(1, keepdim=True)
        return scale * u / torch.where(total == 0, 1.0, total)
    return scale * torch.where(live, torch.gather(s, 1, at), 0.0)


def spread(logits):
    """How far a row's finite logits lie below its largest, or from zero (an argument of exp this far off zero is rounded by so many units)."""
    l = logits.double()
    fine = torch.isfinite(l) & (l.abs() < 1e4)
    top = torch.where(fine, l, -INF).amax(1, keepdim=True)
    away = torch.where(fine, torch.maximum(l.abs(), top - l), 0.0).amax(1, keepdim=True)
    return away.clamp(max=200.0)


def route_gradient(logits, idx, g, score, renormalize, scale, dscores=None):
    """(dlogits, sum of the magnitudes of its terms) in 64 bits."""
    T, E = logits.shape
    s = scores(logits, score)
    live = (idx >= 0) & (idx < E)
    at = idx.clamp(0, E - 1).long()
    g = torch.where(live, g.double(), 0.0)
    dl, mag = torch.zeros_like(s), torch.zeros_like(s)
    d = torch.zeros_like(s) if dscores is None else dscores.double().expand(T, E)
    d = torch.where(s > 0, d, 0.0)  # masked experts, whatever their gradient
    mine = torch.where(live, torch.gather(s, 1, at), 0.0)
    if renormalize and idx.shape[1] > 1:
        w = weights(logits, idx, score, True, scale, s)
        share = w / scale if scale else weights(logits, idx, score, True, 1.0, s)
        mean, size = (g * share).sum(1, keepdim=True), (g.abs() * share).sum(1, keepdim=True)
        slope = 1 - mine if score == SIGMOID else torch.ones_like(mine)
        dl.scatter_add_(1, at, torch.where(live, w * (g - mean) * slope, 0.0))
        mag.scatter_add_(1, at, torch.where(live, w.abs() * (g.abs() + size) * slope, 0.0))
    elif score == SIGMOID:
        dl.scatter_add_(1, at, scale * g * mine * (1 - mine))
        mag.scatter_add_(1, at, abs(scale) * g.abs() * mine * (1 - mine))
    else:
        d = d.scatter_add(1, at, scale * g)
    if score == SIGMOID:
        dl += d * s * (1 - s)
        mag += d.abs() * s * (1 - s)
    else:
        size = torch.where(s > 0, dscores.double().expand(T, E).abs(), 0.0) if dscores is not None else torch.zeros_like(s)
        if not (renormalize and idx.shape[1] > 1):
            size = size.scatter_add(1, at, abs(scale) * g.abs())
        dl += s * (d - (s * d).sum(1, keepdim=True))
        mag += s * (size + (s * size).sum(1, keepdim=True))
    return dl, mag


def assert_close(got, ref, mag, units, what=""):
    """Each of the terms, of magnitude `mag` together, is off by at most `units` units roundoff of fp32; then one rounding to the type of `got`."""
    g, half = got.double(), 2.0 ** -8 if got.dtype == torch.bfloat16 else U32
    lim = units * U32 * mag
    lim = lim + half * 1.01 * (ref.abs() + lim) + (2.0 ** -133 if got.dtype == torch.bfloat16 else 2.0 ** -126)
    bad = ~((g - ref).abs() <= lim)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} outside, at {torch.nonzero(bad)[0].tolist()}: {g[bad][0]} and {ref[bad][0]}, allowed {lim.expand_as(ref)[bad][0]:.3e}"


def assignments(T, k, E_local, g, kept=1.0):
    """(sorted_of_src [T*k], src_of_sorted) of random experts; a share of the assignments is not kept."""
    e = torch.randint(0, E_local, (T * k,), generator=g)
    e = torch.where(torch.rand(T * k, generator=g) < kept, e, E_local)
    order = torch.argsort(e, stable=True)
    n = int((e < E_local).sum())
    position = torch.full((T * k,), -1, dtype=torch.int32)
    position[order[:n]] = torch.arange(n, dtype=torch.int32)
    return position, order[:n]


def q4_values(q, scale, zero):
    """What packed codes [..., k/2], scales and zero points (or None) [..., k/group] stand for, in 64 bits."""
    code = torch.stack((q % 16, q // 16), -1).flatten(-2).double()
    group = code.shape[-1] // scale.shape[-1]
    at = 8.0 if zero is None else zero.double().repeat_interleave(group, -1)
    return (code - at) * scale.double().repeat_interleave(group, -1)


def q4_quantised(x, group, symmetric):
    """(codes [..., k], scale, zero or None) of rows, by the definition."""
    v = x.double().reshape(*x.shape[:-1], -1, group)
    broken = ~torch.isfinite(v).all(-1)
    v = torch.where(broken[..., None], 0.0, v)
    lo, hi = v.amin(-1).clamp(max=0), v.amax(-1).clamp(min=0)
    scale = (torch.maximum(hi, -lo) / 7 if symmetric else (hi - lo) / 15).float().to(x.dtype)
    by = torch.where(scale == 0, 1.0, scale.double())
    zero = torch.full_like(by, 8.0) if symmetric else torch.round(-lo / by).clamp(max=15)
    zero = torch.where(scale == 0, 8.0 if symmetric else 0.0, zero)
    code = (torch.round(v / by[..., None]) + zero[..., None]).clamp(0, 15)
    code = torch.where((scale == 0)[..., None], zero[..., None], code)
    scale = torch.where(broken, torch.full_like(scale, float("nan")), scale)
    return code.reshape(x.shape).to(torch.uint8), scale, None if symmetric else zero.to(torch.uint8)
