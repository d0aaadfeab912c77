"""Routing to many experts with its gradient, the rows of more than two experts a token with theirs, and the experts' products with weights in 4-bit
integers with group scales, as programs call them.

``listed()`` names the cases that stand for each range, ``draw(rng)`` gives further ones of the same ranges.  A case is a dict
of plain values with a ``kind``; T tokens, E experts, k of them chosen by a token:

  route         ids and weights from logits (``score``: softmax or sigmoid; ``bias``: of each expert, for balance; ``groups`` of experts, the best
                ``top`` stay, by the sum of their ``best`` highest keys; ``renorm``, ``scale``: of the weights; ``scores``: wanted as well)
  route_grad    gradient of the logits from that of the weights (``balance``: and from that of the scores, the same for all tokens)
  combine       out[t] = sum_j w[t][j] y_sorted[position of (t, j)] (``weighted`` false: with weights of one, the gradient of the dispatch)
  combine_grad  gradients of the sorted rows and of the weights of combine
  q4            y = x W^T + b with W [E,n,k] in 4 bits, ``group`` elements with a common scale and (``zeros``) zero point
  quantise      rows into such groups, and back

The weight of a token's only expert (k = 1) is its score, as in moe_gate_topk: nothing is renormalised.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda"
DTYPE = {"bf16": torch.bfloat16, "f32": torch.float32}
MAX_LOGITS = 32768 * 256
MAX_ROWS = 16384 * 8 * 2048          # elements of the sorted rows of combine ...
MAX_ROWS_GRAD = 8192 * 8 * 2048      # ... and of combine_grad
MAX_WEIGHTS = 64 * 16384 * 4096
MAX_FLOPS = 2.0 * 512 * 16384 * 4096
MAX_PADDED_FLOPS = 1.2e12            # of groups padded to the largest
MAX_HELD = 32 * 8192 * 2048


def _route(T, E, k, score, dtype="f32", bias=False, groups=1, top=1, best=1, renorm=True, scale=1.0, scores=False):
    return dict(kind="route", T=T, E=E, k=k, score=score, dtype=dtype, bias=bias, groups=groups, top=top, best=best, renorm=renorm and k > 1, scale=scale, scores=scores)


def _route_grad(T, E, k, score, dtype="f32", renorm=True, scale=1.0, balance=False):
    return dict(kind="route_grad", T=T, E=E, k=k, score=score, dtype=dtype, renorm=renorm and k > 1, scale=scale, balance=balance)


def _rows(kind, T, d, k, dtype="bf16", E=64, E_local=64, weighted=True):
    return dict(kind=kind, T=T, d=d, k=k, dtype=dtype, E=E, E_local=E_local, weighted=weighted)


def _q4(A, n, k, E, group=128, dtype="bf16", zeros=True, bias=False, skew=0.0):
    return dict(kind="q4", A=A, n=n, k=k, E=E, group=group, dtype=dtype, zeros=zeros, bias=bias, skew=skew)


def listed():
    return [
        # the smallest call of a serving loop: one token among 128 experts, latency
        dict(name="route_one_token", **_route(1, 128, 8, "softmax", dtype="bf16")),
        # prefill with experts in groups and a bias that keeps them balanced
        dict(name="route_prefill_grouped", **_route(32768, 256, 8, "sigmoid", bias=True, groups=8, top=4, best=2, scale=2.5)),
        # training of an odd number of tokens on an odd number of experts: renormalised weights
        dict(name="route_grad_odd", **_route_grad(777, 60, 6, "sigmoid", dtype="bf16")),
        # a training step's whole batch, with the gradient of a balance loss
        dict(name="route_grad_balance", **_route_grad(32768, 256, 8, "softmax", renorm=False, balance=True)),
        # prefill of an XL-shaped layer with eight experts a token
        dict(name="combine_top8", **_rows("combine", 16384, 2048, 8)),
        # gradient of the dispatch of a short ragged fp32 batch, of which a GPU holds a share of the experts
        dict(name="combine_ragged_share", **_rows("combine", 333, 1028, 6, dtype="f32", E=48, E_local=12, weighted=False)),
        # a training step of that layer
        dict(name="combine_grad_top8", **_rows("combine_grad", 8192, 2048, 8)),
        # ... of the tokens of a short fp32 batch
        dict(name="combine_grad_short", **_rows("combine_grad", 129, 520, 3, dtype="f32", E=8, E_local=8)),
        # one token through one expert of the 350M-shaped model: latency
        dict(name="q4_one_token", **_q4(1, 4096, 1024, 8)),
        # decode of the widest layer: 256 tokens, top-2, every one of 64 experts' weights (2.2 GB) is read once
        dict(name="q4_decode_wide", **_q4(512, 16384, 4096, 64)),
        # one fp32 expert of the 350M-shaped model, symmetric, short groups
        dict(name="quantise_one_expert", kind="quantise", A=4096, k=1024, group=32, dtype="f32", zeros=False),
        # all experts' weights of an XL-shaped layer, as a program that loads a checkpoint quantises them
        dict(name="quantise_weights_xl", kind="quantise", A=32 * 8192, k=2048, group=128, dtype="bf16", zeros=True),
    ]


# ---------------------------------------------------------------------------------------------- drawn cases
def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    while True:
        kind = rng.choice(("route", "route", "route_grad", "combine", "combine_grad", "q4", "q4", "quantise"))
        dtype = rng.choice(("bf16", "f32"))
        if kind in ("route", "route_grad"):
            score = rng.choice(("softmax", "sigmoid"))
            groups = rng.choice((1, 1, 2, 4, 8)) if kind == "route" else 1
            E = groups * _log_int(rng, 2, 512 // groups)
            T = _log_int(rng, 1, 65536)
            top = rng.randint(1, groups)
            k = _log_int(rng, 1, min(16, top * E // groups))
            if T * E > MAX_LOGITS:
                continue
            renorm, scale = rng.random() < 0.6, rng.choice((1.0, 1.0, 2.5))
            if kind == "route":
                best = rng.choice((1, 2)) if groups > 1 else 1
                return _route(T, E, k, score, dtype, rng.random() < 0.5, groups, top, best, renorm, scale, rng.random() < 0.2)
            return _route_grad(T, E, k, score, dtype, renorm, scale, rng.random() < 0.4)
        if kind in ("combine", "combine_grad"):
            step = 8 if dtype == "bf16" else 4
            c = _rows(kind, _log_int(rng, 1, 65536), step * _log_int(rng, 1, 8192 // step), _log_int(rng, 1, 16), dtype, E=64,
                      E_local=rng.choice((64, 64, 16)), weighted=kind != "combine" or rng.random() < 0.6)
            most = (MAX_ROWS if kind == "combine" else MAX_ROWS_GRAD) // (1 if dtype == "bf16" else 2)
            if c["T"] * c["k"] * c["d"] <= most:
                return c
            continue
        group = rng.choice((32, 64, 128, 128))
        k = group * _log_int(rng, 1, 16384 // group)
        zeros = rng.random() < 0.6
        if kind == "quantise":
            A = _log_int(rng, 1, 32 * 8192)
            if A * k <= MAX_HELD // (1 if dtype == "bf16" else 2):
                return dict(kind=kind, A=A, k=k, group=group, dtype=dtype, zeros=zeros)
            continue
        if rng.random() < 0.5:
            dtype = "bf16"
        step = 8 if dtype == "bf16" else 4
        A, n, E = _log_int(rng, 1, 2048 if dtype == "bf16" else 256), step * _log_int(rng, 1, 16384 // step), _log_int(rng, 1, 64)
        c = _q4(A, n, k, E, group, dtype, zeros, rng.random() < 0.5, rng.choice((0.0, 0.0, 0.5)))
        largest = A * (3.0 if c["skew"] else 1.0) + 4 * E  # about what the groups are padded to, times E
        limit = MAX_FLOPS if dtype == "bf16" else MAX_FLOPS / 8
        if E * n * k <= MAX_WEIGHTS // (1 if dtype == "bf16" else 8) and 2.0 * A * n * k <= limit and 2.0 * largest * n * k <= MAX_PADDED_FLOPS:
            return c


# ---------------------------------------------------------------------------------------------- inputs
def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _normal(shape, std, dtype, g):
    return torch.empty(shape, dtype=dtype, device=DEV).normal_(0.0, std, generator=g)


def _chosen(T, E, k, g):
    """k different experts of every token, some of them preferred by all."""
    liking = torch.rand((T, E), device=DEV, generator=g) + 0.3 * torch.rand((1, E), device=DEV, generator=g)
    return torch.argsort(liking, dim=1, descending=True)[:, :k].contiguous()


def _held(rows, k, group, dtype, zeros, g):
    """Weights ~ N(0, 0.02) held in 4 bits: packed codes [rows, k/2] (low half first), scales and zero points [rows, k/group].  A program has them from
    a checkpoint."""
    q = torch.empty((rows, k // 2), dtype=torch.uint8, device=DEV)
    scale = torch.empty((rows, k // group), dtype=dtype, device=DEV)
    zero = torch.empty((rows, k // group), dtype=torch.uint8, device=DEV) if zeros else None
    most = max(1, (1 << 26) // k)
    for lo in range(0, rows, most):
        v = _normal((min(most, rows - lo), k // group, group), 0.02, torch.float32, g)
        low, high = v.amin(-1), v.amax(-1)
        s = ((high - low) / 15 if zeros else torch.maximum(high, -low) / 7).to(dtype)
        at = torch.round(-low / s.float()) if zeros else torch.full_like(low, 8.0)
        code = (torch.round(v / s.float()[..., None]) + at[..., None]).clamp(0, 15).to(torch.uint8).view(-1, k // 2, 2)
        q[lo:lo + most] = code[..., 0] + 16 * code[..., 1]
        scale[lo:lo + most] = s
        if zeros:
            zero[lo:lo + most] = at.clamp(0, 15).to(torch.uint8)
    return q, scale, zero


def prepare(case, seed):
    c, g, dt = case, _gen(seed), DTYPE[case["dtype"]]
    s = dict(case=c)
    if c["kind"] in ("route", "route_grad"):
        T, E, k = c["T"], c["E"], c["k"]
        s["logits"] = _normal((T, E), 1.5, dt, g)
        if c["kind"] == "route":
            s["bias"] = _normal((E,), 0.05 if c["score"] == "sigmoid" else 0.2 / E, torch.float32, g) if c["bias"] else None
        else:
            s["idx"] = torch.argsort(s["logits"].float() + _normal((1, E), 0.3, torch.float32, g), dim=1, descending=True, stable=True)[:, :k].int().contiguous()
            s["dw"] = _normal((T, k), 1e-2, torch.float32, g)
            s["dscores"] = _normal((E,), 1e-3, torch.float32, g) if c["balance"] else None
        return s
    if c["kind"] in ("combine", "combine_grad"):
        T, d, k = c["T"], c["d"], c["k"]
        e = _chosen(T, c["E"], k, g).view(-1)
        order = torch.argsort(torch.where(e < c["E_local"], e, c["E"]), stable=True)
        s["kept"] = kept = int((e < c["E_local"]).sum())
        s["src"] = order[:kept]
        position = torch.full((T * k,), -1, dtype=torch.int32, device=DEV)
        position[order[:kept]] = torch.arange(kept, dtype=torch.int32, device=DEV)
        s["position"] = position
        s["y"] = _normal((T * k, d), 1.0, dt, g)
        s["w"] = torch.rand((T, k), device=DEV, generator=g) / k if c["weighted"] else None
        if c["kind"] == "combine":
            s["out"] = torch.empty((T, d), dtype=dt, device=DEV)
        else:
            s["dout"] = _normal((T, d), 1e-2, dt, g)
            s["dy"] = torch.zeros((T * k, d), dtype=dt, device=DEV)  # rows behind the last kept one stay as they are
        return s
    if c["kind"] == "quantise":
        # rows of different magnitude, as tokens and channels have
        s["x"] = (_normal((c["A"], c["k"]), 0.02, torch.float32, g) * torch.exp2(torch.randint(-3, 4, (c["A"], 1), device=DEV, generator=g))).to(dt)
        s["out"] = torch.empty((c["A"], c["k"]), dtype=dt, device=DEV)
        s["q"] = torch.empty((c["A"], c["k"] // 2), dtype=torch.uint8, device=DEV)
        s["scale"] = torch.empty((c["A"], c["k"] // c["group"]), dtype=dt, device=DEV)
        s["zero"] = torch.empty((c["A"], c["k"] // c["group"]), dtype=torch.uint8, device=DEV) if c["zeros"] else None
        return s
    A, n, k, E = c["A"], c["n"], c["k"], c["E"]
    h = torch.Generator()
    h.manual_seed(seed)
    loads = (1.0 / torch.arange(1, E + 1, dtype=torch.float64) ** c["skew"])[torch.randperm(E, generator=h)]
    sizes = torch.bincount(torch.multinomial(loads, A, replacement=True, generator=h), minlength=E)
    offsets = torch.zeros(E + 1, dtype=torch.int32)
    offsets[1:] = torch.cumsum(sizes, 0)
    s["offsets"], s["largest"] = offsets.to(DEV), int(sizes.max())
    s["x"] = _normal((A, k), 1.0, dt, g)
    q, scale, zero = _held(E * n, k, c["group"], dt, c["zeros"], g)
    s["q"], s["scale"], s["zero"] = q.view(E, n, -1), scale.view(E, n, -1), None if zero is None else zero.view(E, n, -1)
    s["bias"] = _normal((E, n), 0.02, dt, g) if c["bias"] else None
    s["out"] = torch.empty((A, n), dtype=dt, device=DEV)
    return s


# ---------------------------------------------------------------------------------------------- plain forms
def _softmax(logits):
    e = torch.exp(logits - logits.amax(1, keepdim=True))
    return e / e.sum(1, keepdim=True)


def _plain_route(s):
    c, logits, b = s["case"], s["logits"], s["bias"]
    T, E, k = c["T"], c["E"], c["k"]
    # which experts: keys in 64 bits (values next to a border); without a bias the logits say the order by themselves
    wide = _softmax(logits.double()) if c["score"] == "softmax" else torch.sigmoid(logits.double())
    key = logits.double() if b is None else wide + b.double()
    if c["groups"] > 1:
        by = (wide if b is None else key) if c["best"] == 2 else key
        size = E // c["groups"]
        high = torch.sort(by.view(T, c["groups"], size), dim=2, descending=True)[0]
        value = high[..., 0] + high[..., 1] if c["best"] == 2 and size > 1 else high[..., 0]
        stay = torch.sort(value, dim=1, descending=True, stable=True)[1][:, :c["top"]]
        mask = torch.zeros((T, c["groups"]), dtype=torch.bool, device=DEV).scatter_(1, stay, True)
        key = torch.where(mask.repeat_interleave(size, 1), key, -math.inf)
    idx = torch.sort(key, dim=1, descending=True, stable=True)[1][:, :k]
    scores = _softmax(logits.float()) if c["score"] == "softmax" else torch.sigmoid(logits.float())
    w = torch.gather(scores, 1, idx)
    if c["renorm"]:
        w = w / w.sum(1, keepdim=True)
    w = w * c["scale"]
    return (idx.int(), w, scores) if c["scores"] else (idx.int(), w)


def _plain_route_grad(s):
    c, l, idx, g = s["case"], s["logits"].float(), s["idx"].long(), s["dw"] * s["case"]["scale"]
    p = _softmax(l) if c["score"] == "softmax" else torch.sigmoid(l)
    mine = torch.gather(p, 1, idx)
    if c["renorm"]:
        total = mine.sum(1, keepdim=True)
        g = (g - (g * mine).sum(1, keepdim=True) / total) / total
    dp = torch.zeros_like(p).scatter_add_(1, idx, g)
    if s["dscores"] is not None:
        dp = dp + s["dscores"]
    if c["score"] == "softmax":
        dl = p * (dp - (dp * p).sum(1, keepdim=True))
    else:
        dl = dp * p * (1 - p)
    return dl.to(s["logits"].dtype)


def _plain_combine(s):
    c = s["case"]
    out = torch.zeros((c["T"], c["d"]), device=DEV)
    position = s["position"].view(c["T"], c["k"]).long()
    for j in range(c["k"]):
        at = position[:, j]
        w = (at >= 0).float()
        if s["w"] is not None:
            w = w * s["w"][:, j]
        out += w[:, None] * torch.where(at[:, None] >= 0, s["y"][at.clamp(min=0)].float(), 0.0)
    return out.to(DTYPE[c["dtype"]])


def _plain_combine_grad(s):
    c, src = s["case"], s["src"]
    rows = s["dout"][src // c["k"]].float()
    dy = torch.zeros((c["T"] * c["k"], c["d"]), dtype=DTYPE[c["dtype"]], device=DEV)
    dy[:s["kept"]] = (rows * s["w"].view(-1)[src][:, None]).to(dy.dtype)
    dw = torch.zeros(c["T"] * c["k"], device=DEV)
    dw[src] = (rows * s["y"][:s["kept"]].float()).sum(1)
    return dy, dw.view(c["T"], c["k"])


def _values(q, scale, zero, group):
    """What packed codes [..., k/2], scales and zero points [..., k/group] stand for, in 32 bits."""
    code = torch.stack((q & 15, q >> 4), -1).view(*q.shape[:-1], -1, group).float()
    at = 8.0 if zero is None else zero[..., None].float()
    return ((code - at) * scale[..., None].float()).view(*q.shape[:-1], -1)


def _plain_q4(s):
    c, off, largest = s["case"], s["offsets"], s["largest"]
    at = off[:-1, None].long() + torch.arange(largest, device=DEV)
    there = at < off[1:, None]
    x = torch.where(there[..., None], s["x"][at.clamp(max=c["A"] - 1)].float(), 0.0)
    y = torch.bmm(x, _values(s["q"], s["scale"], s["zero"], c["group"]).transpose(1, 2))
    if s["bias"] is not None:
        y = y + s["bias"].float()[:, None, :]
    r = torch.arange(c["A"], device=DEV)
    e = torch.searchsorted(off[1:], r.int(), right=True, out_int32=True).long()
    return y[e, r - off[e]].to(DTYPE[c["dtype"]])


def _plain_quantise(s):
    c, dt = s["case"], DTYPE[s["case"]["dtype"]]
    parts = []
    for rows in s["x"].split(max(1, (1 << 27) // c["k"])):
        v = rows.view(rows.shape[0], -1, c["group"])
        if c["zeros"]:
            low, high = v.amin(-1).clamp(max=0).double(), v.amax(-1).clamp(min=0).double()
            scale = ((high - low) / 15).float().to(dt)
        else:
            low, scale = None, (v.abs().amax(-1).double() / 7).float().to(dt)
        # (quotients next to the middle between two codes: in 64 bits)
        by = torch.where(scale == 0, 1.0, scale.double())
        at = torch.round(-low / by).clamp(0, 15)[..., None] if c["zeros"] else 8.0
        code = torch.clamp(torch.round(v.double() / by[..., None]) + at, 0, 15)
        parts.append(((code - at).float() * scale.float()[..., None]).to(dt).view(rows.shape))
    return torch.cat(parts)


PLAIN = dict(route=_plain_route, route_grad=_plain_route_grad, combine=_plain_combine, combine_grad=_plain_combine_grad, q4=_plain_q4, quantise=_plain_quantise)


def run(state):
    if not own:
        return PLAIN[state["case"]["kind"]](state)
    import paper_2401_08383_amd as exf

    s, c = state, state["case"]
    kind = c["kind"]
    if kind in ("route", "route_grad"):
        score = exf.EXF_SCORE_SOFTMAX if c["score"] == "softmax" else exf.EXF_SCORE_SIGMOID
    if kind == "route":
        idx, w, scores = exf.moe_route(s["logits"], c["k"], bias=s["bias"], score=score, renormalize=c["renorm"], scale=c["scale"], groups=c["groups"],
                                       top_groups=c["top"], group_best=c["best"], want_scores=c["scores"])
        return (idx, w, scores) if c["scores"] else (idx, w)
    if kind == "route_grad":
        return exf.moe_route_backward(s["dw"], s["logits"], s["idx"], score=score, renormalize=c["renorm"], scale=c["scale"], dscores=s["dscores"])
    if kind == "combine":
        if s["w"] is None:
            return exf.moe_dispatch_backward(s["y"], s["position"], c["k"], out=s["out"])
        return exf.moe_combine(s["y"], s["position"], s["w"], out=s["out"])
    if kind == "combine_grad":
        return exf.moe_combine_backward(s["dout"], s["y"], s["position"], s["w"], out=s["dy"])
    if kind == "q4":
        return exf.moe_grouped_product_q4(s["x"], s["offsets"], exf.Q4(s["q"], s["scale"], s["zero"]), s["bias"], out=s["out"])
    held = exf.q4_quantize(s["x"], c["group"], symmetric=not c["zeros"], out=exf.Q4(s["q"], s["scale"], s["zero"]))
    return exf.q4_dequantize(held, out=s["out"])


# ---------------------------------------------------------------------------------------------- work
def work(case):
    c = case
    el = 2 if c["dtype"] == "bf16" else 4
    if c["kind"] == "route":
        return {"bytes": c["T"] * (c["E"] * (el + 4 * c["scores"]) + 8 * c["k"]) + 4 * c["E"] * c["bias"], "flops": 4.0 * c["T"] * c["E"]}
    if c["kind"] == "route_grad":
        sparse = c["renorm"] and not c["balance"] or c["score"] == "sigmoid" and not c["balance"]  # the chosen experts' logits only
        return {"bytes": c["T"] * ((c["k"] if sparse else c["E"]) * el + c["E"] * el + 8 * c["k"]) + 4 * c["E"] * c["balance"], "flops": 4.0 * c["T"] * c["E"]}
    if c["kind"] in ("combine", "combine_grad"):
        kept = c["T"] * c["k"] * c["E_local"] / c["E"]
        if c["kind"] == "combine":
            return {"bytes": (kept + c["T"]) * c["d"] * el + c["T"] * c["k"] * (4 + 4 * c["weighted"]), "flops": 2.0 * kept * c["d"]}
        return {"bytes": (2 * kept + c["T"]) * c["d"] * el + 12 * c["T"] * c["k"], "flops": 3.0 * kept * c["d"]}
    held = 1 / 2 + (el + c["zeros"]) / c["group"]  # bytes an element
    if c["kind"] == "quantise":
        return {"bytes": 2 * c["A"] * c["k"] * (el + held), "flops": 2.0 * c["A"] * c["k"]}
    A, n, k, E = c["A"], c["n"], c["k"], c["E"]
    busy = E * (1 - (1 - 1 / E) ** A)  # experts that have rows (even loads)
    return {"bytes": busy * n * k * held + A * (n + k) * el + (busy * n * el if c["bias"] else 0), "flops": 2.0 * A * n * k}


# ---------------------------------------------------------------------------------------------- 64 bits
def _scores64(c, logits):
    l = logits.double()
    if c["score"] == "sigmoid":
        return 1 / (1 + torch.exp(-l))
    return torch.exp(l - torch.logsumexp(l, 1, keepdim=True))


def _best64(key, count):
    """Indices of the `count` largest of each row, one after the other, the lowest of equals first."""
    key, out = key.clone(), []
    place = torch.arange(key.shape[1], device=DEV)
    for _ in range(count):
        top = key.amax(1, keepdim=True)
        i = torch.where(key == top, place, key.shape[1]).amin(1, keepdim=True)
        out.append(i)
        key.scatter_(1, i, -math.inf)
    return torch.cat(out, 1)


def _exact_route(c, s):
    T, E = c["T"], c["E"]
    p = _scores64(c, s["logits"])
    key = s["logits"].double() if s["bias"] is None else p + s["bias"].double()
    if c["groups"] > 1:
        by = p if c["best"] == 2 and s["bias"] is None else key
        size = E // c["groups"]
        values = []
        for q in range(c["groups"]):
            part = by[:, q * size:(q + 1) * size]
            first = _best64(part, min(c["best"], size))
            values.append(torch.gather(part, 1, first).sum(1))
        stay = _best64(torch.stack(values, 1), c["top"])
        member = (torch.arange(E, device=DEV) // size)[None, :]
        left = torch.zeros((T, E), dtype=torch.bool, device=DEV)
        for q in range(c["top"]):
            left |= member == stay[:, q:q + 1]
        key = torch.where(left, key, -math.inf)
    idx = _best64(key, c["k"])
    w = torch.gather(p, 1, idx)
    w = c["scale"] * (w / w.sum(1, keepdim=True) if c["renorm"] else w)
    return (idx.int(), w, p) if c["scores"] else (idx.int(), w)


def _exact_route_grad(c, s):
    """By the chain of its steps: weights from the chosen scores, scores from the logits."""
    p, g = _scores64(c, s["logits"]), s["dw"].double()
    dp = torch.zeros_like(p)
    if s["dscores"] is not None:
        dp += s["dscores"].double()
    sel = torch.gather(p, 1, s["idx"].long())
    total = sel.sum(1) if c["renorm"] else torch.ones_like(sel[:, 0])
    along = (g * sel).sum(1) / total ** 2 if c["renorm"] else torch.zeros_like(total)
    for j in range(c["k"]):
        dp.scatter_add_(1, s["idx"][:, j:j + 1].long(), (c["scale"] * (g[:, j] / total - along))[:, None])
    if c["score"] == "sigmoid":
        return dp * (p - p * p)
    return p * dp - p * (p * dp).sum(1, keepdim=True)


def _exact_combine(c, s):
    out = torch.zeros((c["T"], c["d"]), dtype=torch.float64, device=DEV)
    y, src = s["y"], s["src"]
    for lo in range(0, s["kept"], 1 << 14):
        a = src[lo:lo + (1 << 14)]
        v = y[lo:lo + a.numel()].double()
        if s["w"] is not None:
            v = v * s["w"].view(-1)[a].double()[:, None]
        out.index_add_(0, a // c["k"], v)
    return out


def _exact_combine_grad(c, s):
    dy = torch.zeros((c["T"] * c["k"], c["d"]), dtype=torch.float64, device=DEV)
    dw = torch.zeros((c["T"], c["k"]), dtype=torch.float64, device=DEV)
    position = s["position"].view(c["T"], c["k"]).long()
    for j in range(c["k"]):
        t = torch.nonzero(position[:, j] >= 0)[:, 0]
        at = position[t, j]
        v = s["dout"][t].double()
        dy[at] = s["w"][t, j].double()[:, None] * v
        dw[t, j] = torch.linalg.vecdot(s["y"][at].double(), v)
    return dy, dw


def _exact_q4(c, s):
    lo = s["offsets"].tolist()
    out = torch.zeros((c["A"], c["n"]), dtype=torch.float64, device=DEV)
    for e in range(c["E"]):
        if lo[e] == lo[e + 1]:
            continue
        q = s["q"][e].int()
        w = torch.empty((c["n"], c["k"]), dtype=torch.float64, device=DEV)
        w[:, 0::2], w[:, 1::2] = q % 16, q // 16
        w -= 8 if s["zero"] is None else s["zero"][e].double().repeat_interleave(c["group"], 1)
        w *= s["scale"][e].double().repeat_interleave(c["group"], 1)
        out[lo[e]:lo[e + 1]] = s["x"][lo[e]:lo[e + 1]].double() @ w.t()
        if s["bias"] is not None:
            out[lo[e]:lo[e + 1]] += s["bias"][e].double()
    return out


def _exact_quantise(c, s):
    """Of all sixteen values of a group, the nearest to each element; halfway: the one an even number of steps from zero."""
    dt, parts = DTYPE[c["dtype"]], []
    for rows in s["x"].split(max(1, (1 << 25) // c["k"])):
        v = rows.double().view(rows.shape[0], -1, c["group"])
        if c["zeros"]:
            low, high = v.amin(-1, keepdim=True).clamp(max=0), v.amax(-1, keepdim=True).clamp(min=0)
            step = ((high - low) / 15).float().to(dt).double()
            unit = torch.where(step == 0, 1.0, step)
            first = -torch.round(-low / unit).clamp(0, 15)
        else:
            step = (v.abs().amax(-1, keepdim=True) / 7).float().to(dt).double()
            unit, first = torch.where(step == 0, 1.0, step), torch.full_like(step, -8.0)
        t = v / unit
        down = torch.floor(t)
        up = (t - down > 0.5) | ((t - down == 0.5) & (down % 2 != 0))
        steps = torch.minimum(torch.maximum(down + up, first), first + 15)
        parts.append((steps * step).view(rows.shape))
    return torch.cat(parts)


EXACT = dict(route=_exact_route, route_grad=_exact_route_grad, combine=_exact_combine, combine_grad=_exact_combine_grad, q4=_exact_q4, quantise=_exact_quantise)


def exact(case, seed):
    return EXACT[case["kind"]](case, prepare(case, seed))
