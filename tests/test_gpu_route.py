"""moe_route and moe_route_backward against their definitions in 64 bits."""
import pytest
import torch

import many_experts_reference as R
import paper_2401_08383_amd as exf

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
BF, F32, INF = torch.bfloat16, torch.float32, float("inf")


def _logits(T, E, dt, seed, std=2.0):
    return (torch.randn(T, E, generator=torch.Generator().manual_seed(seed)) * std).to(dt)


def _masked(l, seed):
    """Experts taken out of a row, all of them in some rows; some rows' masks are the type's lowest value."""
    g = torch.Generator().manual_seed(seed)
    T, E = l.shape
    out = torch.rand(T, E, generator=g) < torch.rand(T, 1, generator=g)
    value = torch.where(torch.rand(T, 1, generator=g) < 0.5, -INF, torch.finfo(l.dtype).min).to(l.dtype)
    l = torch.where(out, value, l)
    l[0] = -INF
    l[T // 2] = torch.finfo(l.dtype).min
    l[T - 1, :] = -INF
    l[T - 1, E - 1] = 0.5
    return l


def _check(l, k, bias=None, **how):
    print(f"[case] route {tuple(l.shape)} {l.dtype} k={k} bias={bias is not None} {how}", flush=True)
    want_idx, want_w, want_s = R.route(l, k, bias, **how)
    idx, w, s = exf.moe_route(l.to(DEV), k, None if bias is None else bias.to(DEV), want_scores=True, **how)
    torch.cuda.synchronize()
    assert idx.dtype == torch.int32 and torch.equal(idx.cpu().long(), want_idx), torch.nonzero(idx.cpu().long() != want_idx)[:3]
    # exp: an argument rounded by half a unit of its size, and two units; a sum of as many as 512, a quotient, a product
    units = 2 * R.spread(l) + 40
    R.assert_close(w.cpu(), want_w, want_w.abs(), units, "weights")
    R.assert_close(s.cpu(), want_s, want_s, units, "scores")
    again = exf.moe_route(l.to(DEV), k, None if bias is None else bias.to(DEV), **how)
    assert torch.equal(again[0], idx) and torch.equal(again[1], w) and again[2] is None


SIZES = [(1, 1, 1), (3, 2, 2), (17, 7, 3), (65, 60, 6), (1, 64, 8), (33, 65, 16), (130, 128, 8), (9, 200, 5), (257, 256, 8), (5, 257, 16), (1000, 500, 10), (31, 512, 16), (4, 16, 16)]


@pytest.mark.parametrize("T,E,k", SIZES)
@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("score", [R.SOFTMAX, R.SIGMOID])
def test_sizes(T, E, k, dt, score):
    l = _logits(T, E, dt, T * E)
    _check(l, k, score=score)
    _check(l, k, score=score, renormalize=True, scale=2.5)
    bias = torch.randn(E, generator=torch.Generator().manual_seed(E)) * (0.1 if score else 0.5 / E)
    _check(l, k, bias, score=score, renormalize=True)


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("score", [R.SOFTMAX, R.SIGMOID])
@pytest.mark.parametrize("groups", [1, 4])
def test_the_best_ones_far_apart_in_one_stride(dt, score, groups):
    """Five to sixteen of the best experts at 4 i .. 4 i + 3 past multiples of 64: as a wavefront deals them out, one lane's."""
    r = torch.Generator().manual_seed(3)
    for E in (256, 512):
        l = _logits(96, E, dt, E).clamp(-3, 3)
        for t in range(96):
            first = 4 * int(torch.randint(0, 16 if E == 256 else 32, (1,), generator=r))
            at = (torch.arange(E) % (E // 4) >= first) & (torch.arange(E) % (E // 4) < first + 4)
            ids = torch.nonzero(at).flatten()
            ids = ids[torch.randperm(len(ids), generator=r)][:5 + t % 12]
            l[t, ids] = (4 + torch.randperm(64, generator=r)[:len(ids)] / 16).to(dt)
        bias = 0.01 * torch.randn(E, generator=r)
        for b in (None, bias):
            for best in (1, 2) if groups > 1 else (1,):
                _check(l, 8, b, score=score, groups=groups, top_groups=min(groups, 3), group_best=best, renormalize=True)


@pytest.mark.parametrize("E", [64, 256, 512])
def test_a_bias_that_begins_anywhere(E):
    """A layer's part of all layers' biases."""
    l = _logits(70, E, F32, E + 5)
    every = (torch.randn(4 * E + 8, generator=torch.Generator().manual_seed(E)) * 0.1).to(DEV)
    for at in (1, E + 2, 2 * E + 3, 3 * E + 4):
        idx, w, _ = exf.moe_route(l.to(DEV), 8, every[at:at + E], score=R.SIGMOID, groups=4, top_groups=2, group_best=2)
        same, same_w, _ = exf.moe_route(l.to(DEV), 8, every[at:at + E].clone(), score=R.SIGMOID, groups=4, top_groups=2, group_best=2)
        assert torch.equal(idx, same) and torch.equal(w, same_w)
    _check(l, 8, every[3:3 + E].cpu(), score=R.SIGMOID, groups=4, top_groups=2, group_best=2)


@pytest.mark.parametrize("E,groups,top,k", [(256, 8, 4, 8), (64, 4, 1, 16), (60, 5, 2, 7), (6, 6, 2, 2), (512, 64, 20, 16), (500, 10, 3, 9), (128, 2, 1, 1), (512, 2, 2, 4), (48, 16, 7, 6), (130, 13, 4, 8)])
@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("score", [R.SOFTMAX, R.SIGMOID])
@pytest.mark.parametrize("best", [1, 2])
def test_groups(E, groups, top, k, dt, score, best):
    l = _logits(70, E, dt, E + groups)
    how = dict(score=score, groups=groups, top_groups=top, group_best=best, renormalize=True)
    _check(l, k, **how)
    _check(l, k, torch.randn(E, generator=torch.Generator().manual_seed(E)) * (0.1 if score else 0.5 / E), **how)
    _check(_masked(l, E), k, **how)


@pytest.mark.parametrize("T,E,k", [(40, 64, 4), (50, 256, 16), (7, 9, 9), (20, 300, 8)])
@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("score", [R.SOFTMAX, R.SIGMOID])
def test_masks(T, E, k, dt, score):
    l = _masked(_logits(T, E, dt, T), T)
    for how in (dict(), dict(renormalize=True)):
        _check(l, k, score=score, **how)
        bias = torch.randn(E, generator=torch.Generator().manual_seed(E)) * (0.1 if score else 0.5 / E)
        bias[::3] = -INF
        bias[1] = float("nan")
        _check(l, k, bias, score=score, **how)


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("E,groups", [(64, 1), (256, 8), (512, 4), (60, 6)])
def test_ties_go_to_the_lowest(dt, E, groups):
    g = torch.Generator().manual_seed(E)
    l = torch.randint(0, 3, (90, E), generator=g).to(dt)  # few different values
    l[0] = 0.0
    l[1] = torch.where(torch.arange(E) % 2 == 0, 0.0, -0.0).to(dt)
    for score in (R.SOFTMAX, R.SIGMOID):
        _check(l, 8, score=score, groups=groups, top_groups=max(1, groups // 2), group_best=2)
        _check(l, 8, torch.zeros(E), score=score, groups=groups, top_groups=max(1, groups // 2), group_best=1, renormalize=True)


def _next_up(x, n=1):
    return (x.view(torch.int32) + n).view(torch.float32)


@pytest.mark.parametrize("score", [R.SOFTMAX, R.SIGMOID])
def test_keys_a_last_place_apart(score):
    """Neighbours in fp32, and sums of score and bias that are equal in fp32 and are not in 64 bits: the order is that of the exact keys."""
    E = 128
    g = torch.Generator().manual_seed(1)
    one = torch.full((E,), 1.25)
    l = torch.stack([_next_up(one, 0)[torch.randperm(E, generator=g)] for _ in range(60)])
    l = (l.view(torch.int32) + torch.randint(0, 12, l.shape, generator=g, dtype=torch.int32)).view(torch.float32)
    _check(l, 16, score=score)
    _check(l, 16, torch.full((E,), 3.0), score=score)
    _check(l, 16, torch.full((E,), 3.0), score=score, groups=8, top_groups=3, group_best=2)
    _check(l, 16, score=score, groups=8, top_groups=3, group_best=2)


@pytest.mark.parametrize("std", [30.0, 300.0])
@pytest.mark.parametrize("score", [R.SOFTMAX, R.SIGMOID])
def test_scores_that_underflow(std, score):
    """Renormalised weights of chosen experts whose scores are all tiny: the bias chooses them."""
    l = _logits(60, 96, F32, 4, std).clamp(max=-40.0) if score == R.SIGMOID else _logits(60, 96, F32, 4, std)
    bias = torch.zeros(96)
    bias[10:20] = 10.0 + torch.arange(10)
    for k in (1, 4, 8):
        _check(l, k, bias, score=score, renormalize=True)
        _check(l, k, bias, score=score)
        _check(l, k, score=score, renormalize=True)


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("score", [R.SOFTMAX, R.SIGMOID])
def test_rows_with_nan(dt, score):
    l = _logits(20, 100, dt, 8)
    fine = l.clone()
    l[3, 50], l[7, 0] = float("nan"), float("nan")
    l[9, 99] = INF
    idx, w, _ = (None if t is None else t.cpu() for t in exf.moe_route(l.to(DEV), 6, score=score, renormalize=True))
    want_idx, want_w, _ = R.route(fine, 6, score=score, renormalize=True)
    clean = torch.ones(20, dtype=torch.bool)
    clean[[3, 7, 9]] = False
    assert torch.equal(idx[clean].long(), want_idx[clean])
    assert torch.isnan(w[[3, 7]]).all() and bool(((idx >= -1) & (idx < 100)).all()) and torch.isfinite(w[clean]).all()
    assert 50 not in idx[3].tolist() and 0 not in idx[7].tolist() and idx[9, 0] == 99
    assert torch.isnan(w[9]).all() if score == R.SOFTMAX else torch.isfinite(w[9]).all()


def _check_gradient(l, idx, g, ds, score, renorm, scale):
    print(f"[case] route_backward {tuple(l.shape)} {l.dtype} k={idx.shape[1]} score={score} renorm={renorm} scale={scale} ds={None if ds is None else tuple(ds.shape)}", flush=True)
    ref, mag = R.route_gradient(l, idx, g, score, renorm, scale, ds)
    got = exf.moe_route_backward(g.to(DEV), l.to(DEV), idx.int().to(DEV), score=score, renormalize=renorm, scale=scale, dscores=None if ds is None else ds.to(DEV))
    assert got.dtype == l.dtype
    R.assert_close(got.cpu(), ref, mag, 4 * R.spread(l) + 80 + idx.shape[1], "dlogits")
    return got


@pytest.mark.parametrize("T,E,k", SIZES)
@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("score", [R.SOFTMAX, R.SIGMOID])
@pytest.mark.parametrize("renorm", [False, True])
def test_gradients(T, E, k, dt, score, renorm):
    r = torch.Generator().manual_seed(T + E)
    l = _logits(T, E, dt, T * E + 1)
    idx, g = R.route(l, k)[0], torch.randn(T, k, generator=r)
    for ds in (None, torch.randn(E, generator=r), torch.randn(T, E, generator=r)):
        _check_gradient(l, idx, g, ds, score, renorm, 1.0)
    _check_gradient(l, idx, g, None, score, renorm, -2.5)
    _check_gradient(l, idx, g, torch.randn(E, generator=r), score, renorm, 0.0)


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("score", [R.SOFTMAX, R.SIGMOID])
@pytest.mark.parametrize("renorm", [False, True])
def test_gradients_of_masked_rows_and_given_ids(dt, score, renorm):
    """Ids that are not the best, twice the same, of masked experts, outside the experts; NaN where nothing counts."""
    T, E, k = 80, 70, 5
    r = torch.Generator().manual_seed(2)
    l = _masked(_logits(T, E, dt, 6), 6)
    idx = torch.randint(0, E, (T, k), generator=r)
    idx[5:10, 3] = idx[5:10, 1]
    idx[11, :] = 7
    idx[12], idx[13, 2], idx[14, 0] = -1, E, 1 << 30
    g = torch.randn(T, k, generator=r)
    g[12], g[13, 2], g[14, 0] = float("nan"), INF, float("nan")
    got = _check_gradient(l, idx, g, None, score, renorm, 1.5)
    assert not got[0].any() and (renorm is False or not got[12].any())
    ds = torch.randn(T, E, generator=r)
    ds = torch.where(l == -INF, float("nan"), ds)
    _check_gradient(l, idx, g, ds, score, renorm, 1.5)


@pytest.mark.parametrize("std", [30.0, 300.0])
@pytest.mark.parametrize("score", [R.SOFTMAX, R.SIGMOID])
def test_gradients_where_scores_underflow(std, score):
    l = _logits(60, 96, F32, 5, std)
    if score == R.SIGMOID:
        l = l.clamp(max=-30.0)
    r = torch.Generator().manual_seed(3)
    idx, g = torch.stack([torch.randperm(96, generator=r)[:4] for _ in range(60)]), torch.randn(60, 4, generator=r)
    _check_gradient(l, idx, g, None, score, True, 1.0)
    _check_gradient(l, idx, g, torch.randn(96, generator=r), score, True, 1.0)


def test_rows_past_31_bits_of_bytes():
    """4.3 GB of logits: the last rows are routed as they are by themselves."""
    T, E = (1 << 22) + 5, 256
    l = torch.empty((T, E), device=DEV).normal_(generator=torch.Generator(DEV).manual_seed(1))
    idx, w, _ = exf.moe_route(l, 3, score=exf.EXF_SCORE_SIGMOID, renormalize=True)
    tail = l[-70:].clone()
    few = exf.moe_route(tail, 3, score=exf.EXF_SCORE_SIGMOID, renormalize=True)
    assert torch.equal(idx[-70:], few[0]) and torch.equal(w[-70:], few[1])
    dl = exf.moe_route_backward(w, l, idx, score=exf.EXF_SCORE_SIGMOID, renormalize=True)
    assert torch.equal(dl[-70:], exf.moe_route_backward(few[1], tail, few[0], score=exf.EXF_SCORE_SIGMOID, renormalize=True))


def test_no_tokens():
    l = torch.empty((0, 64), device=DEV)
    idx, w, s = exf.moe_route(l, 4, want_scores=True)
    assert idx.shape == w.shape == (0, 4) and s.shape == (0, 64) and exf.moe_route_backward(w, l, idx).shape == (0, 64)
