"""Routers by scores on the GPU against their definition in 64 bits (oracle/mx4.py).

Selected experts have to be equal: the inputs either leave a gap between scores that are chosen and not, or make exact ties.
Weights: exponential, quotient and sums of k scores in fp32, each at most an ulp or two off: 16 units of 2^-24.
"""
import numpy as np
import pytest
import torch

from oracle import mx4 as M
from paper_2605_17889_amd import binding as B

pytestmark = pytest.mark.gpu
TOL = 16 * 2.0 ** -24


def gapped_logits(rng, T, E, score, correction, groups, top_groups, group_best, k):
    """Logits whose scores are apart where the choice is made."""
    logits = (rng.standard_normal((T, E)) * 1.5).astype(np.float32)
    for _ in range(100):
        l = logits.astype(np.float64)
        s = 1 / (1 + np.exp(-l)) if score == "sigmoid" else np.exp(l - l.max(1, keepdims=True))
        if score == "softmax":
            s = s / s.sum(1, keepdims=True)
        c = s if correction is None else s + correction
        by = np.sort(c.reshape(T, groups, -1), axis=2)[:, :, ::-1][:, :, :group_best].sum(2)
        order = np.sort(by, axis=1)[:, ::-1]
        bad = np.zeros(T, bool)
        if top_groups < groups:
            bad |= order[:, top_groups - 1] - order[:, top_groups] < 1e-5 * np.abs(order[:, top_groups - 1])
            c = np.where((by >= order[:, top_groups - 1:top_groups]).repeat(E // groups, 1), c, -np.inf)
        best = np.sort(c, axis=1)[:, ::-1][:, :k + 1]
        with np.errstate(invalid="ignore"):
            bad |= (best[:, :-1] - best[:, 1:] < 1e-5 * np.abs(best[:, :-1])).any(1)
        if not bad.any():
            return logits
        logits[bad] = (rng.standard_normal((bad.sum(), E)) * 1.5).astype(np.float32)
    raise AssertionError("no such logits")


def run(logits, correction, k, score="sigmoid", groups=1, top_groups=1, group_best=2, renormalise=True, scale=1.0):
    T, E = logits.shape
    ctx = B.MoeContext(T, 512, 128, E, k)
    idx = torch.full((T + 1, k), -7, dtype=torch.int32, device="cuda")
    w = torch.full((T + 1, k), -7.0, device="cuda")
    sc = B.MoeScoring(score, groups, top_groups, group_best, renormalise, scale)
    print(f"route T={T} E={E} k={k} {score} groups={groups}/{top_groups} best={group_best}", flush=True)
    B.moe_route_scored_from_logits(ctx, torch.from_numpy(logits).cuda(),
                                   None if correction is None else torch.from_numpy(correction).cuda(), sc, T, idx[:T], w[:T])
    torch.cuda.synchronize()
    assert (idx[T] == -7).all() and (w[T] == -7).all()
    ctx.close()
    return idx[:T].cpu().numpy(), w[:T].double().cpu().numpy()


def check(logits, correction, k, **kw):
    idx, w = run(logits, correction, k, **kw)
    want_idx, want_w = M.route(logits, correction, k, **kw)
    assert np.array_equal(idx, want_idx), np.argwhere(idx != want_idx)[:5]
    assert (np.abs(w - want_w) <= TOL * np.abs(want_w) + 1e-45).all()


@pytest.mark.parametrize("score", ["sigmoid", "softmax"])
@pytest.mark.parametrize("T", [1, 5, 64, 4096, 4099])
@pytest.mark.parametrize("E,k,groups,top_groups,group_best", [
    (256, 8, 8, 4, 2), (64, 6, 1, 1, 1), (8, 2, 1, 1, 1), (160, 6, 8, 3, 1), (1, 1, 1, 1, 2), (96, 4, 3, 2, 2), (255, 5, 5, 4, 2),
    (252, 7, 9, 5, 2), (256, 4, 64, 9, 2), (128, 8, 32, 20, 1), (34, 3, 17, 8, 2), (256, 40, 2, 1, 2), (72, 64, 1, 1, 2)])
def test_scores_and_groups(score, T, E, k, groups, top_groups, group_best):
    rng = np.random.default_rng(E * 1000 + T + k)
    correction = (rng.standard_normal(E) * 0.05).astype(np.float32) if (E + T) % 2 else None
    logits = gapped_logits(rng, T, E, score, correction, groups, top_groups, group_best, k)
    check(logits, correction, k, score=score, groups=groups, top_groups=top_groups, group_best=group_best,
          renormalise=bool(T % 2), scale=2.5)


@pytest.mark.parametrize("T", [3, 4200])
@pytest.mark.parametrize("E,k,groups,top_groups", [(64, 6, 4, 2), (256, 8, 8, 4), (40, 5, 1, 1)])
def test_ties_go_to_the_lowest_index(T, E, k, groups, top_groups):
    """Few different logits: equal ones have equal scores, and groups equal sums, whatever the rounding."""
    rng = np.random.default_rng(T + E)
    logits = rng.integers(-1, 2, (T, E)).astype(np.float32)
    for score in ("sigmoid", "softmax"):
        check(logits, None, k, score=score, groups=groups, top_groups=top_groups, group_best=1)
        check(np.zeros((T, E), np.float32), None, k, score=score, groups=groups, top_groups=top_groups, group_best=2)


@pytest.mark.parametrize("T", [9, 4300])
def test_nan_infinite_and_masked(T):
    rng = np.random.default_rng(T)
    E, k = 64, 6
    logits = gapped_logits(rng, T, E, "sigmoid", None, 4, 2, 2, k)
    lowest = np.finfo(np.float32).min
    logits[0, :] = np.nan
    logits[1, :] = -np.inf
    logits[2, 5] = np.nan
    logits[3, 7] = np.inf
    logits[3, 20] = np.inf
    logits[4, ::2] = -np.inf
    logits[5, :] = lowest
    logits[6, 3:] = lowest
    logits[7, :60] = -np.inf
    for score in ("sigmoid", "softmax"):
        for groups, top in ((1, 1), (4, 2)):
            check(logits[:9], None, k, score=score, groups=groups, top_groups=top, group_best=1)
    mask = np.zeros(E, np.float32)
    mask[10:] = -np.inf
    mask[2] = np.nan
    for score in ("sigmoid", "softmax"):
        check(logits, mask, k, score=score)
        check(np.zeros((T, E), np.float32), mask, 12, score=score, groups=4, top_groups=3, group_best=2)
        check(np.zeros((T, E), np.float32), np.full(E, -np.inf, np.float32), k, score=score, groups=8, top_groups=2)
    check(np.full((T, E), -200.0, np.float32), None, k)            # scores of 0: their sum is


def test_results_do_not_depend_on_the_number_of_tokens():
    rng = np.random.default_rng(1)
    logits = (rng.standard_normal((5000, 256)) * 2).astype(np.float32)
    for score in ("sigmoid", "softmax"):
        kw = dict(score=score, groups=8, top_groups=4, group_best=2, renormalise=True, scale=1.5)
        for k in (8, 40):
            many, few = run(logits, None, k, **kw), run(logits[1000:1100], None, k, **kw)
            assert np.array_equal(many[0][1000:1100], few[0]) and np.array_equal(many[1][1000:1100], few[1])


@pytest.mark.parametrize("E,k", [(8, 2), (64, 6), (256, 8)])
def test_router_from_tokens(E, k):
    """x and the router's matrix: moe_route's logits, then the selection from them."""
    g = torch.Generator(device="cuda").manual_seed(E)
    for T in (1, 33, 600):
        x = torch.randn(T, 1024, generator=g, device="cuda").to(torch.bfloat16)
        w = torch.randn(1024, E, generator=g, device="cuda") * 0.05
        bias = torch.randn(E, generator=g, device="cuda") * 0.1
        corr = torch.randn(E, generator=g, device="cuda") * 0.1
        ctx = B.MoeContext(T, 1024, 128, E, k)
        new = lambda: (torch.empty((T, k), dtype=torch.int32, device="cuda"), torch.empty((T, k), device="cuda"))
        logits = torch.empty((T, E), device="cuda")
        want_logits = torch.empty((T, E), device="cuda")
        sc = B.MoeScoring("sigmoid", groups=4, top_groups=2, renormalise=True, scale=2.0)
        a, b, c, d = new(), new(), new(), new()
        B.moe_route(ctx, x, w, bias, T, *d, logits_out=want_logits)
        B.moe_route_scored(ctx, x, w, bias, corr, sc, T, *a, logits_out=logits)
        B.moe_route_scored(ctx, x, w, bias, corr, sc, T, *b)
        B.moe_route_scored_from_logits(ctx, logits, corr, sc, T, *c)
        assert torch.equal(logits, want_logits)
        for got in (b, c):
            assert torch.equal(a[0], got[0]) and torch.equal(a[1], got[1])
        ctx.close()
