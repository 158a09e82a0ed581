"""The router's gradient where a score, or the sum of the chosen ones, is nearly nothing.

The 64-bit formula takes 1 - p as 1 / (1 + e^l), which loses nothing where p is near 1, and the share of a choice,
p / (sum of the chosen p), before anything is multiplied by it.
"""
import numpy as np
import pytest

from paper_2607_19539_amd import binding as B
from tests.gpu_helpers import log
from tests.test_gpu_route import SIG, SOFT, ULP, run_backward, score64

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

TINY = 2.0 ** -148  # two roundings to the subnormal fp32 grid


def gradient64(cfg, l, ids, dw, ds):
    """The gradient in 64 bits, the magnitude of its terms, and what the scores' last bits are worth in it where
    they are subnormal (a score is then within TINY, however small it is)."""
    T, E = l.shape
    p = score64(l, cfg.score)
    with np.errstate(over="ignore"):
        rest = 1.0 / (1.0 + np.exp(l.astype(np.float64)))
    u = np.zeros((T, E)) if ds is None else p * ds.astype(np.float64)
    mag, grain = np.abs(u), np.zeros((T, E))
    for t in range(T):
        have = (ids[t] >= 0) & (ids[t] < E)
        i, d = ids[t][have], dw[t][have].astype(np.float64)
        share, mean, amean, total = p[t, i], 0.0, 0.0, 1.0
        if cfg.renormalise:
            total = share.sum()
            share = share / total if total > 0 else share * 0
            mean, amean = (d * share).sum(), (np.abs(d) * share).sum()
        np.add.at(u[t], i, cfg.scale * share * (d - mean))
        np.add.at(mag[t], i, cfg.scale * share * (np.abs(d) + amean))
        if total > 0:
            np.add.at(grain[t], i, cfg.scale * (np.abs(d) + amean) * (2 + len(i)) * TINY / total)
    if cfg.score == SIG:
        return u * rest, mag * rest, grain * rest
    more = grain + p * grain.sum(1, keepdims=True)
    return u - p * u.sum(1, keepdims=True), mag + p * mag.sum(1, keepdims=True), more


def check(cfg, l, ids, dw, ds, bf=False):
    got = run_backward(cfg, l, ids, dw, ds, bf)
    want, mag, grain = gradient64(cfg, l, ids, dw, ds)
    assert np.isfinite(got).all()
    # Sums of at most 1024 terms in a tree over lanes, factors within a few units each.
    assert np.all(np.abs(got - want) <= 200 * ULP * mag + grain + (2.0 ** -8 * np.abs(want) if bf else 0) + 1e-37)


def choices(rng, T, E, k):
    return np.stack([rng.permutation(E)[:k] for _ in range(T)]).astype(np.int32)


@pytest.mark.parametrize("bf", [False, True])
@pytest.mark.parametrize("dscores", [False, True])
@pytest.mark.parametrize("T", [37, 2061])
@pytest.mark.parametrize("c", [dict(experts=16, k=4, scale=2.5), dict(experts=16, k=4, renormalise=False),
                               dict(experts=100, k=6), dict(experts=384, k=8, renormalise=False, scale=0.5)],
                         ids=lambda c: "-".join(f"{k}{v}" for k, v in c.items()))
def test_sigmoid_scores_near_one_and_near_nothing(c, T, dscores, bf):
    """Logits of 8 to 30 and of -30 to -8: the derivative p (1 - p) keeps its relative accuracy."""
    cfg = B.make_route_config(score=SIG, **c)
    log(f"route backward, steep logits {c} T={T} dscores={dscores} bf16={bf}")
    rng = np.random.default_rng(cfg.experts + T + dscores)
    l = (rng.uniform(8, 30, (T, cfg.experts)) * rng.choice([-1, 1], (T, cfg.experts))).astype(np.float32)
    l = torch.from_numpy(l).to(torch.bfloat16).float().numpy()
    dw = rng.standard_normal((T, cfg.k)).astype(np.float32)
    ds = rng.standard_normal((T, cfg.experts)).astype(np.float32) if dscores else None
    check(cfg, l, choices(rng, T, cfg.experts, cfg.k), dw, ds, bf)


def test_sigmoid_scores_at_the_ends():
    """The gradient is 0 and not NaN where the score is 0 or 1 (an infinity, or e^-l that overflows)."""
    cfg = B.make_route_config(8, 2, score=SIG, renormalise=False)
    l = np.array([[np.inf, -np.inf, 200, -200, 104, -104, 89, -89]], np.float32)
    for j in range(0, 8, 2):
        got = run_backward(cfg, l, np.array([[j, j + 1]], np.int32), np.ones((1, 2), np.float32), np.ones((1, 8), np.float32))
        assert np.all(np.abs(got) < 1e-37)


@pytest.mark.parametrize("dscores", [False, True])
@pytest.mark.parametrize("T", [29, 2061])
@pytest.mark.parametrize("scale", [2.5, 50.0])
@pytest.mark.parametrize("k", [1, 3])
@pytest.mark.parametrize("score", [SOFT, SIG])
def test_chosen_scores_that_sum_to_a_subnormal(score, k, scale, T, dscores):
    """A bias can steer a token to experts whose scores are below 2^-126; scale over their sum overflows (three
    sigmoid scores by 2.5 aside), the shares do not."""
    cfg = B.make_route_config(16, k, score=score, scale=scale)
    log(f"route backward, tiny scores {score} k={k} T={T} dscores={dscores}")
    rng = np.random.default_rng(T + k)
    ids = choices(rng, T, 16, k)
    if score == SOFT:
        # One expert, not a chosen one, has nearly all of the sum; the chosen have e^-92 to e^-90 of it.
        l = rng.uniform(-4, -2, (T, 16))
        np.put_along_axis(l, ids.astype(np.int64), rng.uniform(-92, -90, (T, k)), 1)
        for t in range(T):
            l[t, np.setdiff1d(np.arange(16), ids[t])[0]] = 0.0
    else:
        l = rng.uniform(-3, 3, (T, 16))
        np.put_along_axis(l, ids.astype(np.int64), rng.uniform(-88.5, -87.5, (T, k)), 1)
    l = l.astype(np.float32)
    p = np.take_along_axis(score64(l, score), ids.astype(np.int64), 1).sum(1)
    assert np.all((p > 1e-41) & (p < 4e-38)) and ((p < scale / 3.4e38).any() or (score, k, scale) == (SIG, 3, 2.5))
    dw = rng.standard_normal((T, k)).astype(np.float32)
    ds = rng.standard_normal((T, 16)).astype(np.float32) if dscores else None
    check(cfg, l, ids, dw, ds)
