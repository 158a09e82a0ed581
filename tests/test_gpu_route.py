"""The router and its gradient against the definition in 64 bits.

Choices are compared where they are clear: a token takes part if no two of its picks (and of its groups'
values) that differ at all differ by less than 1e-6 of their terms, some times what fp32 scores and their sums
can be off by.  Equal logits with equal biases are exact ties and stay in.  Weights: a score is within 4 units of
2^-24, their sum of up to 64 terms within 70.
"""
import numpy as np
import pytest

from paper_2607_19539_amd import binding as B
from tests.gpu_helpers import log

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

ULP, GAP = 2.0 ** -24, 1e-6
SIG, SOFT = B.MOE_SCORE_SIGMOID, B.MOE_SCORE_SOFTMAX


def score64(l, kind):
    l = l.astype(np.float64)
    with np.errstate(all="ignore"):
        if kind == SIG:
            return 1.0 / (1.0 + np.exp(-l))
        m = l.max(1, keepdims=True)
        e = np.exp(l - np.where(m == -np.inf, 0.0, m))
        s = e.sum(1, keepdims=True)
        return np.where(s > 0, e / np.where(s > 0, s, 1.0), 0.0)


def reference(cfg, l, bias):
    """ids, weights, scores and which tokens are clear; one token after another."""
    T, E = l.shape
    p = score64(l, cfg.score)
    pick = p + (0.0 if bias is None else bias.astype(np.float64))
    pick = np.where(l == -np.inf, -np.inf, pick)
    ids, w, clear = np.full((T, cfg.k), -1, np.int32), np.zeros((T, cfg.k)), np.ones(T, bool)
    size = E // cfg.groups

    mags = p + (0.0 if bias is None else np.abs(bias))

    def unclear(v, mag):
        at = np.argsort(v[np.isfinite(v)])
        v, mag = v[np.isfinite(v)][at], mag[np.isfinite(v)][at]
        d = np.diff(v)
        return bool(((d > 0) & (d < GAP * np.maximum(mag[1:], mag[:-1]))).any())

    for t in range(T):
        v = pick[t].copy()
        # Equal logits with another bias, or another logit that rounds to the same pick, are no ties in fp32.
        clear[t] = not unclear(v, mags[t])
        if cfg.groups > 1:
            g = np.sort(v.reshape(cfg.groups, size), 1)[:, ::-1][:, :cfg.group_best].sum(1)
            clear[t] &= not unclear(g, np.sort(mags[t].reshape(cfg.groups, size), 1)[:, ::-1][:, :cfg.group_best].sum(1))
            keep = np.argsort(-g, kind="stable")[:cfg.top_groups]
            mask = np.isin(np.arange(E) // size, keep)
            v = np.where(mask, v, -np.inf)
        order = np.argsort(-v, kind="stable")[:cfg.k]
        order = order[v[order] > -np.inf]
        ids[t, :len(order)] = order
        c = p[t, order]
        if cfg.renormalise:
            c = c / c.sum() if c.sum() > 0 else c * 0
        w[t, :len(order)] = c * cfg.scale
    return ids, w, p, clear


def dev(a, bf=False):
    t = torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).cuda()
    return t.to(torch.bfloat16) if bf else t


def run_route(cfg, l, bias, bf=False, scores=True, stream=None):
    T, E = l.shape
    ids = torch.full((T, cfg.k), -99, dtype=torch.int32, device="cuda")
    w = torch.full((T, cfg.k), -99.0, device="cuda")
    s = torch.full((T, E), -99.0, device="cuda") if scores else None
    B.moe_route(cfg, dev(l, bf), ids, w, bias=None if bias is None else dev(bias), scores=s, stream=stream)
    torch.cuda.synchronize()
    return ids.cpu().numpy(), w.cpu().numpy(), None if s is None else s.cpu().numpy()


def grid_logits(rng, T, E, step=2.0 ** -4):
    """Logits on a grid that bf16 holds, so that there are ties."""
    return (np.round(rng.standard_normal((T, E)) * 1.5 / step) * step).astype(np.float32)


CONFIGS = [
    dict(experts=8, k=2), dict(experts=8, k=8), dict(experts=1, k=1), dict(experts=2, k=2, score=SIG),
    dict(experts=60, k=4, renormalise=False), dict(experts=64, k=6, score=SIG, renormalise=False, scale=2.5),
    dict(experts=65, k=7, score=SIG), dict(experts=64, k=64), dict(experts=100, k=64, score=SIG, scale=0.5),
    dict(experts=256, k=8, groups=8, top_groups=4, group_best=2, score=SIG, scale=2.5),
    dict(experts=256, k=8, groups=8, top_groups=1, group_best=1), dict(experts=160, k=6, groups=8, top_groups=3),
    dict(experts=128, k=8, groups=64, top_groups=5, group_best=2, score=SIG),
    dict(experts=48, k=20, groups=3, top_groups=1, group_best=2, score=SIG),   # fewer experts than choices
    dict(experts=384, k=8), dict(experts=513, k=9, score=SIG), dict(experts=1024, k=16, groups=4, top_groups=2),
    dict(experts=1000, k=3, groups=10, top_groups=10, score=SIG),
]


@pytest.mark.parametrize("bf", [False, True])
@pytest.mark.parametrize("T", [1, 7, 130])
@pytest.mark.parametrize("c", CONFIGS, ids=lambda c: "-".join(f"{k}{v}" for k, v in c.items()))
def test_route(c, T, bf):
    cfg = B.make_route_config(**c)
    log(f"route {c} T={T} bf16={bf}")
    rng = np.random.default_rng(cfg.experts * 7 + T)
    l = grid_logits(rng, T, cfg.experts)
    if cfg.experts > 8:
        l[:, rng.random(cfg.experts) < 0.1] = -np.inf
    bias = (0.05 * rng.standard_normal(cfg.experts)).astype(np.float32) if cfg.score == SIG else None
    ids, w, s = run_route(cfg, l, bias, bf)
    rids, rw, rp, clear = reference(cfg, l, bias)
    assert clear.mean() > 0.2 or T < 8 or bias is not None
    assert np.array_equal(ids[clear], rids[clear])
    assert np.all(np.abs(w[clear] - rw[clear]) <= 80 * ULP * rw[clear] + 1e-37)
    assert np.all(np.abs(s - rp) <= 4 * ULP * np.abs(rp) + 1e-37)


@pytest.mark.parametrize("score", [SOFT, SIG])
def test_route_without_scores_or_with_many_tokens(score):
    cfg = B.make_route_config(64, 6, score=score)
    rng = np.random.default_rng(3)
    l = grid_logits(rng, 5000, 64)
    ids, w, _ = run_route(cfg, l, None, scores=False)
    rids, rw, _, clear = reference(cfg, l, None)
    assert clear.mean() > 0.5
    assert np.array_equal(ids[clear], rids[clear])
    assert np.all(np.abs(w[clear] - rw[clear]) <= 80 * ULP * rw[clear])


@pytest.mark.parametrize("score", [SOFT, SIG])
@pytest.mark.parametrize("E", [8, 100, 256])
def test_route_odd_rows(E, score):
    """Tokens with no expert left, with the type's lowest value as a mask, with one expert, with NaN."""
    cfg = B.make_route_config(E, 4, score=score)
    low = np.finfo(np.float32).min
    l = np.zeros((7, E), np.float32)
    l[0] = -np.inf
    l[1] = low
    l[2], l[2, 5] = -np.inf, 1.0
    l[3], l[3, 6], l[3, 2] = low, 1.0, 1.0
    l[4, 3] = np.nan
    l[5, 3] = np.inf
    ids, w, s = run_route(cfg, l, None)
    assert ids[0].tolist() == [-1] * 4 and w[0].tolist() == [0] * 4 and float(np.abs(s[0]).max()) == 0
    assert ids[1].tolist() == [0, 1, 2, 3]
    assert w[1].tolist() == ([0.25] * 4 if score == SOFT else [0.0] * 4)
    assert ids[2].tolist() == [5, -1, -1, -1] and w[2].tolist() == [1, 0, 0, 0]
    assert ids[3].tolist() == [2, 6, 0, 1] and w[3].tolist() == [0.5, 0.5, 0, 0]
    assert ids[4].tolist() == [0, 1, 2, 3] and np.isnan(w[4]).all()
    if score == SOFT:
        assert ids[5].tolist() == [0, 1, 2, 3] and np.isnan(w[5]).all()
    else:
        assert ids[5].tolist() == [3, 0, 1, 2] and np.all(np.abs(w[5] - [0.4, 0.2, 0.2, 0.2]) < 1e-6)
    assert ids[6].tolist() == [0, 1, 2, 3] and np.all(w[6] == 0.25)


def test_route_odd_biases():
    cfg = B.make_route_config(8, 3, score=SIG, groups=4, top_groups=4)
    l = np.zeros((2, 8), np.float32)
    l[1, 4] = -np.inf
    bias = np.zeros(8, np.float32)
    bias[7], bias[0] = np.inf, -np.inf
    ids, w, _ = run_route(cfg, l, bias)
    assert ids.tolist() == [[7, 1, 2]] * 2 and np.all(np.abs(w - 1 / 3) < 1e-6)
    bias[5] = np.nan
    ids, w, _ = run_route(cfg, l, bias)
    assert ids.tolist() == [[0, 1, 2]] * 2 and np.isnan(w).all()


def loss64(cfg, l, ids, dw, ds):
    p = score64(l, cfg.score)
    have = (ids >= 0) & (ids < cfg.experts)
    v = np.where(have, np.take_along_axis(p, np.where(have, ids, 0), 1), 0.0)
    if cfg.renormalise:
        v = v / v.sum(1, keepdims=True)
    out = (v * cfg.scale * np.where(have, dw, 0.0)).sum(1)
    return out + (p * ds).sum(1) if ds is not None else out


def gradient64(cfg, l, ids, dw, ds):
    """The formula in 64 bits, and the magnitude of its terms."""
    T, E = l.shape
    p = score64(l, cfg.score)
    g = np.zeros((T, E)) if ds is None else ds.astype(np.float64).copy()
    mag = np.abs(g)
    for t in range(T):
        have = (ids[t] >= 0) & (ids[t] < E)
        i, d = ids[t][have], dw[t][have].astype(np.float64)
        v = p[t, i]
        total, mean, amean = 1.0, 0.0, 0.0
        if cfg.renormalise:
            total = v.sum()
            mean, amean = (d * v).sum() / total, (np.abs(d) * v).sum() / total
        np.add.at(g[t], i, cfg.scale / total * (d - mean))
        np.add.at(mag[t], i, cfg.scale / total * (np.abs(d) + amean))
    if cfg.score == SIG:
        return g * p * (1 - p), mag * p
    return p * (g - (g * p).sum(1, keepdims=True)), p * (mag + (mag * p).sum(1, keepdims=True))


def run_backward(cfg, l, ids, dw, ds, bf=False):
    out = torch.full(l.shape, -99.0, dtype=torch.bfloat16 if bf else torch.float32, device="cuda")
    B.moe_route_backward(cfg, dev(l, bf), torch.from_numpy(ids).cuda(), dev(dw), out,
                         dscores=None if ds is None else dev(ds))
    torch.cuda.synchronize()
    return out.float().cpu().numpy().astype(np.float64)


@pytest.mark.parametrize("bf", [False, True])
@pytest.mark.parametrize("dscores", [False, True])
@pytest.mark.parametrize("c", CONFIGS, ids=lambda c: "-".join(f"{k}{v}" for k, v in c.items()))
def test_route_backward(c, dscores, bf):
    cfg = B.make_route_config(**c)
    log(f"route backward {c} dscores={dscores} bf16={bf}")
    rng = np.random.default_rng(cfg.experts * 3 + cfg.k)
    T, E = 37, cfg.experts
    l = grid_logits(rng, T, E)
    ids = np.stack([rng.permutation(E)[:cfg.k] for _ in range(T)]).astype(np.int32)
    if cfg.k > 1:
        ids[3, 1:] = -1
        ids[5, 0] = E
        ids[6, 1] = ids[6, 0]
    if E > 8:
        l[9, ids[9, cfg.k - 1]] = -np.inf
    dw = rng.standard_normal((T, cfg.k)).astype(np.float32)
    ds = rng.standard_normal((T, E)).astype(np.float32) if dscores else None
    got = run_backward(cfg, l, ids, dw, ds, bf)
    want, mag = gradient64(cfg, l, ids, dw, ds)
    # Sums of at most 1024 terms in a tree over lanes, factors within a few units each.
    assert np.all(np.abs(got - want) <= 200 * ULP * mag + (2.0 ** -8 * np.abs(want) if bf else 0) + 1e-37)


@pytest.mark.parametrize("c", [dict(experts=12, k=3), dict(experts=12, k=3, renormalise=False, scale=1.7),
                               dict(experts=12, k=3, score=SIG, scale=2.5), dict(experts=12, k=3, score=SIG, renormalise=False)])
def test_route_backward_against_differences(c):
    """Central differences with a step of 1e-5 in 64 bits: within 1e-9 of the gradient; the kernel's fp32
    within 1e-6 of the size of its terms."""
    cfg = B.make_route_config(**c)
    rng = np.random.default_rng(11)
    T, E = 4, 12
    l = rng.standard_normal((T, E)).astype(np.float32)
    ids = np.stack([rng.permutation(E)[:3] for _ in range(T)]).astype(np.int32)
    dw, ds = rng.standard_normal((T, 3)).astype(np.float32), rng.standard_normal((T, E)).astype(np.float32)
    got = run_backward(cfg, l, ids, dw, ds)
    step = 1e-5
    for e in range(E):
        d = np.zeros((T, E))
        d[:, e] = step
        want = (loss64(cfg, l.astype(np.float64) + d, ids, dw, ds) - loss64(cfg, l.astype(np.float64) - d, ids, dw, ds)) / (2 * step)
        assert np.all(np.abs(got[:, e] - want) <= 1e-5)


def test_route_backward_of_tokens_without_experts():
    """No expert chosen, or chosen scores of 0: no gradient, and none of it NaN."""
    for score in (SOFT, SIG):
        cfg = B.make_route_config(8, 2, score=score)
        l = np.zeros((3, 8), np.float32)
        l[0] = -np.inf
        l[1], l[1, 0] = np.finfo(np.float32).min, 0.0
        ids = np.array([[-1, -1], [3, 4], [-1, 2]], np.int32)
        got = run_backward(cfg, l, ids, np.ones((3, 2), np.float32), None)
        assert np.all(got[:2] == 0) and np.all(np.abs(got[2]) < 1e-6)


def test_route_of_no_tokens():
    cfg = B.make_route_config(8, 2)
    B.moe_route(cfg, torch.zeros((0, 8), device="cuda"), torch.zeros((0, 2), dtype=torch.int32, device="cuda"),
                torch.zeros((0, 2), device="cuda"))


def test_route_on_another_stream():
    cfg = B.make_route_config(64, 6)
    l = grid_logits(np.random.default_rng(5), 300, 64)
    a = run_route(cfg, l, None)
    b = run_route(cfg, l, None, stream=torch.cuda.Stream())
    assert all(np.array_equal(x, y) for x, y in zip(a, b))
