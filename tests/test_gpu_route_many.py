"""The router of more than 2048 tokens, whose kernels give a token 16 or 32 lanes, against the definition in 64 bits,
and against the kernels of few tokens."""
import numpy as np
import pytest

from paper_2607_19539_amd import binding as B
from tests.gpu_helpers import log
from tests.test_gpu_route import SIG, ULP, grid_logits, reference, run_route
from tests.test_gpu_route_gradient import check, choices

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

T = 2051  # a last workgroup that is not full

CONFIGS = [
    # 16 lanes a token: whole groups of lanes; three and 64 groups that are none; runs of 1 to 16 experts.
    dict(experts=256, k=8, groups=8, top_groups=4, group_best=2, score=SIG, scale=2.5), dict(experts=256, k=8),
    dict(experts=256, k=16, groups=16, top_groups=3, score=SIG), dict(experts=48, k=6, groups=3, top_groups=2, group_best=2, score=SIG),
    dict(experts=128, k=8, groups=64, top_groups=5, group_best=2, score=SIG), dict(experts=160, k=6, groups=8, top_groups=3),
    dict(experts=1, k=1), dict(experts=8, k=2), dict(experts=100, k=16, renormalise=False, score=SIG),
    # 32 lanes: more than 256 experts, or 17 to 32 choices.
    dict(experts=384, k=8, score=SIG, scale=0.5), dict(experts=512, k=8, groups=16, top_groups=5, group_best=2, score=SIG),
    dict(experts=320, k=8, groups=40, top_groups=9), dict(experts=320, k=6, groups=5, top_groups=2, group_best=2),
    dict(experts=60, k=20, score=SIG), dict(experts=256, k=32, groups=4, top_groups=2), dict(experts=265, k=32),
    # 64 lanes.
    dict(experts=1000, k=3, groups=10, top_groups=4, score=SIG), dict(experts=64, k=40),
]
names = lambda c: "-".join(f"{k}{v}" for k, v in c.items())  # noqa: E731


def inputs(cfg):
    rng = np.random.default_rng(cfg.experts * 5 + cfg.k)
    l = grid_logits(rng, T, cfg.experts)
    if cfg.experts > 8:
        l[:, rng.random(cfg.experts) < 0.1] = -np.inf
        l[17] = -np.inf
        l[T - 1, 1:] = -np.inf
    bias = (0.05 * rng.standard_normal(cfg.experts)).astype(np.float32) if cfg.score == SIG else None
    return rng, l, bias


@pytest.mark.parametrize("bf", [False, True])
@pytest.mark.parametrize("c", CONFIGS, ids=names)
def test_route_of_many_tokens(c, bf):
    cfg = B.make_route_config(**c)
    log(f"route {c} T={T} bf16={bf}")
    _, l, bias = inputs(cfg)
    ids, w, s = run_route(cfg, l, bias, bf)
    rids, rw, rp, clear = reference(cfg, l, bias)
    assert clear.mean() > 0.2
    assert np.array_equal(ids[clear], rids[clear])
    assert np.all(np.abs(w[clear] - rw[clear]) <= 80 * ULP * rw[clear] + 1e-37)
    assert np.all(np.abs(s - rp) <= 4 * ULP * np.abs(rp) + 1e-37)


@pytest.mark.parametrize("bf", [False, True])
@pytest.mark.parametrize("c", CONFIGS, ids=names)
def test_a_token_is_routed_alike_among_few_and_many(c, bf):
    """Unclear tokens too: the same bits from every number of lanes."""
    cfg = B.make_route_config(**c)
    log(f"route few and many {c} bf16={bf}")
    _, l, bias = inputs(cfg)
    many = run_route(cfg, l, bias, bf)
    for first in (0, T - 300):
        for a, b in zip(many, run_route(cfg, l[first:first + 300], bias, bf)):
            assert np.array_equal(a[first:first + 300], b)


@pytest.mark.parametrize("bf", [False, True])
@pytest.mark.parametrize("dscores", [False, True])
@pytest.mark.parametrize("c", CONFIGS, ids=names)
def test_route_backward_of_many_tokens(c, dscores, bf):
    cfg = B.make_route_config(**c)
    log(f"route backward {c} T={T} dscores={dscores} bf16={bf}")
    rng, l, _ = inputs(cfg)
    ids = choices(rng, T, cfg.experts, cfg.k)
    if cfg.k > 1:
        ids[3, 1:] = -1
        ids[T - 2, 0] = cfg.experts
        ids[6, 1] = ids[6, 0]
    dw = rng.standard_normal((T, cfg.k)).astype(np.float32)
    check(cfg, l, ids, dw, rng.standard_normal(l.shape).astype(np.float32) if dscores else None, bf)
