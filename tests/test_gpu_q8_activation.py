"""The gated product's activation silu(g) * u over the whole range of g and u, against the fp32 formula: the
exponential e^-g is infinite from g = -88.73 down, where silu is -0 (NaN for g = -infinity, as -infinity over infinity is).

One product of 1 and 1 makes each sum, so that g and u are the weights' scales.  Tolerance as for the other gated
products, and the bf16 grid below 2^-126."""
import numpy as np
import pytest

from paper_2607_19539_amd import binding as B
from tests.gpu_helpers import log
from tests.test_gpu_q8 import KINDS, REL, run_kind

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

INF, NAN = np.float32(np.inf), np.float32(np.nan)
G = [0.0, 1e-30, -1e-30, 1e-3, -1e-3, 1.0, -1.0, 20.0, -20.0, 60.0, -60.0, 80.0, -80.0, 87.0, -87.0, -87.5, -88.0, -88.5, -88.7,
     88.7, 100.0, -100.0, 127.0, 130.0, 1e4, -1e4, 3e20, -3e20, 2.3e38, 2.5e38, 3.3e38, -2.3e38, -2.5e38, -3.3e38, INF, -INF, NAN]
U = [0.0, 1.0, -1.0, 1e-3, -1e-3, 1e20, -1e20, 1e38, -1e38, 3e38, 1e-36, INF, -INF, NAN]


def silu_times(g, u):
    """The formula with fp32's range of e^-g, otherwise in 64 bits."""
    g, u = g.astype(np.float64), u.astype(np.float64)
    with np.errstate(all="ignore"):
        e = np.exp(-g)
        e[e > float(np.finfo(np.float32).max)] = np.inf
        return g / (1 + e) * u


@pytest.mark.parametrize("rows", [1, 40, 300])
@pytest.mark.parametrize("kind", KINDS)
def test_every_gate_and_factor(kind, rows):
    log(f"q8 activation {kind} rows={rows}")
    g, u = (a.reshape(-1) for a in np.meshgrid(np.array(G, np.float32), np.array(U, np.float32), indexing="ij"))
    pad = -len(g) % 8
    g, u = np.concatenate([g, np.ones(pad, np.float32)]), np.concatenate([u, np.ones(pad, np.float32)])
    N, K = len(g), 16
    x, w = np.zeros((rows, K), np.int8), np.zeros((2, 1, N, K), np.int8)
    x[:, 3] = w[..., 3] = 1
    got = run_kind(kind, x, np.ones(rows, np.float32), w, np.stack([g, u])[:, None], None, None, rows, True)
    want = silu_times(g, u)
    assert np.array_equal(got, np.broadcast_to(got[0], got.shape), equal_nan=True)
    got = got[0]
    bad = np.isnan(got) != np.isnan(want)
    assert not bad.any(), [(float(a), float(b), float(c), float(d)) for a, b, c, d in zip(g[bad], u[bad], got[bad], want[bad])]
    largest = float(torch.finfo(torch.bfloat16).max) * (1 + 2.0 ** -9)  # from here on bf16 rounds to infinity
    want = np.where(np.abs(want) >= largest, np.copysign(np.inf, want), want)
    fine = np.isfinite(want)
    bad = np.zeros(N, bool)
    bad[~fine] = (got != want)[~fine] & ~np.isnan(want[~fine])
    bad[fine] = ~(np.abs(got[fine] - want[fine]) <= REL * np.abs(want[fine]) + 2.0 ** -133)
    assert not bad.any(), [(float(a), float(b), float(c), float(d)) for a, b, c, d in zip(g[bad], u[bad], got[bad], want[bad])]
