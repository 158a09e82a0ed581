"""The gated activation and its gradient against 64 bits.

s is within 5 2^-24 of itself (an exponential and a reciprocal of one fp32 ulp each, an addition), silu(g) u within
8 2^-24.  1 - s is off by 6 2^-24 and is multiplied by g, so 1 + g (1 - s) is off by 8 (|g| + 2) 2^-24.  Results are
rounded to bf16 (2^-8).  s is 0 below g = -88.7, where it is at most 2^-127, and so are values below fp32's normal ones.
"""
import numpy as np
import pytest

from paper_2607_19539_amd import binding as B
from tests.gpu_helpers import log

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

SMALL = 2.0 ** -117


def formulas(g, u, da):
    with np.errstate(over="ignore", invalid="ignore"):
        s = 1.0 / (1.0 + np.exp(-g))
        c = 1.0 / (1.0 + np.exp(g))
        return s, g * s * u, da * u * s * (1.0 + g * c), da * g * s


def near(got, want, tol):
    assert np.array_equal(np.isnan(got), np.isnan(want))
    both = np.isfinite(want) & np.isfinite(got)
    # A value within rounding of bf16's largest may become an infinity.
    edge = ~both & ~np.isnan(want)
    assert np.all((np.abs(want[edge]) > 3.3e38) & (np.sign(got[edge]) == np.sign(want[edge])))
    off = np.abs(got - want)[both] - 2.0 ** -8 * np.abs(want)[both] - tol[both]
    assert off.size == 0 or off.max() <= 0, float(off.max())


def run(g, u, da, offsets=None, in_place=False):
    dev = lambda a: torch.from_numpy(a.astype(np.float32)).to(torch.bfloat16).cuda()  # noqa: E731
    gu, dact = dev(np.concatenate([g, u], 1)), dev(da)
    F = g.shape[1]
    act, again = torch.full_like(dact, 7.0), torch.full_like(dact, 7.0)
    off = None if offsets is None else torch.tensor(offsets, dtype=torch.int32, device="cuda")
    B.moe_gate(gu, act, expert_offsets=off)
    dgu = gu if in_place else torch.full_like(gu, 7.0)
    before = gu.double().cpu().numpy()
    B.moe_gate_backward(gu, dact, dgu, act=again, expert_offsets=off)
    torch.cuda.synchronize()
    assert torch.equal(act, again) or bool((act.isnan() == again.isnan()).all())
    out = [t.double().cpu().numpy() for t in (act, dgu)]
    return out[0], out[1][:, :F], out[1][:, F:], before[:, :F], before[:, F:], dact.double().cpu().numpy()


def check(act, dg, du, g, u, da, rows=None):
    g, u, da = g[:rows], u[:rows], da[:rows]
    s, a, wg, wu = formulas(g, u, da)
    with np.errstate(over="ignore", invalid="ignore"):
        finite = np.isfinite(g) & np.isfinite(u) & np.isfinite(da)
        size = np.where(finite, np.abs(da * u), 0.0)
        near(act[:rows], a, 8 * 2.0 ** -24 * np.abs(np.where(np.isfinite(a), a, 0)) + SMALL * (1 + np.where(finite, np.abs(u), 0)))
        near(dg[:rows], wg, size * np.where(finite, s * 8 * (np.minimum(np.abs(g), 128) + 2) * 2.0 ** -24, 0) + SMALL * (1 + size))
        near(du[:rows], wu, 8 * 2.0 ** -24 * np.abs(np.where(np.isfinite(wu), wu, 0)) + SMALL * (1 + np.where(finite, np.abs(da), 0)))


@pytest.mark.parametrize("rows,F", [(1, 8), (1, 1408), (3, 24), (7, 40), (64, 512), (257, 576), (1000, 88), (33, 2048), (2, 65536)])
def test_gate(rows, F):
    log(f"gate {rows} x {F}")
    rng = np.random.default_rng(rows + F)
    g, u, da = (rng.standard_normal((rows, F)) * s for s in (4.0, 2.0, 0.1))
    check(*run(g, u, da))
    check(*run(g, u, da, in_place=True))


def test_the_whole_range():
    """Every bf16 value of g, with u and da of very different sizes."""
    bits = np.arange(65536, dtype=np.uint16)
    g = torch.from_numpy(bits.view(np.int16)).view(torch.bfloat16).double().numpy().reshape(64, 1024)
    for u, da in ((1.0, 1.0), (-3.0, 1e-3), (1e30, 1e-30), (1e-30, 1e20)):
        check(*run(g, np.full_like(g, u), np.full_like(g, da)))


def test_rows_past_the_last_are_left_alone():
    rng = np.random.default_rng(1)
    g, u, da = (rng.standard_normal((50, 64)) for _ in range(3))
    g[30:] = np.nan
    act, dg, du, *rest = run(g, u, da, offsets=[0, 10, 10, 30])
    check(act, dg, du, *rest, rows=30)
    assert np.all(act[30:] == 7.0) and np.all(dg[30:] == 7.0) and np.all(du[30:] == 7.0)
    act, dg, du, *rest = run(g[:30], u[:30], da[:30], offsets=[0, 4000])   # past the rows: cut
    check(act, dg, du, *rest)
    act, *_ = run(g[:30], u[:30], da[:30], offsets=[0, 0])
    assert np.all(act == 7.0)


def test_gradient_by_differences():
    """d(act)/dg by the difference of two activations, whose bf16 rounding is 2^-8 of each; curvature below one."""
    g = np.linspace(-6, 6, 512).reshape(8, 64)
    u, da = np.full_like(g, 1.0), np.full_like(g, 1.0)
    h = 0.25
    low, high = run(g - h, u, da), run(g + h, u, da)
    _, dg, du, g0, *_ = run(g, u, da)
    gl, gh = low[3], high[3]
    slope = (high[0] - low[0]) / (gh - gl)
    assert np.all(np.abs(slope - dg) <= 2.0 ** -8 * (np.abs(high[0]) + np.abs(low[0])) / (gh - gl) + 2.0 ** -8 * np.abs(dg) + 0.5 * (2 * h) ** 2)
    _, act, _, _ = formulas(g0, 1.0, 1.0)
    assert np.all(np.abs(du - act) <= 2.0 ** -8 * np.abs(act) + 1e-6)
