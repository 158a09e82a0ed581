"""The norm, its gradients and 8-bit rows against the formulas in 64 bits.

Tolerances.  bf16 keeps 8 significant bits, so rounding to it moves a value by at most 2^-8 of it.  An fp32
sum of up to 65536 positive terms, taken in at most 256 steps per thread and a tree, is within 2^-14 of the
exact one; r, a square root and a division more, within 2^-14 too; y within 2^-13.
"""
import numpy as np
import pytest

from paper_2607_19539_amd import binding as B
from tests.gpu_helpers import log

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

U16, F32 = 2.0 ** -8, 2.0 ** -13
EPS = 1e-5
SHAPES = [(1, 8), (3, 16), (5, 72), (2, 504), (7, 512), (4, 520), (33, 1024), (9, 2056), (6, 4096), (5, 7168),
          (3, 8200), (2, 16384), (3, 20008), (1, 65536), (1500, 64), (700, 1032), (300, 2048), (4099, 320)]


def bf16(rng, shape, scale=1.0):
    return torch.from_numpy((rng.standard_normal(shape) * scale).astype(np.float32)).to(torch.bfloat16)


def inputs(T, H, seed=0):
    rng = np.random.default_rng(seed * 100003 + T * 131 + H)
    x, res = bf16(rng, (T, H)), bf16(rng, (T, H), 2.0)
    x[:, H // 3] *= 16
    w = bf16(rng, (H,), 0.2) + 1.0
    return x, res, w


def run_norm(x, w, eps=EPS, residual=None, q8=True, out=True, rstd=True, sum_out=True, stream=None):
    T, H = x.shape
    dev = lambda t: None if t is None else t.cuda()  # noqa: E731
    d = dict(sum_out=torch.full((T, H), -7.0, dtype=torch.bfloat16, device="cuda") if sum_out else None,
             out=torch.full((T, H), -7.0, dtype=torch.bfloat16, device="cuda") if out else None,
             out_q=torch.full((T, H), 99, dtype=torch.int8, device="cuda") if q8 else None,
             scale=torch.full((T,), -7.0, device="cuda") if q8 else None,
             rstd=torch.full((T,), -7.0, device="cuda") if rstd else None)
    B.moe_norm(dev(x), dev(w), eps, residual=dev(residual), stream=stream, **d)
    torch.cuda.synchronize()
    return {k: None if v is None else v.cpu() for k, v in d.items()}


def check_norm(x, w, residual, got, eps=EPS):
    h = x if residual is None else (x.float() + residual.float()).to(torch.bfloat16)
    h64 = h.double()
    r = 1.0 / torch.sqrt(h64.pow(2).mean(1, keepdim=True) + eps)
    y = h64 * r * w.double()
    if got["sum_out"] is not None:
        assert torch.equal(got["sum_out"], h)
    if got["rstd"] is not None:
        assert bool(((got["rstd"].double() - r[:, 0]).abs() <= F32 * r[:, 0]).all())
    if got["out"] is not None:
        assert bool(((got["out"].double() - y).abs() <= (U16 + F32) * y.abs()).all())
    if got["out_q"] is not None:
        check_q8(y, got["out_q"], got["scale"], F32)


def check_q8(y, q, scale, rel):
    """q * scale is within half a step of y, and a share `rel` of y (rounding the division moves a tie)."""
    top = y.abs().amax(1)
    s = scale.double()
    assert bool(((s - top / 127).abs() <= 2 * rel * top / 127).all())
    assert int(q.min()) >= -127
    off = (q.double() * s[:, None] - y).abs()
    assert bool((off <= s[:, None] * 0.5 + 4 * rel * top[:, None]).all())


@pytest.mark.parametrize("T,H", SHAPES)
def test_norm(T, H):
    log(f"norm T={T} H={H}")
    x, res, w = inputs(T, H)
    check_norm(x, w, res, run_norm(x, w, residual=res))


@pytest.mark.parametrize("T,H", [(5, 72), (48, 4096), (2049, 256)])
@pytest.mark.parametrize("q8,out,rstd,sum_out,residual", [
    (True, False, False, True, True), (False, True, False, False, False), (True, False, False, False, False),
    (False, False, True, False, True), (False, True, True, True, True)])
def test_norm_outputs_asked_for(T, H, q8, out, rstd, sum_out, residual):
    x, res, w = inputs(T, H, 1)
    res = res if residual else None
    check_norm(x, w, res, run_norm(x, w, residual=res, q8=q8, out=out, rstd=rstd, sum_out=sum_out))


@pytest.mark.parametrize("T,H", [(6, 1024), (700, 4096)])
def test_norm_in_place(T, H):
    x, res, w = inputs(T, H, 2)
    a, b = x.cuda(), res.cuda()
    B.moe_norm(a, w.cuda(), EPS, residual=b, sum_out=b, out=a)
    check_norm(x, w, res, dict(sum_out=b.cpu(), out=a.cpu(), out_q=None, rstd=None))


def test_norm_of_no_rows():
    e = torch.zeros((0, 64), dtype=torch.bfloat16, device="cuda")
    B.moe_norm(e, torch.ones(64, dtype=torch.bfloat16, device="cuda"), EPS, out=e)
    dw = torch.full((64,), 5.0, device="cuda")
    B.moe_norm_backward(e, e, torch.ones(64, dtype=torch.bfloat16, device="cuda"), torch.zeros(0, device="cuda"), e, dw)
    assert float(dw.abs().max()) == 0.0


def test_norm_odd_values():
    """Rows of zeros, of tiny and huge values, with an infinity, with a NaN."""
    H = 264
    x = torch.ones((6, H), dtype=torch.bfloat16)
    x[0] = 0.0
    x[1] = 2.0 ** -130
    x[2, 5], x[3, 7] = float("inf"), float("nan")
    x[4] = 2.0 ** 40
    w = torch.ones(H, dtype=torch.bfloat16)
    got = run_norm(x, w, eps=0.0)
    assert torch.isnan(got["scale"][2:4]).all() and int(got["out_q"][2:4].abs().max()) == 0
    assert torch.isnan(got["out"][3]).all() and torch.isnan(got["out"][2, 5])
    for r in (4, 5):
        assert int((got["out_q"][r] - 127).abs().max()) == 0 and bool((got["out"][r].float() == 1.0).all())
    got = run_norm(x, w, eps=1e-6)
    assert float(got["out"][0].abs().max()) == 0.0 and float(got["scale"][0]) == 0.0 and int(got["out_q"][0].abs().max()) == 0


@pytest.mark.parametrize("T,H", SHAPES)
def test_q8_rows_and_back(T, H):
    x, _, _ = inputs(T, H, 3)
    if T > 4:
        x[1], x[2], x[3, 1], x[4, 0] = 0.0, 2.0 ** -110, float("inf"), float("nan")
    q, s = torch.full((T, H), 99, dtype=torch.int8, device="cuda"), torch.full((T,), -7.0, device="cuda")
    B.moe_q8_rows(x.cuda(), q, s)
    back = torch.full((T, H), -7.0, dtype=torch.bfloat16, device="cuda")
    B.moe_q8_restore(q, s, back)
    q, s, back = q.cpu(), s.cpu(), back.cpu()
    fine = torch.ones(T, dtype=torch.bool)
    if T > 4:
        fine[1:5] = False
        assert bool((s[1:3] == 0).all()) and float(back[1:3].abs().max()) == 0.0
        assert torch.isnan(s[3:5]).all() and torch.isnan(back[3:5]).all() and int(q[1:5].abs().max()) == 0
    check_q8(x[fine].double(), q[fine], s[fine], 2.0 ** -22)
    assert torch.equal(back[fine], (q[fine].float() * s[fine][:, None]).to(torch.bfloat16))


def gradients64(dy, h, w, dsum, eps=EPS):
    """dx, dweight and the sums of the magnitudes of their terms, in 64 bits from the formula."""
    dy, h, w = dy.double(), h.double(), w.double()
    r = 1.0 / torch.sqrt(h.pow(2).mean(1, keepdim=True) + eps)
    g = dy * w
    c = (g * h).mean(1, keepdim=True)
    dx = r * (g - h * r * r * c)
    mag = r * (g.abs() + h.abs() * r * r * (g * h).abs().mean(1, keepdim=True))
    if dsum is not None:
        dx, mag = dx + dsum.double(), mag + dsum.double().abs()
    return dx, mag, (dy * h * r).sum(0), (dy * h * r).abs().sum(0)


def run_backward(dy, x, w, dsum, eps=EPS, in_place=False):
    T, H = x.shape
    h, rstd = torch.empty_like(x, device="cuda"), torch.empty(T, device="cuda")
    B.moe_norm(x.cuda(), w.cuda(), eps, sum_out=h, rstd=rstd)
    ds = None if dsum is None else dsum.cuda()
    dx = ds if in_place else torch.full((T, H), -7.0, dtype=torch.bfloat16, device="cuda")
    dw = torch.full((H,), -7.0, device="cuda")
    B.moe_norm_backward(dy.cuda(), h, w.cuda(), rstd, dx, dw, dsum=ds)
    torch.cuda.synchronize()
    return dx.cpu(), dw.cpu()


@pytest.mark.parametrize("dsum,in_place", [(False, False), (True, False), (True, True)])
@pytest.mark.parametrize("T,H", SHAPES)
def test_norm_backward(T, H, dsum, in_place):
    log(f"norm backward T={T} H={H}")
    x, res, w = inputs(T, H, 4)
    rng = np.random.default_rng(T + H)
    dy, ds = bf16(rng, (T, H), 0.1), bf16(rng, (T, H), 0.1) if dsum else None
    dx, dw = run_backward(dy, x, w, ds, in_place=in_place)
    rx, mx, rw, mw = gradients64(dy, x, w, ds)
    assert bool(((dx.double() - rx).abs() <= U16 * rx.abs() + F32 * mx).all())
    # A sum of T terms in 32 bits, one after another at worst, each term within 2^-13.
    assert bool(((dw.double() - rw).abs() <= (F32 + T * 2.0 ** -24) * mw).all())


def test_norm_backward_against_differences():
    """The gradient of sum(dy * y) + sum(dsum * h) by central differences of the forward formula in 64 bits.
    A step of 1e-4 leaves an error of 1e-8; the kernel's bf16 outputs are within 2^-8."""
    T, H = 3, 40
    x, _, w = inputs(T, H, 5)
    rng = np.random.default_rng(7)
    dy, ds = bf16(rng, (T, H)), bf16(rng, (T, H))
    dx, dw = run_backward(dy, x, w, ds)

    def loss(x64, w64):
        r = 1.0 / torch.sqrt(x64.pow(2).mean(1, keepdim=True) + EPS)
        return float((dy.double() * x64 * r * w64).sum() + (ds.double() * x64).sum())

    _, mag, _, mag_w = gradients64(dy, x, w, ds)
    step = 1e-4
    for t, c in [(0, 0), (0, H // 3), (1, 5), (2, 39), (2, H // 3)]:
        d = torch.zeros((T, H), dtype=torch.float64)
        d[t, c] = step
        want = (loss(x.double() + d, w.double()) - loss(x.double() - d, w.double())) / (2 * step)
        assert abs(float(dx[t, c]) - want) <= U16 * abs(want) + F32 * float(mag[t, c]) + 1e-6
    for c in (0, 11, H // 3):
        d = torch.zeros(H, dtype=torch.float64)
        d[c] = step
        want = (loss(x.double(), w.double() + d) - loss(x.double(), w.double() - d)) / (2 * step)
        assert abs(float(dw[c]) - want) <= F32 * float(mag_w[c]) + 1e-6


def test_norm_backward_is_repeatable():
    x, _, w = inputs(1777, 1032, 6)
    dy = bf16(np.random.default_rng(8), x.shape)
    a, b = run_backward(dy, x, w, None), run_backward(dy, x, w, None)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_norm_on_another_stream():
    x, res, w = inputs(257, 2048, 9)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    check_norm(x, w, res, run_norm(x, w, residual=res, stream=s))


def test_norm_rows_past_four_gigabytes():
    """Offsets into a tensor of over 2^32 bytes."""
    T, H = 35000, 65536
    x = torch.ones((T, H), dtype=torch.bfloat16, device="cuda")
    x[T - 1, 3] = 5.0
    q, s = torch.empty((T, H), dtype=torch.int8, device="cuda"), torch.empty(T, device="cuda")
    B.moe_q8_rows(x, q, s)
    assert bool((s[:T - 1] == 1.0 / 127.0).all()) and float(s[T - 1]) == np.float32(5.0) / np.float32(127.0)
    assert q[T - 1, :5].tolist() == [25, 25, 25, 127, 25] and bool((q[T - 2] == 127).all())


@pytest.mark.parametrize("T,H", [(1, 64), (2, 20008), (16, 2048), (17, 2048), (8, 4096), (4, 8192), (2, 16384)])
def test_norm_backward_of_few_rows_into_any_float(T, H):
    """One or two turns of rows need no workspace; dweight may begin at any float."""
    x, _, w = inputs(T, H, 11)
    dy = bf16(np.random.default_rng(12), (T, H), 0.1)
    h, rstd = torch.empty((T, H), dtype=torch.bfloat16, device="cuda"), torch.empty(T, device="cuda")
    B.moe_norm(x.cuda(), w.cuda(), EPS, sum_out=h, rstd=rstd)
    room = torch.full((H + 2,), -7.0, device="cuda")
    dx = torch.empty_like(h)
    B.moe_norm_backward(dy.cuda(), h, w.cuda(), rstd, dx, room[1:H + 1])
    _, _, rw, mw = gradients64(dy, x, w, None)
    got = room.cpu().double()
    assert float(got[0]) == -7.0 and float(got[H + 1]) == -7.0
    assert bool(((got[1:H + 1] - rw).abs() <= (F32 + T * 2.0 ** -24) * mw).all())
