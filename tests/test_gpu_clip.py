"""The norm of many tensors and their clipping against exact sums.

Squares of fp32 and bf16 values are off by 2^-53 in fp64 and so is each of n additions: the total is within n 2^-52.
The norm is rounded to fp32 (2^-24), the scale too, and each product once more to its type (2^-24 or 2^-8).
"""
import math

import numpy as np
import pytest

from paper_2607_19539_amd import binding as B
from tests.gpu_helpers import log

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

F32, BF16 = torch.float32, torch.bfloat16


def make(sizes, seed, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return [(torch.randn(n, generator=g) * scale).to(dt).cuda() for n, dt in sizes]


def exact_total(tensors):
    return math.fsum(float((t.double() ** 2).sum()) for t in tensors)


def check(tensors, max_norm, in_place=False, stream=None):
    n = sum(t.numel() for t in tensors)
    before = [t.clone() for t in tensors]
    out = None if in_place else [torch.full_like(t, 7.0) for t in tensors]
    total, norm = torch.full((1,), -1.0, dtype=torch.float64, device="cuda"), torch.full((1,), -1.0, device="cuda")
    torch.cuda.synchronize()
    B.moe_squares(tensors, total, stream=stream)
    B.moe_clip(tensors, total, max_norm, out=out, norm=norm, stream=stream)
    torch.cuda.synchronize()
    want = exact_total(before)
    assert abs(float(total) - want) <= (n + 1) * 2.0 ** -52 * want
    root = math.sqrt(want)
    assert abs(float(norm) - root) <= 2.0 ** -23 * root
    scale = max_norm / root if root > max_norm else 1.0
    for b, a in zip(before, tensors if in_place else out):
        v, got = b.double(), a.double()
        if scale == 1.0:
            assert torch.equal(a, b)
        else:
            rounding = 2.0 ** -8 if a.dtype == BF16 else 2.0 ** -24
            assert bool(((got - v * scale).abs() <= (rounding + 2.0 ** -23) * (v * scale).abs() + 1e-38).all())
    if not in_place:
        for b, t in zip(before, tensors):
            assert torch.equal(b, t)


LISTS = {
    "one": [(1, F32)], "one16": [(1, BF16)], "odd": [(3, F32), (7, BF16), (1, F32), (8191, BF16), (4097, F32)],
    "empty_between": [(0, F32), (100, BF16), (0, BF16), (5, F32), (0, F32)], "none_held": [(0, F32), (0, BF16)],
    "long": [(3000001, F32), (5000003, BF16)], "many": [(1 + 37 * i % 5000, F32 if i % 3 else BF16) for i in range(300)],
    "table_full": [(65, F32)] * 128, "table_and_one": [(65, F32)] * 129, "larger_than_the_grid": [(40000000, BF16), (9, F32)],
}


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("name", list(LISTS))
def test_clip(name, in_place):
    log(f"clip {name} in_place={in_place}")
    tensors = make(LISTS[name], len(name))
    check([t.clone() for t in tensors], 0.5, in_place)
    check([t.clone() for t in tensors], 1e9, in_place)
    check([t.clone() for t in tensors], 0.0, in_place, stream=torch.cuda.Stream())


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("shift,out_shift", [(1, 1), (3, 3), (1, 0), (0, 5), (2, 6)])
def test_tensors_that_start_anywhere(dtype, shift, out_shift):
    """Parts of larger tensors, aligned to their elements alone, in and out alike or not."""
    room = make([(20000, dtype)], 3)[0]
    space = torch.full((20000,), 7.0, dtype=dtype, device="cuda")
    v, out = room[shift:shift + 9001], space[out_shift:out_shift + 9001]
    total = torch.zeros(1, dtype=torch.float64, device="cuda")
    B.moe_squares([v], total)
    want = exact_total([v])
    assert abs(float(total) - want) <= 9002 * 2.0 ** -52 * want
    B.moe_clip([v], total, 2.0, out=[out])
    scale = 2.0 / math.sqrt(want)
    bound = ((2.0 ** -8 if dtype == BF16 else 2.0 ** -24) + 2.0 ** -23) * (v.double() * scale).abs()
    assert bool(((out.double() - v.double() * scale).abs() <= bound).all())
    assert bool((space[:out_shift] == 7.0).all()) and bool((space[out_shift + 9001:] == 7.0).all())


@pytest.mark.parametrize("scale", [1e-40, 1e-25, 1e18, 1e30])
def test_values_whose_squares_leave_32_bits(scale):
    tensors = make([(5000, F32), (4000, BF16)], 9, scale)
    want = exact_total(tensors)
    total, norm = torch.zeros(1, dtype=torch.float64, device="cuda"), torch.zeros(1, device="cuda")
    B.moe_squares(tensors, total)
    B.moe_clip(tensors, total, 1.0, norm=norm, out=[torch.empty_like(t) for t in tensors])
    assert abs(float(total) - want) <= 9001 * 2.0 ** -52 * want
    assert abs(float(norm) - math.sqrt(want)) <= 2.0 ** -23 * math.sqrt(want) + 2.0 ** -149


@pytest.mark.parametrize("value", [float("inf"), float("nan")])
def test_a_norm_that_is_not_finite_changes_nothing(value):
    tensors = make([(5000, F32), (4000, BF16)], 2)
    tensors[0][77] = value
    before, out = [t.clone() for t in tensors], [torch.zeros_like(t) for t in tensors]
    total, norm = torch.zeros(1, dtype=torch.float64, device="cuda"), torch.zeros(1, device="cuda")
    B.moe_squares(tensors, total)
    B.moe_clip(tensors, total, 1.0, norm=norm, out=out)
    B.moe_clip(tensors, total, 1.0)
    assert not bool(norm.isfinite())
    for b, t, o in zip(before, tensors, out):
        assert torch.equal(b.nan_to_num(), t.nan_to_num()) and torch.equal(b.nan_to_num(), o.nan_to_num())


def test_no_tensors():
    total, norm = torch.ones(1, dtype=torch.float64, device="cuda"), torch.ones(1, device="cuda")
    B.moe_squares([], total)
    B.moe_clip([], total, 1.0, norm=norm)
    assert float(total) == 0.0 and float(norm) == 0.0


def test_totals_of_two_ranks_add_up():
    a, b = make([(1000, F32)], 1), make([(2000, BF16)], 2)
    ta, tb = torch.zeros(1, dtype=torch.float64, device="cuda"), torch.zeros(1, dtype=torch.float64, device="cuda")
    B.moe_squares(a, ta)
    B.moe_squares(b, tb)
    want, norm = exact_total(a + b), torch.zeros(1, device="cuda")
    B.moe_clip(a, ta + tb, 1.0, norm=norm)
    assert abs(float(norm) - math.sqrt(want)) <= 2.0 ** -23 * math.sqrt(want)


def test_the_same_bits_every_time():
    tensors = make(LISTS["many"] + LISTS["long"], 6)
    totals = []
    for _ in range(4):
        t = torch.zeros(1, dtype=torch.float64, device="cuda")
        B.moe_squares(tensors, t)
        totals.append(float(t))
    assert len(set(totals)) == 1


def test_an_out_that_overlaps_another_tensor_is_refused():
    room = torch.zeros(1000, device="cuda")
    total = torch.zeros(1, dtype=torch.float64, device="cuda")
    a, b, c = room[:500], room[499:900], room[500:900]
    for tensors, out in (([a, b], None), ([a, a], None), ([a], [room[1:501]]), ([a, room[500:]], [room[500:], a]), ([a, c], [a, room[600:1000]])):
        with pytest.raises(B.MoeError, match="overlaps"):
            B.moe_clip(tensors, total, 1.0, out=out)
    B.moe_clip([a, c], total, 1.0)
    B.moe_clip([a, a[:0], c], total, 1.0)
    B.moe_squares([a, a, b], total)


@pytest.mark.parametrize("value", [3e38, -3e38])
def test_a_norm_that_32_bits_do_not_hold_changes_nothing(value):
    """Finite in 64 bits, infinite in the norm that the caller sees."""
    tensors = [torch.full((100,), value, device="cuda"), torch.full((64,), 2.0, dtype=BF16, device="cuda")]
    before, out = [t.clone() for t in tensors], [torch.zeros_like(t) for t in tensors]
    total, norm = torch.zeros(1, dtype=torch.float64, device="cuda"), torch.zeros(1, device="cuda")
    B.moe_squares(tensors, total)
    assert math.isfinite(float(total))
    B.moe_clip(tensors, total, 1.0, norm=norm, out=out)
    B.moe_clip(tensors, total, 1.0)
    assert math.isinf(float(norm))
    for b, t, o in zip(before, tensors, out):
        assert torch.equal(b, t) and torch.equal(b, o)


@pytest.mark.parametrize("max_norm", [2.0 ** -23, 2.0 ** -30, 2.0 ** -43, 2.0 ** -66])
def test_a_scale_that_32_bits_hold_as_a_subnormal(max_norm):
    """From a norm of some 1e33 down: the scale is below 2^-126 but the results are ordinary values."""
    tensors = make([(5000, F32), (4000, BF16)], 12, 1e31)
    check([t.clone() for t in tensors], max_norm)
    check(tensors, max_norm, in_place=True)
