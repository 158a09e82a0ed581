"""The gradient by the weights added to what dw holds, by each of its kernels and numbers of parts, against 64 bits.

Bounds as in test_gpu_product.py, n 2^-23 of the magnitudes for n products.  Those of bf16 values are exact in fp32, which
leaves n 2^-24 for the additions of up to eight parts and of the former value, whose magnitude counts as well.
"""
import ctypes

import numpy as np
import pytest

from paper_2607_19539_amd import binding as B
from tests.gpu_helpers import log
from tests.test_gpu_product import EACH, SENTINEL, DwPlan, ProductDwArgs, case, check_dw, host, ptr

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


def add(plan, d, before):
    """dw after the launch, with room behind it that has to stay as it was."""
    f = B.load()._ZN3moe22launch_product_dw_planERKNS_6DwPlanERKNS_13ProductDwArgsEP12ihipStream_t
    f.argtypes, f.restype = [ctypes.POINTER(DwPlan), ctypes.POINTER(ProductDwArgs), ctypes.c_void_p], ctypes.c_int
    n = before.size
    room = torch.full((n + 1024,), SENTINEL, device="cuda")
    room[:n] = torch.from_numpy(before.astype(np.float32)).flatten()
    parts = torch.full((plan.split, *d["w"].shape), np.nan, device="cuda")
    args = ProductDwArgs(ptr(d["dy_dev"]), ptr(d["x_dev"]), ptr(d["index_dev"]), ptr(d["off_dev"]), ptr(room), ptr(parts), d["n"],
                         d["rows"], d["E"], d["K"], d["N"], 0, 1)
    torch.cuda.synchronize()
    assert f(ctypes.byref(plan), ctypes.byref(args), torch.cuda.current_stream().cuda_stream) == 0
    got = host(room)
    assert (got[n:] == SENTINEL).all()
    return got[:n].reshape(before.shape)


def former(d):
    rng = np.random.default_rng(d["K"] + 13 * d["N"])
    return rng.standard_normal(d["w"].shape).astype(np.float32).astype(np.float64)


PLANS = [(64, 1), (64, 4), (128, 1), (128, 2), (256, 1), (256, 3)]


@pytest.mark.parametrize("gather", [False, True])
@pytest.mark.parametrize("tile,split", PLANS)
@pytest.mark.parametrize("counts,K,N", EACH, ids=lambda v: str(v)[:24])
def test_each_dw_kernel_adds(counts, K, N, tile, split, gather):
    log(f"dw added, tiles of {tile}, {split} parts {str(counts)[:60]} K={K} N={N} gather={gather}")
    d = case(counts, K, N, gather, K * 13 + N)
    if gather and d["end"] > 8:
        d["index"][d["end"] // 2] = d["n"]
        d["index_dev"] = torch.from_numpy(d["index"]).cuda()
    before = former(d)
    got = add(DwPlan(tile, split), d, before)
    check_dw(got, d, before=before)
    for e, c in enumerate(d["c"]):
        if c == 0:
            assert np.array_equal(got[e], before[e])


@pytest.mark.parametrize("tile,split", PLANS)
def test_a_sum_added_twice(tile, split):
    """Whole numbers, so that every sum is exact: dw holds three of them after an assignment and two additions."""
    d = case([300, 0, 64, 1, 700], 264, 520, True, 17)
    rng = np.random.default_rng(18)
    for name in ("x", "dy"):
        d[name] = rng.integers(-3, 4, d[name].shape).astype(np.float64)
        d[name + "_dev"] = torch.from_numpy(d[name]).to(torch.bfloat16).cuda()
    once = add(DwPlan(tile, split), d, np.zeros(d["w"].shape))
    twice = add(DwPlan(tile, split), d, once)
    lo = 0
    for e, c in enumerate(d["c"]):
        want = d["dy"][lo:lo + c].T @ d["x"][d["index"][lo:lo + c]]
        assert np.array_equal(once[e], want) and np.array_equal(twice[e], 2 * want)
        lo += c


def test_the_call_adds_where_training_sizes_lead():
    """Sizes for which the call itself takes whole tiles, and parts of rows."""
    g = B.load()._ZN3moe15product_dw_planEliii
    g.argtypes, g.restype = [ctypes.c_int64] + [ctypes.c_int32] * 3, DwPlan
    seen = set()
    for counts, K, N in (([900, 0, 1100, 1040], 2048, 2816), ([2600, 3100], 256, 512), (8192, 512, 512)):
        log(f"dw added by the call {counts} K={K} N={N}")
        d = case(counts, K, N, False, K)
        p = g(d["rows"], d["E"], K, N)
        seen.add((p.tile, p.split > 1))
        before = former(d)
        dw = torch.from_numpy(before.astype(np.float32)).cuda()
        B.moe_product_dw(d["dy_dev"], d["x_dev"], dw, expert_offsets=d["off_dev"], accumulate=True)
        check_dw(host(dw), d, before=before)
    assert (256, False) in seen and any(parts for _, parts in seen), seen
