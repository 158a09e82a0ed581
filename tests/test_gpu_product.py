"""The 16-bit products and their gradients against sums in 64 bits.

A sum of n products in fp32, in whatever order, is off by at most n 2^-23 of the sum of their magnitudes (each product
and each addition rounds by 2^-24 at most, the matrix instruction's additions by one bit more).  A bf16 result is
rounded once more, by 2^-8 of itself.
"""
import ctypes

import numpy as np
import pytest

from paper_2607_19539_amd import binding as B
from tests.gpu_helpers import log

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

SENTINEL = -4096.0


def bf16(rng, *shape, std=1.0):
    """bf16 values, held as float64, and the device tensor of them."""
    t = torch.from_numpy((rng.standard_normal(shape) * std).astype(np.float32)).to(torch.bfloat16)
    return t.double().numpy(), t.cuda()


def near(got, want, size, n, rounding):
    """got [..] against want, where sums of n products have the magnitude `size`."""
    assert np.array_equal(np.isnan(got), np.isnan(want))
    fine = np.isfinite(want)
    assert np.array_equal(got[~fine & ~np.isnan(want)], want[~fine & ~np.isnan(want)])
    off = np.abs(got - want)[fine] - rounding * np.abs(want)[fine] - n * 2.0 ** -23 * size[fine] - 1e-37
    assert off.size == 0 or off.max() <= 0, float(off.max())


def case(counts, K, N, gather, seed):
    """Inputs on the host (float64) and the device, the offsets and the index."""
    rng = np.random.default_rng(seed)
    grouped = not isinstance(counts, int)
    c = list(counts) if grouped else [counts]
    off = np.concatenate([[0], np.cumsum(c)]).astype(np.int32)
    rows = int(off[-1]) + (5 if grouped else 0)      # rows that belong to nobody
    n = max(1, rows // 3) if gather else rows
    d = {"off": off if grouped else None, "end": int(off[-1]), "c": c, "rows": rows, "n": n, "E": len(c), "K": K, "N": N, "index": None}
    for name, shape, std in (("x", (n, K), 1.0), ("w", (len(c), N, K), 0.1), ("dy", (rows, N), 0.5)):
        d[name], d[name + "_dev"] = bf16(rng, *shape, std=std)
    if gather:
        d["index"] = rng.integers(0, n, rows).astype(np.int32)
        d["index"][d["end"]:] = -1
    d["off_dev"] = None if d["off"] is None else torch.from_numpy(d["off"]).cuda()
    d["index_dev"] = None if d["index"] is None else torch.from_numpy(d["index"]).cuda()
    return d


def experts(d):
    lo = 0
    for e, c in enumerate(d["c"]):
        if c:
            yield e, slice(lo, lo + c)
        lo += c


def x_rows(d, rows):
    """x of these rows; NaN where the index names none."""
    if d["index"] is None:
        return d["x"][rows]
    i = d["index"][rows]
    ok = (i >= 0) & (i < d["n"])
    x = d["x"][np.where(ok, i, 0)]
    x[~ok] = np.nan
    return x


def magnitude(a):
    return np.where(np.isfinite(a), np.abs(a), 0.0)


def filled(shape, dtype=torch.bfloat16):
    return torch.full(shape, SENTINEL, dtype=dtype, device="cuda")


def host(t):
    torch.cuda.synchronize()
    return t.double().cpu().numpy()


def check_rows(got, d, a_of, width, w_side):
    want, size = np.full((d["rows"], width), SENTINEL), np.zeros((d["rows"], width))
    for e, r in experts(d):
        w = d["w"][e].T if w_side == "rows" else d["w"][e]
        a = a_of(r)
        want[r], size[r] = a @ w, magnitude(a) @ np.abs(w)
    near(got, want, size, d["K"] if w_side == "rows" else d["N"], 2.0 ** -8)


def check_dw(got, d, before=None, rounding=2.0 ** -24):
    want, size = np.zeros(d["w"].shape), np.zeros(d["w"].shape)
    for e, r in experts(d):
        x, dy = x_rows(d, r), d["dy"][r]
        want[e], size[e] = dy.T @ x, magnitude(dy).T @ magnitude(x)
    if before is not None:
        want, size = want + before, size + np.abs(before)
    near(got, want, size, max(d["c"]) + 2, rounding)


SIZES = [
    (1, 8, 8), (3, 16, 24), (2, 64, 64), (17, 72, 40), (64, 56, 136), (65, 128, 72), (130, 200, 264), (300, 320, 576), (513, 264, 1032),
    (1, 1408, 520), (200, 2056, 64),
    ([0, 5, 0, 0, 17, 1, 0], 64, 72), ([1, 1, 1, 1], 8, 8), ([0, 0, 300, 0], 136, 256), ([3, 64, 65, 128, 129, 31], 176, 520),
    ([256, 1, 257, 300, 0, 90], 72, 320), ([0, 0, 0], 64, 64), ([i % 5 for i in range(200)], 80, 136),
]


@pytest.mark.parametrize("gather", [False, True])
@pytest.mark.parametrize("counts,K,N", SIZES, ids=lambda v: str(v)[:24])
def test_product_and_gradients(counts, K, N, gather):
    log(f"product {str(counts)[:60]} K={K} N={N} gather={gather}")
    d = case(counts, K, N, gather, K + N)
    y, dx = filled((d["rows"], N)), filled((d["rows"], K))
    B.moe_product(d["x_dev"], d["w_dev"], y, row_index=d["index_dev"], expert_offsets=d["off_dev"])
    check_rows(host(y), d, lambda r: x_rows(d, r), N, "rows")
    B.moe_product_dx(d["dy_dev"], d["w_dev"], dx, expert_offsets=d["off_dev"])
    check_rows(host(dx), d, lambda r: d["dy"][r], K, "k")
    for dtype, rounding in ((torch.float32, 2.0 ** -24), (torch.bfloat16, 2.0 ** -8)):
        dw = filled((d["E"], N, K), dtype)
        B.moe_product_dw(d["dy_dev"], d["x_dev"], dw, row_index=d["index_dev"], expert_offsets=d["off_dev"])
        check_dw(host(dw), d, rounding=rounding)
    before = host(dw.float())
    dw = torch.from_numpy(before.astype(np.float32)).cuda()
    B.moe_product_dw(d["dy_dev"], d["x_dev"], dw, row_index=d["index_dev"], expert_offsets=d["off_dev"], accumulate=True)
    check_dw(host(dw), d, before=before)


class ProductArgs(ctypes.Structure):
    """The launchers' arguments (csrc/ops.hpp)."""
    _fields_ = [(n, ctypes.c_void_p) for n in ("x", "index", "offsets", "w", "out")] + \
               [("x_rows", ctypes.c_int64), ("rows", ctypes.c_int64), ("experts", ctypes.c_int32), ("K", ctypes.c_int32),
                ("N", ctypes.c_int32)]


class ProductDwArgs(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("dy", "x", "index", "offsets", "dw", "parts")] + \
               [("x_rows", ctypes.c_int64), ("rows", ctypes.c_int64)] + \
               [(n, ctypes.c_int32) for n in ("experts", "K", "N", "bf16", "accumulate")]


class DwPlan(ctypes.Structure):
    _fields_ = [("tile", ctypes.c_int), ("split", ctypes.c_int)]


KINDS = ["slim1", "slim2", "tiles64", "tiles128", "tiles256", "tiles128x64", "deep128"]


def ptr(t):
    return None if t is None else t.data_ptr()


def launch_kind(kind, d, by_k):
    f = B.load()._ZN3moe19launch_product_kindENS_11ProductKindERKNS_11ProductArgsEbP12ihipStream_t
    f.argtypes, f.restype = [ctypes.c_int, ctypes.POINTER(ProductArgs), ctypes.c_bool, ctypes.c_void_p], ctypes.c_int
    K, N = (d["N"], d["K"]) if by_k else (d["K"], d["N"])
    out = filled((d["rows"], N))
    x, index, n = (d["dy_dev"], None, d["rows"]) if by_k else (d["x_dev"], d["index_dev"], d["n"])
    args = ProductArgs(ptr(x), ptr(index), ptr(d["off_dev"]), ptr(d["w_dev"]), ptr(out), n, d["rows"], d["E"], K, N)
    torch.cuda.synchronize()
    assert f(KINDS.index(kind), ctypes.byref(args), by_k, torch.cuda.current_stream().cuda_stream) == 0
    return host(out)


# Every height of the whole tiles, several items for each of their workgroups, more experts than a wave has lanes; sums
# of one chunk, of one step, of a few, with every kind of end.
EACH = [
    (1, 8, 8), (300, 24, 72), (257, 56, 256), (520, 64, 264), (65, 72, 520), (193, 128, 136), (700, 136, 1032), (260, 192, 40),
    (129, 200, 264), (64, 320, 520), (33, 968, 264),
    ([0, 5, 0, 0, 17, 1, 0], 64, 72), ([3, 64, 65, 128, 129, 31, 192, 193, 256, 257, 0, 1], 88, 520),
    ([1300, 700, 2000, 0, 1096, 33, 64, 65, 128, 129, 1, 192, 193, 256, 257, 600], 136, 2080),
    ([i % 5 for i in range(200)], 40, 136), ([i * 37 % 290 for i in range(130)], 72, 520),
]


@pytest.mark.parametrize("gather", [False, True])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("counts,K,N", EACH, ids=lambda v: str(v)[:24])
def test_each_product_kernel(counts, K, N, kind, gather):
    log(f"product {kind} {str(counts)[:60]} K={K} N={N} gather={gather}")
    d = case(counts, K, N, gather, K * 3 + N)
    if gather and d["rows"] > 8:
        d["index"][d["rows"] // 2], d["index"][1] = -5, d["n"]
        d["index_dev"] = torch.from_numpy(d["index"]).cuda()
    check_rows(launch_kind(kind, d, False), d, lambda r: x_rows(d, r), N, "rows")
    if not gather:
        check_rows(launch_kind(kind, d, True), d, lambda r: d["dy"][r], K, "k")
        # With the matrix the other way round, so that the long side is summed over and the short one comes out.
        t = case(counts, N, K, False, K * 5 + N)
        check_rows(launch_kind(kind, t, True), t, lambda r: t["dy"][r], N, "k")


@pytest.mark.parametrize("gather", [False, True])
@pytest.mark.parametrize("tile,split", [(64, 1), (64, 4), (128, 1), (128, 2), (256, 1), (256, 3)])
@pytest.mark.parametrize("counts,K,N", EACH, ids=lambda v: str(v)[:24])
def test_each_dw_kernel(counts, K, N, tile, split, gather):
    log(f"dw tiles of {tile}, {split} parts {str(counts)[:60]} K={K} N={N} gather={gather}")
    d = case(counts, K, N, gather, K * 7 + N)
    f = B.load()._ZN3moe22launch_product_dw_planERKNS_6DwPlanERKNS_13ProductDwArgsEP12ihipStream_t
    f.argtypes, f.restype = [ctypes.POINTER(DwPlan), ctypes.POINTER(ProductDwArgs), ctypes.c_void_p], ctypes.c_int
    dw, parts = filled((d["E"], N, K), torch.float32), torch.full((split, d["E"], N, K), np.nan, device="cuda")
    args = ProductDwArgs(ptr(d["dy_dev"]), ptr(d["x_dev"]), ptr(d["index_dev"]), ptr(d["off_dev"]), ptr(dw), ptr(parts), d["n"],
                         d["rows"], d["E"], K, N, 0, 0)
    torch.cuda.synchronize()
    assert f(ctypes.byref(DwPlan(tile, split)), ctypes.byref(args), torch.cuda.current_stream().cuda_stream) == 0
    check_dw(host(dw), d)


@pytest.mark.parametrize("gather", [False, True])
@pytest.mark.parametrize("tile,split", [(64, 1), (128, 1), (128, 2), (256, 1)])
@pytest.mark.parametrize("counts,K,N", EACH, ids=lambda v: str(v)[:24])
def test_each_dw_kernel_in_16_bits(counts, K, N, tile, split, gather):
    """Nothing is written past dw, and a row that is not there shows in its expert's values alone."""
    log(f"dw in bf16, tiles of {tile}, {split} parts {str(counts)[:60]} K={K} N={N} gather={gather}")
    d = case(counts, K, N, gather, K * 11 + N)
    if gather and d["end"] > 8:
        d["index"][d["end"] // 2] = d["n"]
        d["index_dev"] = torch.from_numpy(d["index"]).cuda()
    f = B.load()._ZN3moe22launch_product_dw_planERKNS_6DwPlanERKNS_13ProductDwArgsEP12ihipStream_t
    f.argtypes, f.restype = [ctypes.POINTER(DwPlan), ctypes.POINTER(ProductDwArgs), ctypes.c_void_p], ctypes.c_int
    room, parts = filled((d["E"] * N * K + 1024,)), torch.full((split, d["E"], N, K), np.nan, device="cuda")
    args = ProductDwArgs(ptr(d["dy_dev"]), ptr(d["x_dev"]), ptr(d["index_dev"]), ptr(d["off_dev"]), ptr(room), ptr(parts), d["n"],
                         d["rows"], d["E"], K, N, 1, 0)
    torch.cuda.synchronize()
    assert f(ctypes.byref(DwPlan(tile, split)), ctypes.byref(args), torch.cuda.current_stream().cuda_stream) == 0
    got = host(room)
    assert (got[-1024:] == SENTINEL).all()
    check_dw(got[:-1024].reshape(d["w"].shape), d, rounding=2.0 ** -8)


@pytest.mark.parametrize("tile,split", [(64, 1), (64, 4), (128, 2), (256, 1), (256, 3)])
def test_a_row_that_is_not_there_shows_in_its_experts_dw(tile, split):
    d = case([300, 40, 0, 700], 136, 264, True, 5)
    d["index"][310] = d["n"]
    d["index_dev"] = torch.from_numpy(d["index"]).cuda()
    f = B.load()._ZN3moe22launch_product_dw_planERKNS_6DwPlanERKNS_13ProductDwArgsEP12ihipStream_t
    f.argtypes, f.restype = [ctypes.POINTER(DwPlan), ctypes.POINTER(ProductDwArgs), ctypes.c_void_p], ctypes.c_int
    dw, parts = filled((4, 264, 136), torch.float32), torch.full((split, 4, 264, 136), np.nan, device="cuda")
    args = ProductDwArgs(ptr(d["dy_dev"]), ptr(d["x_dev"]), ptr(d["index_dev"]), ptr(d["off_dev"]), ptr(dw), ptr(parts), d["n"],
                         d["rows"], 4, 136, 264, 0, 0)
    torch.cuda.synchronize()
    assert f(ctypes.byref(DwPlan(tile, split)), ctypes.byref(args), torch.cuda.current_stream().cuda_stream) == 0
    check_dw(host(dw), d)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("K", [40, 72, 200])
def test_values_past_the_end_of_a_sum_do_not_enter_it(K, kind):
    """Infinities and NaN of other rows and other experts, and an infinity that a sum's last step would meet twice."""
    d = case([70, 33, 130], K, 72, False, K)
    for name in ("x", "dy"):
        v, t = d[name], d[name + "_dev"]
        v[d["end"]:], v[69], v[75] = np.nan, np.inf, -np.inf
        t[d["end"]:], t[69], t[75] = float("nan"), float("inf"), -float("inf")
        v[71, K // 2 if name == "x" else 36] = np.inf
        t[71, K // 2 if name == "x" else 36] = float("inf")
    with np.errstate(invalid="ignore"):
        check_rows(launch_kind(kind, d, False), d, lambda r: d["x"][r], 72, "rows")
        check_rows(launch_kind(kind, d, True), d, lambda r: d["dy"][r], K, "k")


@pytest.mark.parametrize("tile", [64, 128, 256])
def test_rows_of_other_experts_do_not_enter_dw(tile):
    d = case([70, 33, 130, 64], 72, 136, False, 3)
    for name in ("x", "dy"):
        for rows, v in ((slice(70, 103), np.nan), (slice(d["end"], None), np.inf)):
            d[name][rows] = v
            d[name + "_dev"][rows] = v
    f = B.load()._ZN3moe22launch_product_dw_planERKNS_6DwPlanERKNS_13ProductDwArgsEP12ihipStream_t
    f.argtypes, f.restype = [ctypes.POINTER(DwPlan), ctypes.POINTER(ProductDwArgs), ctypes.c_void_p], ctypes.c_int
    dw = filled((4, 136, 72), torch.float32)
    args = ProductDwArgs(ptr(d["dy_dev"]), ptr(d["x_dev"]), None, ptr(d["off_dev"]), ptr(dw), None, d["n"], d["rows"], 4, 72, 136, 0, 0)
    torch.cuda.synchronize()
    assert f(ctypes.byref(DwPlan(tile, 1)), ctypes.byref(args), torch.cuda.current_stream().cuda_stream) == 0
    check_dw(host(dw), d)


def test_offsets_outside_the_rows_are_cut():
    d = case([10, 0, 40], 64, 32, False, 2)
    d["rows"] = 50
    for n in ("x", "dy"):
        d[n], d[n + "_dev"] = d[n][:50], d[n + "_dev"][:50].contiguous()
    off = torch.tensor([0, 10, 5, 1000], dtype=torch.int32, device="cuda")
    y, dx, dw = filled((50, 32)), filled((50, 64)), filled((3, 32, 64), torch.float32)
    B.moe_product(d["x_dev"], d["w_dev"], y, expert_offsets=off)
    B.moe_product_dx(d["dy_dev"], d["w_dev"], dx, expert_offsets=off)
    B.moe_product_dw(d["dy_dev"], d["x_dev"], dw, expert_offsets=off)
    check_rows(host(y), d, lambda r: d["x"][r], 32, "rows")
    check_rows(host(dx), d, lambda r: d["dy"][r], 64, "k")
    check_dw(host(dw), d)


def test_gradients_by_differences():
    """The gradients of sum(c * out) against differences of the products themselves, one value moved at a time.

    A value v moves by a quarter of itself (exact in bf16), so a row of out moves by c v w / 4 with the errors of two
    bf16 roundings, 2^-8 of each term of the sum."""
    K, N = 40, 24
    d = case([9, 0, 14], K, N, False, 11)
    dx, dw = filled((d["rows"], K)), filled((3, N, K), torch.float32)
    B.moe_product_dx(d["dy_dev"], d["w_dev"], dx, expert_offsets=d["off_dev"])
    B.moe_product_dw(d["dy_dev"], d["x_dev"], dw, expert_offsets=d["off_dev"])
    dx, dw = host(dx), host(dw)

    def loss(x, w):
        y = filled((d["rows"], N))
        B.moe_product(x, w, y, expert_offsets=d["off_dev"])
        terms = (host(y) * d["dy"])[:d["end"]]
        return terms.sum(1), np.abs(terms).sum(1)

    base, size = loss(d["x_dev"], d["w_dev"])
    for i, k in ((0, 3), (8, 39), (9, 0), (22, 17)):
        x = d["x_dev"].clone()
        x[i, k] *= 1.25
        step = float(x[i, k].double() - d["x_dev"][i, k].double())
        moved, more = loss(x, d["w_dev"])
        assert abs((moved[i] - base[i]) - dx[i, k] * step) <= 2.0 ** -8 * (size[i] + more[i] + abs(dx[i, k] * step))
    for e, n, k in ((0, 5, 7), (2, 23, 39)):
        w = d["w_dev"].clone()
        w[e, n, k] *= 1.25
        step = float(w[e, n, k].double() - d["w_dev"][e, n, k].double())
        moved, more = loss(d["x_dev"], w)
        assert abs((moved - base).sum() - dw[e, n, k] * step) <= 2.0 ** -8 * (size + more).sum()


def test_other_stream_and_repeats_give_the_same_bits():
    d = case([200, 60, 1, 439, 1300], 512, 392, True, 4)

    def all_three(stream=None):
        y, dx, dw = filled((d["rows"], 392)), filled((d["rows"], 512)), filled((5, 392, 512), torch.float32)
        torch.cuda.synchronize()
        B.moe_product(d["x_dev"], d["w_dev"], y, row_index=d["index_dev"], expert_offsets=d["off_dev"], stream=stream)
        B.moe_product_dx(d["dy_dev"], d["w_dev"], dx, expert_offsets=d["off_dev"], stream=stream)
        B.moe_product_dw(d["dy_dev"], d["x_dev"], dw, row_index=d["index_dev"], expert_offsets=d["off_dev"], stream=stream)
        torch.cuda.synchronize()
        return y, dx, dw

    first = all_three()
    for _ in range(3):
        for a, b in zip(first, all_three(torch.cuda.Stream())):
            assert torch.equal(a, b)


def test_tensors_past_4_gib():
    """The last expert's weights, the last rows, and the last expert's gradient."""
    K, N, E, rows = 4096, 4096, 160, 40
    w = torch.zeros((E, N, K), dtype=torch.bfloat16, device="cuda")
    w[E - 1] = 1
    x = torch.ones((rows, K), dtype=torch.bfloat16, device="cuda")
    off = torch.zeros(E + 1, dtype=torch.int32)
    off[E] = rows
    off = off.cuda()
    out = torch.zeros((rows, N), dtype=torch.bfloat16, device="cuda")
    B.moe_product(x, w, out, expert_offsets=off)
    assert bool((out == 4096).all())
    out.zero_()
    B.moe_product_dx(x, w, out, expert_offsets=off)
    assert bool((out == 4096).all())
    B.moe_product_dw(x, x, w, expert_offsets=off)      # w is the gradient now
    assert bool((w[E - 1] == rows).all()) and not bool(w[:E - 1].any())
    del w
    rows = 600000
    x = torch.zeros((rows, K), dtype=torch.bfloat16, device="cuda")
    x[rows - 1] = 1
    w = torch.ones((1, 8, K), dtype=torch.bfloat16, device="cuda")
    out = torch.zeros((rows, 8), dtype=torch.bfloat16, device="cuda")
    B.moe_product(x, w, out)
    assert bool((out[rows - 1] == 4096).all()) and float(out[:rows - 1].abs().max()) == 0.0
    dw = torch.zeros((1, 8, K), device="cuda")
    B.moe_product_dw(out, x, dw)
    assert bool((dw == 4096).all())
    x.zero_()
    B.moe_product_dx(out, w, x)
    assert bool((x[rows - 1] == 8 * 4096).all()) and not bool(x[:rows - 1].any())


@pytest.mark.parametrize("rows,K,N", [(2, 8, 8), (70, 264, 72), (600, 512, 256)])
def test_an_index_into_no_rows(rows, K, N):
    """Every entry of row_index is outside: NaN, and nothing is read past a tensor."""
    x = torch.zeros((0, K), dtype=torch.bfloat16, device="cuda")
    index = torch.zeros(rows, dtype=torch.int32, device="cuda")
    g = torch.Generator().manual_seed(0)
    w, dy = torch.randn((1, N, K), generator=g).to(torch.bfloat16).cuda(), torch.randn((rows, N), generator=g).to(torch.bfloat16).cuda()
    y, dw = filled((rows, N)), filled((1, N, K), torch.float32)
    B.moe_product(x, w, y, row_index=index)
    B.moe_product_dw(dy, x, dw, row_index=index)
    assert bool(y.isnan().all()) and bool(dw.isnan().all())


def test_no_rows():
    w, none = filled((2, 16, 8)), torch.zeros((0, 8), dtype=torch.bfloat16, device="cuda")
    off, dy = torch.zeros(3, dtype=torch.int32, device="cuda"), torch.zeros((0, 16), dtype=torch.bfloat16, device="cuda")
    B.moe_product(none, w, dy, expert_offsets=off)
    B.moe_product_dx(dy, w, none, expert_offsets=off)
    dw = filled((2, 16, 8), torch.float32)
    B.moe_product_dw(dy, none, dw, expert_offsets=off, accumulate=True)
    assert bool((dw == SENTINEL).all())
    B.moe_product_dw(dy, none, dw, expert_offsets=off)
    assert not bool(dw.any())
