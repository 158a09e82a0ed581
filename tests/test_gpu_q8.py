"""The 8-bit products against whole-number sums in 64 bits.

The integer sums are exact, so a product differs from the definition by the roundings of the sum to fp32, of the
two scales' product and of their product (3 units of 2^-24), and by the rounding to bf16 (2^-8).  The gated
activation adds an exponential of g, whose error grows with |g|, below 2^-16 for |g| up to 60.
"""
import ctypes

import numpy as np
import pytest

from paper_2607_19539_amd import binding as B
from tests.gpu_helpers import log

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

REL = 2.0 ** -8 + 2.0 ** -15
SENTINEL = -4096.0


def make(rng, n, K, N, E, wide=False):
    lo = -128 if wide else -127
    x = rng.integers(lo, 128, (n, K), dtype=np.int8)
    xs = (rng.random(n) + 0.5).astype(np.float32) / 64
    # Scales that leave g between about -8 and 8 (products of K terms of size 73 each).
    ws = ((rng.random((2, E, N)) + 0.5) * (32.0 / 73.0 ** 2 / K ** 0.5 * 8)).astype(np.float32)
    w = rng.integers(lo, 128, (2, E, N, K), dtype=np.int8)
    return x, xs, w, ws


def reference(x, xs, w, ws, off, index, rows, gated):
    """[rows, N] float64; NaN rows where the index has none, SENTINEL past the last expert's rows."""
    N = w.shape[2]
    out = np.full((rows, N), SENTINEL)
    for e in range(w.shape[1]):
        lo, hi = (0, rows) if off is None else (off[e], off[e + 1])
        r = np.arange(lo, hi) if index is None else index[lo:hi]
        ok = (r >= 0) & (r < x.shape[0])
        r = np.where(ok, r, 0)
        if lo == hi:
            continue
        v = []
        for i in range(2 if gated else 1):
            acc = x[r].astype(np.float64) @ w[i, e].astype(np.float64).T   # below 2^53: exact
            v.append(acc * xs[r].astype(np.float64)[:, None] * ws[i, e].astype(np.float64))
        y = v[0] / (1 + np.exp(-v[0])) * v[1] if gated else v[0]
        y[~ok] = np.nan
        out[lo:hi] = y
    return out


def run(x, xs, w, ws, off, index, rows, gated, stream=None):
    d = lambda a: None if a is None else torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
    out = torch.full((rows, w.shape[2]), SENTINEL, dtype=torch.bfloat16, device="cuda")
    kw = dict(row_index=d(index), expert_offsets=d(off), stream=stream)
    args = (d(x), d(xs), d(w[0]), d(ws[0]))
    more = (d(w[1]), d(ws[1]))
    torch.cuda.synchronize()
    if gated:
        B.moe_q8_gated(*args, *more, out, **kw)
    else:
        B.moe_q8_product(*args, out, **kw)
    torch.cuda.synchronize()
    return out.float().cpu().numpy().astype(np.float64)


def check(got, want):
    assert np.array_equal(np.isnan(got), np.isnan(want))
    fine = ~np.isnan(want)
    assert np.array_equal(got[fine] == SENTINEL, want[fine] == SENTINEL)
    off = np.abs(got[fine] - want[fine])
    # Subnormal sums aside (e^-g of a very negative g), within the roundings.
    assert np.all(off <= REL * np.abs(want[fine]) + 1e-30), float((off / np.maximum(np.abs(want[fine]), 1e-30)).max())


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("rows", [1, 2, 15, 16, 17, 33, 64, 65, 130, 257, 513])
@pytest.mark.parametrize("K,N", [(16, 8), (48, 24), (64, 64), (112, 40), (128, 128), (144, 136), (320, 264), (1040, 520)])
def test_one_matrix(K, N, rows, gated):
    rng = np.random.default_rng(K * 1000 + N * 10 + rows)
    x, xs, w, ws = make(rng, rows, K, N, 1)
    check(run(x, xs, w, ws, None, None, rows, gated), reference(x, xs, w, ws, None, None, rows, gated))


COUNTS = {
    "empty_between": [0, 5, 0, 0, 17, 1, 0], "ones": [1, 1, 1, 1], "one_busy": [0, 0, 300, 0],
    "ragged": [3, 64, 65, 128, 129, 31], "large": [256, 1, 257, 300, 0, 90], "none": [0, 0, 0],
    "many": [i % 5 for i in range(200)],
}


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("K,N", [(64, 72), (176, 256), (512, 320)])
@pytest.mark.parametrize("gather", [False, True])
@pytest.mark.parametrize("counts", list(COUNTS), ids=str)
def test_experts(counts, gather, K, N, gated):
    c = COUNTS[counts]
    log(f"q8 experts {counts} gather={gather} K={K} N={N} gated={gated}")
    rng = np.random.default_rng(len(c) * 100 + K + gather)
    off = np.concatenate([[0], np.cumsum(c)]).astype(np.int32)
    rows = int(off[-1]) + 3                       # three rows that belong to nobody
    n = rows if not gather else max(1, rows // 2)
    x, xs, w, ws = make(rng, n, K, N, len(c))
    index = None
    if gather:
        index = rng.integers(0, n, rows).astype(np.int32)
        index[off[-1]:] = -1
        if off[-1] > 4:
            index[2], index[4] = -1, n
    check(run(x, xs, w, ws, off, index, rows, gated), reference(x, xs, w, ws, off, index, rows, gated))


@pytest.mark.parametrize("rows", [2, 40, 300])
def test_longest_sums_do_not_overflow(rows):
    """The largest sums there are: 131056 products of -128 * 127, and of both signs."""
    K, N = 131056, 8
    x = np.full((rows, K), -128, np.int8)
    x[rows // 2:] = 127
    w = np.full((2, 1, N, K), 127, np.int8)
    w[:, :, 3] = -128
    xs, ws = np.full(rows, 2.0 ** -10, np.float32), np.full((2, 1, N), 2.0 ** -14, np.float32)
    check(run(x, xs, w, ws, None, None, rows, False), reference(x, xs, w, ws, None, None, rows, False))


@pytest.mark.parametrize("rows", [3, 100, 400])
def test_scales_that_are_not_finite(rows):
    """A row quantised from a NaN has a NaN scale: its outputs are NaN, the others untouched by it."""
    rng = np.random.default_rng(rows)
    x, xs, w, ws = make(rng, rows, 128, 64, 1)
    xs[1] = np.nan
    x[1] = 0
    got = run(x, xs, w, ws, None, None, rows, False)
    assert np.isnan(got[1]).all() and not np.isnan(np.delete(got, 1, 0)).any()


def test_offsets_outside_the_rows_are_cut():
    """Offsets past the rows, or that fall, reach no memory outside out."""
    rng = np.random.default_rng(2)
    x, xs, w, ws = make(rng, 50, 64, 32, 3)
    got = run(x, xs, w, ws, np.array([0, 10, 5, 1000], np.int32), None, 50, False)
    want = reference(x, xs, w, ws, np.array([0, 10, 10, 50]), None, 50, False)
    check(got, want)


@pytest.mark.parametrize("gated", [False, True])
def test_other_stream_and_repeats_give_the_same_bits(gated):
    rng = np.random.default_rng(4)
    off = np.array([0, 200, 260, 261, 700], np.int32)
    x, xs, w, ws = make(rng, 700, 512, 392, 4)
    a = run(x, xs, w, ws, off, None, 700, gated)
    b = run(x, xs, w, ws, off, None, 700, gated, stream=torch.cuda.Stream())
    assert np.array_equal(a, b)


def test_rows_of_a_large_tensor():
    """Weights and rows past 4 GiB: the last expert's, and the last rows."""
    K, N, E, rows = 4096, 4096, 300, 40
    w = torch.zeros((E, N, K), dtype=torch.int8, device="cuda")
    w[E - 1] = 1
    x = torch.ones((rows, K), dtype=torch.int8, device="cuda")
    off = torch.zeros(E + 1, dtype=torch.int32)
    off[E] = rows
    out = torch.zeros((rows, N), dtype=torch.bfloat16, device="cuda")
    B.moe_q8_product(x, torch.ones(rows, device="cuda"), w, torch.ones((E, N), device="cuda"), out, expert_offsets=off.cuda())
    assert bool((out == 4096).all())
    del w
    rows = 1100000
    x = torch.zeros((rows, K), dtype=torch.int8, device="cuda")
    x[rows - 1] = 1
    w = torch.ones((1, 8, K), dtype=torch.int8, device="cuda")
    out = torch.zeros((rows, 8), dtype=torch.bfloat16, device="cuda")
    B.moe_q8_product(x, torch.ones(rows, device="cuda"), w, torch.ones((1, 8), device="cuda"), out)
    assert bool((out[rows - 1] == 4096).all()) and float(out[:rows - 1].abs().max()) == 0.0


KINDS = ["slim1", "slim2", "tiles64", "tiles128", "tiles256"]


class Q8Args(ctypes.Structure):
    """The launchers' arguments (csrc/ops.hpp)."""
    _fields_ = [(n, ctypes.c_void_p) for n in ("x", "xs", "index", "offsets", "w", "w3", "ws", "ws3", "out")] + \
               [("x_rows", ctypes.c_int64), ("rows", ctypes.c_int64), ("experts", ctypes.c_int32), ("K", ctypes.c_int32),
                ("N", ctypes.c_int32)]


def run_kind(kind, x, xs, w, ws, off, index, rows, gated):
    """One of the kernels that launch_q8 chooses among, whatever it would choose."""
    launch = B.load()._ZN3moe14launch_q8_kindENS_6Q8KindERKNS_6Q8ArgsEbP12ihipStream_t
    launch.argtypes, launch.restype = [ctypes.c_int, ctypes.POINTER(Q8Args), ctypes.c_bool, ctypes.c_void_p], ctypes.c_int
    t = [None if a is None else torch.from_numpy(np.ascontiguousarray(a)).cuda()
         for a in (x, xs, index, off, w[0], w[1], ws[0], ws[1])]
    out = torch.full((rows, w.shape[2]), SENTINEL, dtype=torch.bfloat16, device="cuda")
    torch.cuda.synchronize()
    args = Q8Args(*[None if a is None else a.data_ptr() for a in t], out.data_ptr(), x.shape[0], rows, w.shape[1],
                  x.shape[1], w.shape[2])
    assert launch(KINDS.index(kind), ctypes.byref(args), gated, torch.cuda.current_stream().cuda_stream) == 0
    torch.cuda.synchronize()
    return out.float().cpu().numpy().astype(np.float64)


# Rows of each expert (or of one matrix), K, N: every height of the whole tiles, several sets of items for each of
# their workgroups, more experts than a wave has lanes; K of one chunk, of one step, of a few, with every kind of end.
SIZES = [
    (1, 16, 8), (300, 48, 72), (257, 112, 256), (520, 128, 264), (65, 144, 520), (193, 256, 136), (700, 272, 1032),
    (260, 384, 40), (129, 400, 264), (64, 640, 520), (33, 1936, 264),
    ([0, 5, 0, 0, 17, 1, 0], 64, 72), ([3, 64, 65, 128, 129, 31, 192, 193, 256, 257, 0, 1], 176, 520),
    ([1300, 700, 2000, 0, 1096, 33, 64, 65, 128, 129, 1, 192, 193, 256, 257, 600], 272, 3080),
    ([i % 5 for i in range(200)], 80, 136), ([i * 37 % 290 for i in range(130)], 144, 520),
]


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("gather", [False, True])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("counts,K,N", SIZES, ids=lambda v: str(v)[:24])
def test_each_kernel(counts, K, N, kind, gather, gated):
    log(f"q8 {kind} {str(counts)[:60]} K={K} N={N} gather={gather} gated={gated}")
    rng = np.random.default_rng(K + N + gather)
    grouped = not isinstance(counts, int)
    c = counts if grouped else [counts]
    off = np.concatenate([[0], np.cumsum(c)]).astype(np.int32)
    rows = int(off[-1]) + (5 if grouped else 0)
    n = max(1, rows // 3) if gather else rows
    x, xs, w, ws = make(rng, n, K, N, len(c))
    index = None
    if gather:
        index = rng.integers(0, n, rows).astype(np.int32)
        index[rows // 2] = -5
        index[rows - 1] = n
    o = off if grouped else None
    check(run_kind(kind, x, xs, w, ws, o, index, rows, gated), reference(x, xs, w, ws, o, index, rows, gated))


@pytest.mark.parametrize("c,N", [
    (4100, 4096), (4353, 4352), (4600, 4600), (5000, 5000),          # 16, 50, 68 and 144 tiles in the second round
    ([600, 0, 1500, 257, 1, 1800], 4096), ([4096], 4096)])
def test_parts_of_the_last_round(c, N):
    """More tiles than compute units: those of the last round are cut by rows, into as many parts as fit."""
    rng = np.random.default_rng(17)
    grouped = not isinstance(c, int)
    c = c if grouped else [c]
    off = np.concatenate([[0], np.cumsum(c)]).astype(np.int32)
    x, xs, w, ws = make(rng, int(off[-1]), 48, N, len(c))
    o = off if grouped else None
    check(run_kind("tiles256", x, xs, w, ws, o, None, int(off[-1]), False), reference(x, xs, w, ws, o, None, int(off[-1]), False))


@pytest.mark.parametrize("rows,grouped,E,K,N,gated,kind", [
    (1, False, 1, 4096, 4096, False, "slim1"), (8, False, 1, 7168, 1024, False, "slim1"),
    (96, True, 64, 1408, 2048, False, "slim2"), (96, True, 64, 2048, 1408, True, "slim1"),
    (300, False, 1, 2000, 3000, False, "tiles64"), (16, False, 1, 4096, 14336, False, "tiles64"),
    (256, False, 1, 4096, 14336, False, "tiles128"), (1024, False, 1, 4096, 4096, False, "tiles128"),
    (4096, False, 1, 4096, 4096, False, "tiles256"), (49152, True, 64, 2048, 1408, True, "tiles256"),
    (8192, True, 8, 14336, 4096, False, "tiles256")])
def test_the_kernel_chosen(rows, grouped, E, K, N, gated, kind):
    f = B.load()._ZN3moe7q8_kindElbiiib
    f.argtypes, f.restype = [ctypes.c_int64, ctypes.c_bool] + [ctypes.c_int32] * 3 + [ctypes.c_bool], ctypes.c_int
    assert KINDS[f(rows, grouped, E, K, N, gated)] == kind
