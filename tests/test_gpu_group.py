"""The order of the routed rows by expert against a stable sort: whole numbers, equal."""
import numpy as np
import pytest

from paper_2607_19539_amd import binding as B
from tests.gpu_helpers import log

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


def reference(ids, E):
    T, k = ids.shape
    flat = ids.reshape(-1)
    ok = (flat >= 0) & (flat < E)
    order = np.argsort(np.where(ok, flat, E), kind="stable")[:ok.sum()]
    off = np.zeros(E + 1, np.int32)
    off[1:] = np.cumsum(np.bincount(flat[ok], minlength=E))
    row = np.full(T * k, -1, np.int32)
    row[:len(order)] = order // k
    slot = np.full(T * k, -1, np.int32)
    slot[order] = np.arange(len(order))
    return off, row, slot.reshape(T, k)


def run_group(ids, E, stream=None, workspace=None):
    T, k = ids.shape
    off = torch.full((E + 1,), -99, dtype=torch.int32, device="cuda")
    row = torch.full((T * k,), -99, dtype=torch.int32, device="cuda")
    slot = torch.full((T, k), -99, dtype=torch.int32, device="cuda")
    d = torch.from_numpy(np.ascontiguousarray(ids)).cuda()
    torch.cuda.synchronize()
    B.moe_group(d, E, off, row, slot, workspace=workspace, stream=stream)
    torch.cuda.synchronize()
    return off.cpu().numpy(), row.cpu().numpy(), slot.cpu().numpy()


@pytest.mark.parametrize("E", [1, 2, 8, 60, 64, 256, 1000, 1024])
@pytest.mark.parametrize("T,k", [(1, 1), (1, 7), (21, 3), (32, 2), (13, 5), (48, 8), (129, 8), (1024, 1), (700, 6),
                                 (1000, 8), (8193, 1), (9001, 7)])
@pytest.mark.parametrize("kind", ["uniform", "one", "dropped", "skewed"])
def test_group(T, k, E, kind):
    rng = np.random.default_rng(T * 31 + k * 7 + E)
    ids = rng.integers(0, E, (T, k))
    if kind == "one":
        ids[:] = E - 1
    elif kind == "dropped":
        ids[rng.random((T, k)) < 0.4] = -1
        ids[rng.random((T, k)) < 0.1] = E
        ids[T // 2:] = np.iinfo(np.int32).min
    elif kind == "skewed":
        ids = np.minimum(ids, rng.integers(0, E, (T, k))) // 2
    ids = ids.astype(np.int32)
    for got, want in zip(run_group(ids, E), reference(ids, E)):
        assert np.array_equal(got, want)


def test_group_of_nothing():
    off, row, slot = run_group(np.zeros((0, 4), np.int32), 16)
    assert off.tolist() == [0] * 17 and row.size == 0 and slot.size == 0
    off, row, slot = run_group(np.full((5000, 2), -1, np.int32), 300)
    assert not off.any() and np.all(row == -1) and np.all(slot == -1)


def test_group_large():
    """As many entries as a large batch routes, with a workspace of the caller's on a stream of its own."""
    rng = np.random.default_rng(1)
    T, k, E = 131072, 8, 256
    ids = rng.integers(0, E, (T, k)).astype(np.int32)
    need = B.load().moe_group_workspace(T * k, E)
    log(f"group {T} x {k}: workspace {need}")
    ws = torch.full((need,), 255, dtype=torch.uint8, device="cuda")
    for stream in (None, torch.cuda.Stream()):
        for got, want in zip(run_group(ids, E, stream, ws), reference(ids, E)):
            assert np.array_equal(got, want)
