"""Rows taken through row_index out of nearly 4 GiB, by each kernel of the product and of the gradient by the weights.

The rows lie behind as much memory of other values, which an offset taken for a signed one would read instead.
"""
import ctypes

import pytest

from paper_2607_19539_amd import binding as B
from tests.gpu_helpers import log
from tests.test_gpu_product import KINDS, DwPlan, ProductArgs, ProductDwArgs, ptr

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

K, N, MOST = 8192, 64, (2 ** 32 - 1) // (2 * 8192)


@pytest.fixture(scope="module")
def far():
    """x of MOST rows, of which those an index names hold small whole numbers; the index; weights and gradients."""
    room = torch.full((2 * MOST, K), 100.0, dtype=torch.bfloat16, device="cuda")
    x = room[MOST:]
    g = torch.Generator().manual_seed(1)
    index = torch.cat([torch.tensor([MOST - 1, MOST // 2, MOST // 2 - 1, 0, MOST - 2]), torch.randint(MOST // 2, MOST, (595,), generator=g)])

    def whole(*shape):
        return torch.randint(-2, 3, shape, generator=g).to(torch.bfloat16).cuda()

    x[index.unique().cuda()] = whole(len(index.unique()), K)
    yield x, index.int().cuda(), whole(1, N, K), whole(600, N), x[index.cuda()].double()
    del room, x
    torch.cuda.empty_cache()


@pytest.mark.parametrize("kind", KINDS)
def test_product(far, kind):
    log(f"far rows, product {kind}")
    x, index, w, _, rows = far
    f = B.load()._ZN3moe19launch_product_kindENS_11ProductKindERKNS_11ProductArgsEbP12ihipStream_t
    f.argtypes, f.restype = [ctypes.c_int, ctypes.POINTER(ProductArgs), ctypes.c_bool, ctypes.c_void_p], ctypes.c_int
    out = torch.full((600, N), 7.0, dtype=torch.bfloat16, device="cuda")
    args = ProductArgs(ptr(x), ptr(index), None, ptr(w), ptr(out), MOST, 600, 1, K, N)
    assert f(KINDS.index(kind), ctypes.byref(args), False, torch.cuda.current_stream().cuda_stream) == 0
    want = rows @ w[0].double().t()
    assert torch.equal(out.double(), want.to(torch.bfloat16).double())


@pytest.mark.parametrize("tile,split", [(64, 1), (64, 4), (128, 1), (128, 2), (256, 1), (256, 3)])
def test_gradient_by_the_weights(far, tile, split):
    log(f"far rows, dw {tile} {split}")
    x, index, _, dy, rows = far
    f = B.load()._ZN3moe22launch_product_dw_planERKNS_6DwPlanERKNS_13ProductDwArgsEP12ihipStream_t
    f.argtypes, f.restype = [ctypes.POINTER(DwPlan), ctypes.POINTER(ProductDwArgs), ctypes.c_void_p], ctypes.c_int
    dw, parts = torch.full((1, N, K), 7.0, device="cuda"), torch.zeros((split, 1, N, K), device="cuda")
    args = ProductDwArgs(ptr(dy), ptr(x), ptr(index), None, ptr(dw), ptr(parts), MOST, 600, 1, K, N, 0, 0)
    assert f(ctypes.byref(DwPlan(tile, split)), ctypes.byref(args), torch.cuda.current_stream().cuda_stream) == 0
    assert torch.equal(dw[0].double(), dy.double().t() @ rows)
