"""The 16-bit products and their gradients with as many rows as a call takes, 2^31 - 1 of 8 features (some 70 GB).

Nearly all rows are zeros and the others small whole numbers, so every sum is exact.
"""
import pytest

from paper_2607_19539_amd import binding as B
from tests.gpu_helpers import log

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

MOST = 2 ** 31 - 1


@pytest.fixture(autouse=True)
def room():
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 120e9:
        pytest.skip("the card has less than 120 GB free")
    yield
    torch.cuda.empty_cache()


def zeros(*shape, dtype=torch.bfloat16):
    return torch.zeros(shape, dtype=dtype, device="cuda")


def eight(start):
    return torch.arange(start, start + 8, device="cuda")


def marked(rows, first):
    """[rows, 8] zeros, but for some rows near the ends and where parts of the rows meet."""
    t, at = zeros(rows, 8), sorted({0, 1, 2 ** 26 - 1, 2 ** 26, rows // 2, rows - 101, rows - 100, rows - 65, rows - 64, rows - 2, rows - 1})
    for i, r in enumerate(at):
        t[r] = (eight(first + i) % 7 - 3).to(t.dtype)
    return t, at


def want_dw(dy, x, at):
    return sum(torch.outer(dy[r].double(), x[r].double()) for r in at)


@pytest.mark.parametrize("rows", [MOST, MOST - 64])
def test_gradient_by_the_weights_of_one_matrix(rows):
    log(f"dw of {rows} rows")
    (dy, at), (x, _) = marked(rows, 0), marked(rows, 3)
    want = want_dw(dy, x, at)
    dw = torch.full((1, 8, 8), 5.0, device="cuda")
    B.moe_product_dw(dy, x, dw)
    assert torch.equal(dw[0].double(), want)
    B.moe_product_dw(dy, x, dw, accumulate=True)
    assert torch.equal(dw[0].double(), 2 * want)


def test_gradient_by_the_weights_of_experts():
    """All rows but a few with one expert, the few with the last."""
    log("dw of experts")
    (dy, at), (x, _) = marked(MOST, 0), marked(MOST, 3)
    off = torch.tensor([0, MOST - 100, MOST - 100, MOST], dtype=torch.int32, device="cuda")
    dw = torch.full((3, 8, 8), 5.0, device="cuda")
    B.moe_product_dw(dy, x, dw, expert_offsets=off)
    want = [want_dw(dy, x, [r for r in at if r < MOST - 100]), zeros(8, 8).double(), want_dw(dy, x, [r for r in at if r >= MOST - 100])]
    assert torch.equal(dw.double(), torch.stack(want))


def test_gradient_by_the_weights_through_an_index():
    log("dw through an index")
    dy, at = marked(MOST, 0)
    x = zeros(16, 8)
    x[1:] = (torch.arange(15 * 8, device="cuda") % 5 - 2).view(15, 8).to(x.dtype)
    index = zeros(MOST, dtype=torch.int32)
    for i, r in enumerate(at):
        index[r] = 1 + i
    dw = torch.full((1, 8, 8), 5.0, device="cuda")
    B.moe_product_dw(dy, x, dw, row_index=index)
    assert torch.equal(dw[0].double(), sum(torch.outer(dy[r].double(), x[1 + i].double()) for i, r in enumerate(at)))


@pytest.mark.parametrize("experts", [1, 3])
def test_product_and_gradient_by_its_rows(experts):
    log(f"product and dx, {experts} experts")
    x, at = marked(MOST, 1)
    w = (torch.arange(experts * 64, device="cuda") % 5 - 2).view(experts, 8, 8).to(x.dtype)
    off = None if experts == 1 else torch.tensor([0, MOST - 100, MOST - 100, MOST], dtype=torch.int32, device="cuda")
    out = torch.full((MOST, 8), 5.0, dtype=torch.bfloat16, device="cuda")
    for call, side in ((lambda: B.moe_product(x, w, out, expert_offsets=off), 1), (lambda: B.moe_product_dx(x, w, out, expert_offsets=off), 0)):
        out.fill_(5.0)
        call()
        for r in at:
            e = experts - 1 if r >= MOST - 100 else 0
            assert torch.equal(out[r].double(), x[r].double() @ (w[e].double().t() if side else w[e].double())), r
            out[r] = 0
        assert not any(bool(out[i:i + 2 ** 28].any()) for i in range(0, MOST, 2 ** 28))
