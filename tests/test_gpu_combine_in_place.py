"""The combine's gradient written over the rows that it reads: the same bits as into a tensor of its own."""
import numpy as np
import pytest

from paper_2607_19539_amd import binding as B
from tests.gpu_helpers import log
from tests.test_gpu_combine_backward import bf16, check

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


def slots(rng, T, k):
    """A row for each choice, but for tokens that name one of theirs two or more times, and slots that are not there."""
    slot = rng.permutation(T * k).astype(np.int32).reshape(T, k)
    if k > 1:
        slot[::2, k - 1] = slot[::2, 0]
        slot[1::4] = slot[1::4, :1]
    if k > 3:
        slot[::3, 1], slot[2::5, 2], slot[2::5, k - 2] = -1, slot[2::5, 3], T * k
    return slot


# One wave a choice and four, a choice alone, 64 of them, many tokens.
@pytest.mark.parametrize("T,k,H", [(1, 1, 8), (1, 64, 520), (1, 64, 7168), (5, 2, 24), (64, 8, 7168), (128, 8, 4104), (129, 8, 4104), (3, 5, 65536),
                                   (777, 6, 2048), (4000, 2, 64)])
def test_drecv_over_recv(T, k, H):
    log(f"combine backward in place {T} x {k} x {H}")
    rng = np.random.default_rng(T + k + H)
    slot = slots(rng, T, k)
    gate = rng.random((T, k)).astype(np.float32)
    dout, recv = bf16(rng, T, H), bf16(rng, T * k, H)
    check(dout, recv, slot, gate)
    d, s, g = dout[1], torch.from_numpy(slot).cuda(), torch.from_numpy(gate).cuda()
    apart, dgate = recv[1].clone(), torch.full((T, k), -1.0, device="cuda")
    B.moe_combine_backward(d, recv[1], s, g, drecv=apart, dgate=dgate)
    alone = torch.full((T, k), -2.0, device="cuda")
    B.moe_combine_backward(d, recv[1], s, g, dgate=alone)
    assert torch.equal(dgate, alone)
    for with_dgate in (True, False):
        rows, again = recv[1].clone(), torch.full((T, k), -3.0, device="cuda")
        B.moe_combine_backward(d, rows, s, g, drecv=rows, dgate=again if with_dgate else None)
        assert torch.equal(rows, apart)
        assert torch.equal(again, dgate if with_dgate else torch.full_like(again, -3.0))
