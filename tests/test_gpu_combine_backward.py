"""The combine's gradient against 64 bits, and against differences of the combine itself.

drecv is one fp32 product rounded to bf16 (2^-24 and 2^-8; a row that a token names twice has a rounded sum of gates
besides).  dgate is a sum of H products in fp32: at most H 2^-23 of the sum of their magnitudes.
"""
import numpy as np
import pytest

from paper_2607_19539_amd import binding as B
from tests.gpu_helpers import log

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

SENTINEL = -4096.0


def bf16(rng, *shape):
    t = torch.from_numpy(rng.standard_normal(shape).astype(np.float32)).to(torch.bfloat16)
    return t.double().numpy(), t.cuda()


def check(dout, recv, slot, gate, want_drecv=True, want_dgate=True, stream=None):
    (d64, d), (r64, r) = dout, recv
    T, k = slot.shape
    rows, H = r64.shape
    drecv = torch.full((rows, H), SENTINEL, dtype=torch.bfloat16, device="cuda") if want_drecv else None
    dgate = torch.full((T, k), SENTINEL, device="cuda") if want_dgate else None
    torch.cuda.synchronize()
    B.moe_combine_backward(d, r, torch.from_numpy(slot).cuda(), torch.from_numpy(gate).cuda(), drecv=drecv, dgate=dgate, stream=stream)
    torch.cuda.synchronize()
    ok = (slot >= 0) & (slot < rows)
    if want_dgate:
        at = np.concatenate([r64, np.zeros((1, H))])[np.where(ok, slot, rows)]
        want, size = np.einsum("th,tkh->tk", d64, at), np.einsum("th,tkh->tk", np.abs(d64), np.abs(at))
        assert np.all(np.abs(dgate.double().cpu().numpy() - want) <= H * 2.0 ** -23 * size)
    if want_drecv:
        sums = {}
        for t in range(T):
            for j in range(k):
                if ok[t, j]:
                    sums.setdefault(int(slot[t, j]), [t, 0.0])[1] += float(gate[t, j])
        want = np.full((rows, H), SENTINEL)
        for row, (t, g) in sums.items():
            want[row] = g * d64[t]
        got = drecv.double().cpu().numpy()
        assert np.all(np.abs(got - want) <= (2.0 ** -8 + 2.0 ** -20) * np.abs(want) + 1e-38)


@pytest.mark.parametrize("T,k,H", [(1, 1, 8), (1, 8, 7168), (3, 2, 24), (5, 3, 520), (64, 8, 1024), (777, 6, 264), (130, 4, 4104), (9, 64, 2048),
                                   (2, 3, 65536), (4000, 2, 64)])
def test_combine_backward(T, k, H):
    log(f"combine backward {T} x {k} x {H}")
    rng = np.random.default_rng(T + k + H)
    slot = rng.permutation(T * k).astype(np.int32).reshape(T, k)
    gate = rng.random((T, k)).astype(np.float32)
    dout, recv = bf16(rng, T, H), bf16(rng, T * k, H)
    check(dout, recv, slot, gate)
    check(dout, recv, slot, gate, want_dgate=False)
    check(dout, recv, slot, gate, want_drecv=False, stream=torch.cuda.Stream())


def test_slots_that_are_not_there():
    rng = np.random.default_rng(3)
    slot = rng.permutation(60).astype(np.int32).reshape(20, 3)
    slot[4, 1], slot[7], slot[0, 0], slot[19, 2] = -1, -1, 60, 2 ** 31 - 1
    check(bf16(rng, 20, 136), bf16(rng, 60, 136), slot, rng.random((20, 3)).astype(np.float32))
    check(bf16(rng, 20, 136), bf16(rng, 0, 136), slot, rng.random((20, 3)).astype(np.float32))


def test_a_row_that_a_token_names_more_than_once():
    rng = np.random.default_rng(4)
    slot = np.array([[0, 0, 1, 0], [2, 3, 3, 2], [4, 5, 6, 7], [-1, 8, -1, 8]], np.int32)
    check(bf16(rng, 4, 520), bf16(rng, 9, 520), slot, rng.random((4, 4)).astype(np.float32))


@pytest.mark.parametrize("T,k,H", [(1, 1, 4096), (128, 8, 4104), (129, 8, 4104), (60, 3, 8200), (5, 7, 16384), (64, 16, 4088)])
def test_long_rows_of_few_and_of_many_choices(T, k, H):
    """One wave a choice and four, with slots that are not there and rows that a token names more than once."""
    log(f"combine backward, long rows {T} x {k} x {H}")
    rng = np.random.default_rng(T * k + H)
    slot = rng.permutation(T * k).astype(np.int32).reshape(T, k)
    if k > 2:
        slot[::3, 1], slot[1::3, 2], slot[T - 1, k - 1] = -1, slot[1::3, 0], T * k
    gate = rng.random((T, k)).astype(np.float32)
    dout, recv = bf16(rng, T, H), bf16(rng, T * k, H)
    check(dout, recv, slot, gate)
    check(dout, recv, slot, gate, want_drecv=False)
    check(dout, recv, slot, gate, want_dgate=False, stream=torch.cuda.Stream())


def test_gradients_by_differences():
    """Against moe_combine: out moves by gate times what recv moves, and by recv times what gate moves, off by two
    roundings of out to bf16, 2^-8 each."""
    rng = np.random.default_rng(5)
    T, k, H = 6, 3, 64
    slot = torch.from_numpy(rng.permutation(T * k).astype(np.int32).reshape(T, k)).cuda()
    gate = torch.from_numpy(rng.random((T, k)).astype(np.float32)).cuda()
    (d64, dout), (_, recv) = bf16(rng, T, H), bf16(rng, T * k, H)
    drecv, dgate = torch.empty_like(recv), torch.empty_like(gate)
    B.moe_combine_backward(dout, recv, slot, gate, drecv=drecv, dgate=dgate)

    def loss(r, g):
        out = torch.empty_like(dout)
        B.moe_combine(r, slot, g, out)
        terms = out.double().cpu().numpy() * d64
        return terms.sum(), np.abs(terms).sum(1)

    base, size = loss(recv, gate)
    for t, j, h in ((0, 0, 5), (5, 2, 63), (3, 1, 0)):
        row = int(slot[t, j])
        moved = recv.clone()
        moved[row, h] += 4.0
        step = float(moved[row, h].double() - recv[row, h].double())
        got, more = loss(moved, gate)
        assert abs(got - base - float(drecv[row, h]) * step) <= 2.0 ** -8 * (size[t] + more[t]) + 2.0 ** -8 * abs(float(drecv[row, h]) * step)
        moved = gate.clone()
        moved[t, j] += 1.0
        step = float(moved[t, j].double() - gate[t, j].double())
        got, more = loss(recv, moved)
        assert abs(got - base - float(dgate[t, j]) * step) <= 2.0 ** -8 * (size[t] + more[t])
