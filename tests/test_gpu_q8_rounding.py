"""Rows to 8 bits are rounded as documented, half steps to the even one: bf16 rows, so that 127 y / max|y| is a ratio
of small whole numbers and the step is known exactly."""
import numpy as np
import pytest

from paper_2607_19539_amd import binding as B
from tests.gpu_helpers import log

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


def steps(y):
    """rne(127 y / max|y|) of float64 rows that bf16 holds, in whole numbers."""
    top = np.abs(y).max(1, keepdims=True)
    unit = np.exp2(np.floor(np.log2(top)) - 30)       # a value that this cuts is below 2^-22 of the row's largest
    a, m = np.trunc(np.abs(y) / unit).astype(np.int64) * 254, np.trunc(top / unit).astype(np.int64)
    q, rest = (a + m) // (2 * m), (a + m) % (2 * m)
    q -= (rest == 0) & (q % 2 == 1)
    return (np.sign(y) * q).astype(np.int8)


def run(y):
    x = torch.from_numpy(y.astype(np.float32)).to(torch.bfloat16)
    assert np.array_equal(x.double().numpy(), y)
    q, s = torch.full(y.shape, 99, dtype=torch.int8, device="cuda"), torch.full((len(y),), -7.0, device="cuda")
    B.moe_q8_rows(x.cuda(), q, s)
    top = np.abs(y).max(1).astype(np.float32)
    assert np.array_equal(s.cpu().numpy(), top / np.float32(127))
    return q.cpu().numpy()


@pytest.mark.parametrize("exponent", [-106, -100, -60, -7, 0, 5, 93, 94, 118])
def test_half_steps_go_to_the_even_one(exponent):
    """max|y| = 127 units, and values of (n + 1/2) units, of 2^exponent, 2 and 4 times as much."""
    log(f"q8 half steps 2^{exponent}")
    n = np.arange(-127, 127) + 0.5
    rows = []
    for size in (1.0, 0.5, 0.25):
        y = np.zeros(320)
        y[7], y[60:60 + len(n)] = 127.0, n
        rows.append(y * size * 2.0 ** (exponent + 2))
    y = np.stack(rows)
    assert np.any(steps(y) != np.round(y / np.abs(y).max(1, keepdims=True) * 127 + 1e-9))   # ties are there
    assert np.array_equal(run(y), steps(y))


@pytest.mark.parametrize("exponent", [-107, -99, 0, 92, 93, 119])
def test_every_significand_by_every_largest(exponent):
    """max|y| of each of the 128 significands, y of each in nine octaves below it."""
    log(f"q8 significands 2^{exponent}")
    sig = np.arange(128, 256, dtype=np.float64)
    below = (sig[None] * np.exp2(-np.arange(9))[:, None]).reshape(-1)
    y = np.zeros((128, 1 + len(below) + 7))
    y[:, 0] = -sig
    y[:, 1:1 + len(below)] = np.where(below[None] <= sig[:, None], below[None], 0.0)
    y *= 2.0 ** exponent
    assert np.array_equal(run(y), steps(y))
