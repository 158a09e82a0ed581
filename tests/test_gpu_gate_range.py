"""The gated activation's gradient where a factor is as large as bf16 holds, against 64 bits (bounds: test_gpu_gate.py).

s (1 + g (1 - s)) reaches 1.1 near g = 2.4, so its product with one factor alone may pass fp32's range where the
gradient, which has the other factor as well, does not.
"""
import numpy as np
import pytest

from tests.test_gpu_gate import check, run

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

LARGEST = 255 * 2.0 ** 120  # of bf16


@pytest.mark.parametrize("u,da", [(LARGEST, 1e-3), (3.2e38, 1e-30), (1e-3, -LARGEST), (-LARGEST, 0.5), (1.0, LARGEST), (LARGEST, 2.0 ** -133),
                                  (2.0 ** -133, 3.1e38), (LARGEST, LARGEST), (2.0 ** -133, 2.0 ** -133), (LARGEST, 0.0)])
def test_the_largest_and_the_smallest_factors(u, da):
    """Every bf16 value of g."""
    bits = np.arange(65536, dtype=np.uint16)
    g = torch.from_numpy(bits.view(np.int16)).view(torch.bfloat16).double().numpy().reshape(64, 1024)
    check(*run(g, np.full_like(g, u), np.full_like(g, da)))


def test_a_finite_gradient_is_not_an_infinity():
    g = np.full((1, 8), 2.40625)
    for u, da, want in ((3.2e38, 1e-3, 3.5e35), (1e-3, 3.2e38, 3.5e35)):
        _, dg, _, *_ = run(g, np.full_like(g, u), np.full_like(g, da))
        assert np.all(np.abs(dg - want) <= 0.02 * want)
