"""A product of so many features that a workgroup for 16 of them each would be more than a launch takes."""
import math

import pytest

from paper_2607_19539_amd import binding as B

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


def test_gated_features_past_two_to_the_28():
    N, K = 2 ** 28 + 8, 16
    w1, w3 = (torch.ones((1, N, K), dtype=torch.int8, device="cuda") for _ in range(2))
    w1[0, N - 1], w3[0, N - 2] = 2, 3
    s1, s3 = torch.full((1, N), 0.125, device="cuda"), torch.full((1, N), 0.5, device="cuda")
    out = torch.zeros((1, N), dtype=torch.bfloat16, device="cuda")
    B.moe_q8_gated(torch.ones((1, K), dtype=torch.int8, device="cuda"), torch.ones(1, device="cuda"), w1, s1, w3, s3, out)
    for got, g, u in ((out[0, 0], 2, 8), (out[0, N - 1], 4, 8), (out[0, N - 2], 2, 24)):
        want = g / (1 + math.exp(-g)) * u
        assert abs(float(got) - want) <= (2.0 ** -8 + 2.0 ** -15) * want
    assert bool((out[0, :N - 2] == out[0, 0]).all())
