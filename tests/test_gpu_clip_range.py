"""Clipping by scales far below fp32's range of normal values, against 64 bits.

The scale is rounded to 24 bits and so is its product with a value (2^-24 each; results below the type's normal values by
half of its smallest one), and a bf16 result once more, by 2^-8.
"""
import math

import numpy as np
import pytest

from paper_2607_19539_amd import binding as B
from tests.gpu_helpers import log

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

LARGE = 1.7 * 2.0 ** 126


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("max_norm", [1e-1, 1e-5, 1e-12, 3e-20, 7e-27, 2e-31, 1.3e-34, 2e-35, 7.7e-37, 1.2e-38, 3e-40, 5e-43, 1.4e-45, 0.0])
def test_a_large_norm_and_a_small_limit(max_norm, in_place, dtype):
    log(f"clip to {max_norm} in place {in_place} {dtype}")
    v = torch.tensor([LARGE, -LARGE / 3, 2.0 ** 100, 1.1 * 2.0 ** 60, -1.0, 2.0 ** -20, 0.0, -LARGE * 0.9] * 40, dtype=torch.float64)
    v[300:] = 0
    v[8:] *= 2.0 ** -40
    t = v.to(dtype).cuda()
    before = t.double().cpu()
    out = t if in_place else torch.full_like(t, 7.0)
    total, norm = torch.zeros(1, dtype=torch.float64, device="cuda"), torch.zeros(1, device="cuda")
    B.moe_squares([t], total)
    B.moe_clip([t], total, max_norm, out=None if in_place else [out], norm=norm)
    torch.cuda.synchronize()
    limit = float(np.float32(max_norm))
    root = math.sqrt(math.fsum(float(x) ** 2 for x in before))
    want = before * (limit / root)
    rounding = 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -24
    least = 2.0 ** -134 if dtype == torch.bfloat16 else 2.0 ** -150
    off = (out.double().cpu() - want).abs() - (rounding + 2.0 ** -23) * want.abs() - (least + 2.0 ** -150)
    assert float(off.max()) <= 0, (float(off.max()), out[:8].tolist(), want[:8].tolist())
    assert abs(float(norm) - root) <= 2.0 ** -23 * root
