"""The division of a sum over rows into parts and K steps, up to the most rows a call takes (no GPU)."""
import ctypes
import subprocess

import pytest

from tests.test_kernel_resources import CSRC

MOST = 2 ** 31 - 1
STEP = 64


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    d = tmp_path_factory.mktemp("parts")
    (d / "parts.cpp").write_text(
        '#include "row_parts.hpp"\n'
        'extern "C" int steps(int n) { return moe::steps_of(n); }\n'
        'extern "C" void part(int lo, int hi, int split, int p, int* out) {\n'
        '  const moe::RowPart r = moe::row_part(lo, hi, split, p);\n  out[0] = r.row0, out[1] = r.rows;\n}\n'
        'extern "C" int row(int step, int lane, int n) { return moe::row_of_step(step, lane, n); }\n')
    subprocess.run(["g++", "-std=c++17", "-O1", "-ftrapv", "-shared", "-fPIC", f"-I{CSRC}", str(d / "parts.cpp"), "-o", str(d / "parts.so")],
                   check=True, capture_output=True)
    return ctypes.CDLL(str(d / "parts.so"))


RANGES = [(0, 0), (0, 1), (7, 70), (0, 64), (0, 65), (100, 4196), (0, 2 ** 20 + 1), (0, MOST), (0, MOST - 62), (0, MOST - 63), (0, MOST - 64),
          (1, MOST), (MOST - 100, MOST), (MOST - 1, MOST), (MOST, MOST), (MOST - 2 ** 20, MOST), (2 ** 30, MOST)]


@pytest.mark.parametrize("split", [1, 2, 3, 4, 8, 16, 32])
@pytest.mark.parametrize("lo,hi", RANGES)
def test_the_parts_are_the_rows(lib, lo, hi, split):
    out, at = (ctypes.c_int * 2)(), lo
    steps = -(-(hi - lo) // STEP)
    each = -(-steps // split) * STEP
    for p in range(split):
        lib.part(lo, hi, split, p, out)
        want = min(each, hi - at)
        assert (out[0], out[1]) == (at, want), p
        at += want
    assert at == hi


@pytest.mark.parametrize("n", [1, 2, 63, 64, 65, 128, 1000, MOST - 64, MOST - 63, MOST - 62, MOST])
def test_steps_and_their_rows(lib, n):
    steps = -(-n // STEP)
    assert lib.steps(n) == steps
    # The last steps, and those that are asked for ahead of them.
    for step in {0, 1, steps // 2, max(steps - 2, 0), steps - 1, steps, steps + 1, steps + 17}:
        for lane in (0, 1, 31, 63):
            assert lib.row(step, lane, n) == min(min(step * STEP, max(n - STEP, 0)) + lane, n - 1), (step, lane)
    assert lib.row(steps - 1, 63, n) == n - 1
