"""The example layer: every operator in one pass, against the layer in fp32 with 16-bit weights, eager and from
a graph.

Rows and weights in 8 bits carry an error of half a step each, step = max / 127: for unit normal rows of some
hundred values (max about 3 to 4 standard deviations) step / sqrt(12) is about 0.008 of a standard deviation,
and the three products see six such errors, of which the first four enter the gated activation: in all about
0.008 sqrt(6), 0.02 of the result's size.  0.05 leaves room for the outliers of the activation's rows.
"""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("moe_layer_q8", os.path.join(ROOT, "examples", "moe_layer_q8.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.mark.parametrize("tokens,hidden,ffn,experts,k", [(1, 256, 512, 8, 2), (16, 320, 576, 8, 2), (48, 1024, 704, 64, 6),
                                                         (777, 1024, 1408, 16, 4), (2500, 256, 512, 40, 3)])
def test_layer(example, tokens, hidden, ffn, experts, k):
    r = example.demo(tokens, hidden, ffn, experts, k, steps=2)
    print(tokens, r, flush=True)
    assert r["sum_exact"] and r["graph_same"]
    assert r["error"] < 0.05
