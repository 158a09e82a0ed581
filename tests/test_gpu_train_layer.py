"""A layer's training step, every operator in one run: gradients against 64 bits, accumulation, a captured step.

Between the operators values are held in bf16, whose roundings have a relative size of some 0.0017 (2^-8 at most) each.
A gradient passes through at most ten of them (normed rows, g and u, the activation, the experts' outputs, and the
gradients of each), in all about 0.0017 sqrt(10), 0.0054; 0.02 leaves room for sums that cancel.  The router's gradient
is a difference of the gates' gradients, of which nothing but their roundings may be left (all of it is, with one choice a
token): each is a sum of products dout y, whose roundings have 0.0054 of the size sqrt(sum of (dout y)^2), so its error
is measured by that size as well.
"""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("moe_layer_train", os.path.join(ROOT, "examples", "moe_layer_train.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


SIZES = [(1, 256, 512, 8, 2), (16, 320, 576, 8, 2), (48, 264, 88, 16, 4), (500, 256, 512, 8, 2), (1500, 128, 176, 40, 3), (300, 1024, 704, 4, 1)]


@pytest.mark.parametrize("tokens,hidden,ffn,experts,k", SIZES)
def test_gradients(example, tokens, hidden, ffn, experts, k):
    errors = example.check(tokens, hidden, ffn, experts, k, seed=tokens)
    print(tokens, errors, flush=True)
    assert all(v < 0.02 for v in errors.values()), errors


@pytest.mark.parametrize("tokens,hidden,ffn,experts,k", [(16, 320, 576, 8, 2), (2000, 256, 512, 16, 4)])
def test_step_in_a_graph(example, tokens, hidden, ffn, experts, k):
    assert example.timed(tokens, hidden, ffn, experts, k, steps=2)["graph_same"]


def test_accumulated_gradients_and_clipping(example):
    layer, _, (x, residual, dout, dsum) = example.make(200, 256, 512, 8, 2)
    layer.forward(x, residual)
    layer.backward(dout, dsum)
    once = {n: g.clone() for n, g in layer.grads.items()}
    layer.backward(dout, dsum, accumulate=True)
    for n, g in layer.grads.items():
        assert torch.equal(g, once[n] + once[n]), n
    norm = float(layer.clip(0.5))
    want = sum(float((2.0 * g.double()).pow(2).sum()) for g in once.values()) ** 0.5
    assert abs(norm - want) <= 2.0 ** -22 * want
    after = sum(float(g.double().pow(2).sum()) for g in layer.grads.values()) ** 0.5
    assert abs(after - 0.5) <= 2.0 ** -20


def test_padded_tokens_have_no_gradient(example):
    """Tokens whose logits leave no expert have no rows; the others' gradients are what they are without them."""
    from paper_2607_19539_amd import binding as B
    layer, _, (x, residual, dout, dsum) = example.make(64, 256, 512, 8, 2)
    cfg, real = layer.cfg, 50
    layer.forward(x, residual)
    layer.logits[real:] = -float("inf")
    B.moe_route(cfg, layer.logits, layer.ids, layer.gates)
    B.moe_group(layer.ids, 8, layer.offsets, layer.row_token, layer.slot, workspace=layer.workspace)
    assert int(layer.offsets[8]) == 2 * real and bool((layer.slot[real:] == -1).all())
    for t in (layer.gu, layer.act, layer.y, layer.dy, layer.dact, layer.dgu, layer.drows):
        t.fill_(float("nan"))          # what lies behind the last row is never used
    B.moe_product(layer.normed, layer.w13, layer.gu, row_index=layer.row_token, expert_offsets=layer.offsets)
    B.moe_gate(layer.gu, layer.act, expert_offsets=layer.offsets)
    B.moe_product(layer.act, layer.w2, layer.y, expert_offsets=layer.offsets)
    B.moe_combine(layer.y, layer.slot, layer.gates, layer.out)
    layer.backward(dout, dsum)
    assert all(bool(g.isfinite().all()) for g in layer.grads.values())
    assert bool(layer.dnormed[:real].isfinite().all()) and not bool(layer.dgates[real:].any())
    few, _, _ = example.make(real, 256, 512, 8, 2)
    few.norm, few.router, few.w13, few.w2 = layer.norm, layer.router, layer.w13, layer.w2
    few.forward(x[:real].contiguous(), residual[:real].contiguous())
    few.backward(dout[:real].contiguous(), dsum[:real].contiguous())
    for n in ("w13", "w2"):
        assert example.relative(layer.grads[n], few.grads[n]) < 1e-5
