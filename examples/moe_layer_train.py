"""A training step of a whole mixture-of-experts layer in 16 bits, on one GPU.

    forward    residual + x -> norm -> router -> rows by expert -> gated FFN of each expert -> weighted sum per token
    backward   the gradients of all of it: of x, of the norm's and the router's weights and of the experts' matrices
    clipping   the norm of all gradients, and the gradients scaled to at most a given norm

Every step but the router's own matrix (torch products) is a call of this library; nothing waits for the host, so a
step of a fixed number of tokens can be captured in a graph.

    python examples/moe_layer_train.py              # a small and a large batch: gradients checked, step timed
"""
from __future__ import annotations

import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2607_19539_amd import binding as B  # noqa: E402


class MoeLayerTrain:
    """Weights: norm [H] bf16, router [E, H] fp32, w13 [E, 2 F, H] (gate rows, then up rows) and w2 [E, H, F] bf16.
    ``tokens`` sizes the layer's buffers; gradients are fp32, in ``grads`` under the weights' names."""

    def __init__(self, tokens, norm, router, w13, w2, cfg: B.moe_route_config_t, eps=1e-6):
        E, F2, H = w13.shape
        k, rows, dev = cfg.k, tokens * cfg.k, "cuda"
        self.norm, self.router, self.w13, self.w2, self.cfg, self.eps, self.E = norm, router, w13, w2, cfg, eps, E

        def buf(*shape, dtype=torch.bfloat16):
            return torch.zeros(shape, dtype=dtype, device=dev)

        i32, f32 = torch.int32, torch.float32
        self.sum, self.normed, self.rstd = buf(tokens, H), buf(tokens, H), buf(tokens, dtype=f32)
        self.logits = buf(tokens, E, dtype=f32)
        self.ids, self.gates = buf(tokens, k, dtype=i32), buf(tokens, k, dtype=f32)
        self.offsets, self.row_token, self.slot = buf(E + 1, dtype=i32), buf(rows, dtype=i32), buf(tokens, k, dtype=i32)
        self.gu, self.act, self.y, self.out = buf(rows, F2), buf(rows, F2 // 2), buf(rows, H), buf(tokens, H)
        # of the backward pass
        self.dy, self.dgates, self.dact = buf(rows, H), buf(tokens, k, dtype=f32), buf(rows, F2 // 2)
        self.dgu, self.drows, self.dnormed = buf(rows, F2), buf(rows, H), buf(tokens, H)
        self.dlogits, self.ones, self.dx = buf(tokens, E, dtype=f32), torch.ones((tokens, k), device=dev), buf(tokens, H)
        self.grads = {"norm": buf(H, dtype=f32), "router": buf(E, H, dtype=f32), "w13": buf(*w13.shape, dtype=f32),
                      "w2": buf(*w2.shape, dtype=f32)}
        self.total, self.grad_norm = buf(1, dtype=torch.float64), buf(1, dtype=f32)
        lib, grads = B.load(), list(self.grads.values())
        need = max(16, lib.moe_group_workspace(rows, E), lib.moe_norm_backward_workspace(tokens, H),
                   lib.moe_product_dw_workspace(rows, E, H, F2), lib.moe_product_dw_workspace(rows, E, F2 // 2, H),
                   lib.moe_squares_workspace(*B._tensor_list(grads)))
        self.workspace = torch.empty(need, dtype=torch.uint8, device=dev)   # one for all: the calls follow one another

    def forward(self, x, residual):
        """(out, residual + x) of tokens [T, H] bf16; both are the layer's own buffers."""
        B.moe_norm(x, self.norm, self.eps, residual=residual, sum_out=self.sum, out=self.normed, rstd=self.rstd)
        torch.mm(self.normed.float(), self.router.t(), out=self.logits)
        B.moe_route(self.cfg, self.logits, self.ids, self.gates)
        B.moe_group(self.ids, self.E, self.offsets, self.row_token, self.slot, workspace=self.workspace)
        B.moe_product(self.normed, self.w13, self.gu, row_index=self.row_token, expert_offsets=self.offsets)
        B.moe_gate(self.gu, self.act, expert_offsets=self.offsets)
        B.moe_product(self.act, self.w2, self.y, expert_offsets=self.offsets)
        B.moe_combine(self.y, self.slot, self.gates, self.out)
        return self.out, self.sum

    def backward(self, dout, dsum, accumulate=False):
        """Gradient of x and residual alike, from those of out and of the sum; the weights' go to ``grads``."""
        g, ws = self.grads, self.workspace
        B.moe_combine_backward(dout, self.y, self.slot, self.gates, drecv=self.dy, dgate=self.dgates)
        B.moe_product_dw(self.dy, self.act, g["w2"], expert_offsets=self.offsets, accumulate=accumulate, workspace=ws)
        B.moe_product_dx(self.dy, self.w2, self.dact, expert_offsets=self.offsets)
        B.moe_gate_backward(self.gu, self.dact, self.dgu, expert_offsets=self.offsets)
        B.moe_product_dw(self.dgu, self.normed, g["w13"], row_index=self.row_token, expert_offsets=self.offsets,
                         accumulate=accumulate, workspace=ws)
        B.moe_product_dx(self.dgu, self.w13, self.drows, expert_offsets=self.offsets)
        B.moe_combine(self.drows, self.slot, self.ones, self.dnormed)           # a token's rows added up
        B.moe_route_backward(self.cfg, self.logits, self.ids, self.dgates, self.dlogits)
        drouter = torch.mm(self.dlogits.t(), self.normed.float())
        self.dnormed.copy_(self.dnormed.float() + torch.mm(self.dlogits, self.router))
        g["router"].copy_(g["router"] + drouter if accumulate else drouter)
        kept = g["norm"].clone() if accumulate else None
        B.moe_norm_backward(self.dnormed, self.sum, self.norm, self.rstd, self.dx, g["norm"], dsum=dsum, workspace=ws)
        if accumulate:
            g["norm"] += kept
        return self.dx

    def clip(self, max_norm):
        """Scales the gradients to a norm of at most ``max_norm``; their norm before it."""
        grads = list(self.grads.values())
        B.moe_squares(grads, self.total, workspace=self.workspace)
        B.moe_clip(grads, self.total, max_norm, norm=self.grad_norm)
        return self.grad_norm


def plain_layer(x, residual, norm, router, w13, w2, ids, eps=1e-6, scale=1.0):
    """The layer with torch operations that have gradients, in the type of its arguments, its experts chosen by ids
    (softmax scores over the chosen ones)."""
    h = x + residual
    n = h * torch.rsqrt((h * h).mean(1, keepdim=True) + eps) * norm
    p = torch.softmax(n @ router.t(), 1)
    have = ids >= 0
    chosen = p.gather(1, ids.clamp(min=0).long()) * have
    gates = scale * chosen / chosen.sum(1, keepdim=True)
    out = torch.zeros_like(n)
    F = w2.shape[2]
    for e in range(w13.shape[0]):
        t, j = torch.nonzero(ids == e, as_tuple=True)
        gu = n[t] @ w13[e].t()
        y = (torch.nn.functional.silu(gu[:, :F]) * gu[:, F:]) @ w2[e].t()
        out = out.index_add(0, t, gates[t, j][:, None] * y)
    return out, h


def make(tokens, hidden, ffn, experts, k, seed=0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)

    def normal(*shape, std=1.0, dtype=torch.bfloat16):
        return torch.empty(shape, dtype=dtype, device="cuda").normal_(0.0, std, generator=g)

    weights = (1.0 + normal(hidden, std=0.1), normal(experts, hidden, std=hidden ** -0.5, dtype=torch.float32),
               normal(experts, 2 * ffn, hidden, std=hidden ** -0.5), normal(experts, hidden, ffn, std=ffn ** -0.5))
    layer = MoeLayerTrain(tokens, *weights, B.make_route_config(experts, k))
    return layer, weights, [normal(tokens, hidden) for _ in range(4)]     # x, residual, dout, dsum


def relative(got, want):
    return float((got.double() - want.double()).norm() / want.double().norm())


def router_terms(layer, dout):
    """The size of what the router's gradient is the difference of.

    A choice's dgate, the sum over h of dout y, is as far off as y's roundings make it: a share of s = sqrt(sum of
    (dout y)^2), however small the sum itself.  The logit's gradient is weight (dgate - sum of weight dgate), and the
    gates' gradients of a token may well be alike."""
    have = layer.slot >= 0
    y = layer.y.double()[layer.slot.clamp(min=0).long()] * have[:, :, None]
    s2 = (dout.double()[:, None, :] * y).pow(2).sum(2)
    w2 = layer.gates.double().pow(2)
    dl2 = (w2 * (s2 + (w2 * s2).sum(1, keepdim=True))).sum(1)
    return float((dl2 * layer.normed.double().pow(2).sum(1)).sum().sqrt())


def check(tokens, hidden, ffn, experts, k, seed=0):
    """Relative errors of the output and of every gradient against the plain layer in 64 bits (the router's relative to
    the size of its terms as well)."""
    layer, weights, (x, residual, dout, dsum) = make(tokens, hidden, ffn, experts, k, seed)
    out, _ = layer.forward(x, residual)
    dx = layer.backward(dout, dsum)
    leaves = [t.double().requires_grad_() for t in (x, residual, *weights)]
    want, total = plain_layer(*leaves, layer.ids)
    torch.autograd.backward([want, total], [dout.double(), dsum.double()])
    errors = {"out": relative(out, want.detach()), "dx": relative(dx, leaves[0].grad)}
    for i, name in enumerate(("norm", "router", "w13", "w2")):
        errors[name] = relative(layer.grads[name], leaves[2 + i].grad)
    off = float((layer.grads["router"].double() - leaves[3].grad).norm())
    errors["router"] = off / (float(leaves[3].grad.norm()) + router_terms(layer, dout))
    return errors


def timed(tokens, hidden, ffn, experts, k, steps=10):
    """Microseconds of a step (forward, backward, clipping), eager and from a graph; whether the replays agree."""
    layer, _, (x, residual, dout, dsum) = make(tokens, hidden, ffn, experts, k)

    def step():
        layer.forward(x, residual)
        layer.backward(dout, dsum)
        layer.clip(1.0)

    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        step()
    torch.cuda.current_stream().wait_stream(stream)
    torch.cuda.synchronize()
    held = [layer.out, layer.dx, layer.grad_norm, *layer.grads.values()]
    first = [t.clone() for t in held]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    same = True
    for _ in range(3):
        for t in held:
            t.fill_(3.0)
        graph.replay()
        torch.cuda.synchronize()
        same &= all(torch.equal(a, b) for a, b in zip(held, first))
    times = []
    for call in (step, graph.replay):
        torch.cuda.synchronize()
        t = time.perf_counter()
        for _ in range(steps):
            call()
        torch.cuda.synchronize()
        times.append((time.perf_counter() - t) / steps * 1e6)
    return {"graph_same": same, "us": times[0], "graph_us": times[1]}


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--hidden", type=int, default=2048)
    ap.add_argument("--ffn", type=int, default=1408)
    ap.add_argument("--experts", type=int, default=64)
    ap.add_argument("--k", type=int, default=6)
    ap.add_argument("--tokens", type=int, nargs="*", default=[64, 8192])
    a = ap.parse_args()
    e = check(500, 256, 512, 8, 2)
    print("relative errors against 64 bits: " + ", ".join(f"{n} {v:.4f}" for n, v in e.items()), flush=True)
    for t in a.tokens:
        r = timed(t, a.hidden, a.ffn, a.experts, a.k)
        print(f"{t} tokens: {r['us']:.0f} us a step, {r['graph_us']:.0f} us from a graph "
              f"(replays {'equal' if r['graph_same'] else 'DIFFER'})", flush=True)


if __name__ == "__main__":
    main()
