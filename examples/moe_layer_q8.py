"""A whole mixture-of-experts layer with its experts in 8 bits, on one GPU.

    residual + x -> norm -> router -> rows by expert -> gated FFN of each expert -> weighted sum per token

Every step but the router's own matrix (a torch product) is a call of this library; nothing waits for the host,
so a step of a fixed number of tokens can be captured in a graph.

    python examples/moe_layer_q8.py                  # a decode step and a prefill batch, checked and timed
"""
from __future__ import annotations

import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2607_19539_amd import binding as B  # noqa: E402


class MoeLayerQ8:
    """Weights: norm [H] bf16, router [E, H] fp32, bias [E] fp32 or None, w1 and w3 [E, F, H], w2 [E, H, F] bf16
    (kept in 8 bits with a scale per output channel).  ``tokens`` sizes the layer's buffers."""

    def __init__(self, tokens, norm, router, bias, w1, w3, w2, cfg: B.moe_route_config_t, eps=1e-6):
        E, F, H = w1.shape
        k, rows, dev = cfg.k, tokens * cfg.k, "cuda"
        self.norm, self.router, self.bias, self.cfg, self.eps, self.E = norm, router, bias, cfg, eps, E
        self.w = [self._weights(w) for w in (w1, w3, w2)]
        bf16 = torch.bfloat16
        self.sum = torch.empty((tokens, H), dtype=bf16, device=dev)
        self.normed = torch.empty((tokens, H), dtype=bf16, device=dev)
        self.q, self.scale = torch.empty((tokens, H), dtype=torch.int8, device=dev), torch.empty(tokens, device=dev)
        self.ids = torch.empty((tokens, k), dtype=torch.int32, device=dev)
        self.gates = torch.empty((tokens, k), device=dev)
        self.offsets = torch.empty(E + 1, dtype=torch.int32, device=dev)
        self.row_token = torch.empty(rows, dtype=torch.int32, device=dev)
        self.slot = torch.empty((tokens, k), dtype=torch.int32, device=dev)
        self.workspace = torch.empty(max(4, B.load().moe_group_workspace(rows, E)), dtype=torch.uint8, device=dev)
        self.act = torch.empty((rows, F), dtype=bf16, device=dev)
        self.act_q, self.act_scale = torch.empty((rows, F), dtype=torch.int8, device=dev), torch.empty(rows, device=dev)
        self.y = torch.zeros((rows, H), dtype=bf16, device=dev)
        self.out = torch.empty((tokens, H), dtype=bf16, device=dev)

    @staticmethod
    def _weights(w):
        E, N, K = w.shape
        q, s = torch.empty((E, N, K), dtype=torch.int8, device="cuda"), torch.empty((E, N), device="cuda")
        B.moe_q8_rows(w.reshape(E * N, K), q.view(E * N, K), s.view(E * N))
        return q, s

    def __call__(self, x, residual):
        """(out, residual + x) of tokens [T, H] bf16; both are the layer's own buffers."""
        (w1, s1), (w3, s3), (w2, s2) = self.w
        B.moe_norm(x, self.norm, self.eps, residual=residual, sum_out=self.sum, out=self.normed, out_q=self.q,
                   scale=self.scale)
        logits = self.normed.float() @ self.router.t()
        B.moe_route(self.cfg, logits, self.ids, self.gates, bias=self.bias)
        B.moe_group(self.ids, self.E, self.offsets, self.row_token, self.slot, workspace=self.workspace)
        B.moe_q8_gated(self.q, self.scale, w1, s1, w3, s3, self.act, row_index=self.row_token,
                       expert_offsets=self.offsets)
        B.moe_q8_rows(self.act, self.act_q, self.act_scale)
        B.moe_q8_product(self.act_q, self.act_scale, w2, s2, self.y, expert_offsets=self.offsets)
        B.moe_combine(self.y, self.slot, self.gates, self.out)
        return self.out, self.sum


def plain_layer(x, residual, norm, router, w1, w3, w2, ids, gates, eps=1e-6):
    """The layer in fp32 with 16-bit weights, its experts chosen by ``ids`` and ``gates``."""
    h = (x.float() + residual.float()).to(torch.bfloat16).float()
    n = h * torch.rsqrt((h * h).mean(1, keepdim=True) + eps) * norm.float()
    out = torch.zeros_like(n)
    for e in range(w1.shape[0]):
        t, j = torch.nonzero(ids == e, as_tuple=True)
        g, u = n[t] @ w1[e].float().t(), n[t] @ w3[e].float().t()
        out.index_add_(0, t, gates[t, j][:, None] * ((g * torch.sigmoid(g) * u) @ w2[e].float().t()))
    return out, h


def demo(tokens, hidden, ffn, experts, k, seed=0, steps=20):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)

    def normal(*shape, std=1.0, dtype=torch.bfloat16):
        return torch.empty(shape, dtype=dtype, device="cuda").normal_(0.0, std, generator=g)

    x, residual = normal(tokens, hidden), normal(tokens, hidden)
    weights = (1.0 + normal(hidden, std=0.1), normal(experts, hidden, std=hidden ** -0.5, dtype=torch.float32))
    mats = (normal(experts, ffn, hidden, std=0.02), normal(experts, ffn, hidden, std=0.02), normal(experts, hidden, ffn, std=0.02))
    layer = MoeLayerQ8(tokens, *weights, None, *mats, B.make_route_config(experts, k))
    out, total = layer(x, residual)
    want, h = plain_layer(x, residual, *weights, *mats, layer.ids, layer.gates)
    error = float((out.float() - want).norm() / want.norm())
    exact_sum = bool(torch.equal(total.float(), h))
    del want, h
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        layer(x, residual)
    torch.cuda.current_stream().wait_stream(stream)
    first = out.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer(x, residual)
    same = True
    for _ in range(3):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        same &= bool(torch.equal(out, first))
    times = []
    for call in (lambda: layer(x, residual), graph.replay):
        torch.cuda.synchronize()
        t = time.perf_counter()
        for _ in range(steps):
            call()
        torch.cuda.synchronize()
        times.append((time.perf_counter() - t) / steps * 1e6)
    return {"error": error, "sum_exact": exact_sum, "graph_same": same, "us": times[0], "graph_us": times[1]}


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--hidden", type=int, default=2048)
    ap.add_argument("--ffn", type=int, default=1408)
    ap.add_argument("--experts", type=int, default=64)
    ap.add_argument("--k", type=int, default=6)
    ap.add_argument("--tokens", type=int, nargs="*", default=[16, 4096])
    a = ap.parse_args()
    for t in a.tokens:
        r = demo(t, a.hidden, a.ffn, a.experts, a.k)
        print(f"{t} tokens: relative error {r['error']:.4f} against 16-bit weights in fp32, {r['us']:.1f} us a layer, "
              f"{r['graph_us']:.1f} us from a graph (replays {'equal' if r['graph_same'] else 'DIFFER'})", flush=True)


if __name__ == "__main__":
    main()
