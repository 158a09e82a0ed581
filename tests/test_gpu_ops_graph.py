"""The operators around the stage in a captured graph: replays with eager work between them give the eager bits."""
import pytest

from paper_2607_19539_amd import binding as B

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


def pipeline(T, H, E, k, F):
    """Everything once, forward and backward, on buffers of its own; returns the call and its outputs."""
    g = torch.Generator(device="cuda")
    g.manual_seed(T)
    d = dict(device="cuda")
    bf = torch.bfloat16

    def normal(*s, std=1.0, dtype=bf):
        return torch.empty(s, dtype=dtype, **d).normal_(0.0, std, generator=g)

    x, res, w = normal(T, H), normal(T, H), normal(H, std=0.1) + 1.0
    logits, dy, dw = normal(T, E, dtype=torch.float32), normal(T, H, std=0.1), normal(T, k, dtype=torch.float32)
    rows = T * k
    s, out, q, sc, r = torch.empty_like(x), torch.empty_like(x), torch.empty((T, H), dtype=torch.int8, **d), torch.empty(T, **d), torch.empty(T, **d)
    dx, dweight = torch.empty_like(x), torch.empty(H, **d)
    ids, gates, dl = torch.empty((T, k), dtype=torch.int32, **d), torch.empty((T, k), **d), torch.empty((T, E), **d)
    off, row, slot = torch.empty(E + 1, dtype=torch.int32, **d), torch.empty(rows, dtype=torch.int32, **d), torch.empty((T, k), dtype=torch.int32, **d)
    mats = [torch.randint(-127, 128, s_, dtype=torch.int8, generator=g, **d) for s_ in ((E, F, H), (E, F, H), (E, H, F))]
    scales = [torch.rand(m.shape[:2], generator=g, **d) * 1e-3 for m in mats]
    act, aq, asc, y = torch.empty((rows, F), dtype=bf, **d), torch.empty((rows, F), dtype=torch.int8, **d), torch.empty(rows, **d), torch.empty((rows, H), dtype=bf, **d)
    back = torch.empty((rows, F), dtype=bf, **d)
    cfg = B.make_route_config(E, k, score=B.MOE_SCORE_SIGMOID, groups=4, top_groups=3, group_best=2, scale=2.5)
    ws = torch.empty(max(16, B.load().moe_group_workspace(rows, E)), dtype=torch.uint8, **d)
    nws = torch.empty(max(16, B.load().moe_norm_backward_workspace(T, H)), dtype=torch.uint8, **d)

    def call():
        B.moe_norm(x, w, 1e-6, residual=res, sum_out=s, out=out, out_q=q, scale=sc, rstd=r)
        B.moe_route(cfg, logits, ids, gates)
        B.moe_group(ids, E, off, row, slot, workspace=ws)
        B.moe_q8_gated(q, sc, mats[0], scales[0], mats[1], scales[1], act, row_index=row, expert_offsets=off)
        B.moe_q8_rows(act, aq, asc)
        B.moe_q8_restore(aq, asc, back)
        B.moe_q8_product(aq, asc, mats[2], scales[2], y, expert_offsets=off)
        B.moe_combine(y, slot, gates, out)
        B.moe_norm_backward(dy, s, w, r, dx, dweight, workspace=nws)
        B.moe_route_backward(cfg, logits, ids, dw, dl)

    return call, [s, out, q, sc, r, dx, dweight, ids, gates, dl, off, row, slot, act, aq, asc, back, y]


@pytest.mark.parametrize("T,H,E,k,F", [(1, 256, 8, 2, 512), (40, 320, 16, 4, 576), (3000, 512, 64, 6, 256)])
def test_replays_equal_the_eager_call(T, H, E, k, F):
    call, outs = pipeline(T, H, E, k, F)
    call()
    torch.cuda.synchronize()
    want = [o.clone() for o in outs]
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        call()
    torch.cuda.current_stream().wait_stream(stream)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for i in range(4):
        for o in outs:
            o.fill_(7)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(outs, want):
            assert torch.equal(a, b), i
        torch.empty(1 << 20, device="cuda").normal_().sum().item()   # eager work between the replays
