"""The operators that train a layer in captured graphs, beside errors that earlier calls left, and two at once."""
import pytest

from paper_2607_19539_amd import binding as B
from tests.test_gpu_ops_errors import run_after_an_error

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


def normal(g, *shape, std=1.0, dtype=torch.bfloat16):
    return torch.empty(shape, dtype=dtype, device="cuda").normal_(0.0, std, generator=g)


def everything(rows, K, N, E, seed=0):
    """Each operator once on buffers of its own; the calls by name, and their outputs."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    counts = torch.bincount(torch.randint(0, E, (rows,), generator=g, device="cuda"), minlength=E)
    off = torch.zeros(E + 1, dtype=torch.int32, device="cuda")
    off[1:] = counts.cumsum(0)
    x, w, dy, gu = normal(g, rows, K), normal(g, E, N, K, std=0.1), normal(g, rows, N), normal(g, rows, 2 * K)
    index = torch.randperm(rows, generator=g, device="cuda").int()
    y, dx, dw, dwb = torch.zeros_like(dy), torch.zeros_like(x), torch.zeros((E, N, K), device="cuda"), torch.zeros_like(w)
    act, dgu, again = torch.zeros_like(x), torch.zeros_like(gu), torch.zeros_like(x)
    T = rows // 2
    slot, gate, dout = torch.randperm(2 * T, generator=g, device="cuda").int().view(T, 2), torch.rand((T, 2), generator=g, device="cuda"), normal(g, T, K)
    drecv, dgate = torch.zeros((2 * T, K), dtype=torch.bfloat16, device="cuda"), torch.zeros((T, 2), device="cuda")
    total, norm, clipped = torch.zeros(1, dtype=torch.float64, device="cuda"), torch.zeros(1, device="cuda"), [torch.zeros_like(x), torch.zeros_like(w)]
    lib = B.load()
    ws = torch.empty(max(16, lib.moe_product_dw_workspace(rows, E, K, N)), dtype=torch.uint8, device="cuda")
    sq = torch.empty(1 << 15, dtype=torch.uint8, device="cuda")
    calls = dict(
        product=lambda: B.moe_product(x, w, y, row_index=index, expert_offsets=off), product_dx=lambda: B.moe_product_dx(dy, w, dx, expert_offsets=off),
        product_dw=lambda: B.moe_product_dw(dy, x, dw, row_index=index, expert_offsets=off, workspace=ws),
        product_dw16=lambda: B.moe_product_dw(dy, x, dwb, expert_offsets=off, workspace=ws),
        gate=lambda: B.moe_gate(gu, act), gate_backward=lambda: B.moe_gate_backward(gu, x, dgu, act=again),
        combine_backward=lambda: B.moe_combine_backward(dout, x[:2 * T], slot, gate, drecv=drecv, dgate=dgate),
        squares=lambda: B.moe_squares([x, w], total, workspace=sq), clip=lambda: B.moe_clip([x, w], total, 1.0, out=clipped, norm=norm))
    return calls, [y, dx, dw, dwb, act, dgu, again, drecv, dgate, total, norm, *clipped]


SIZES = [(2, 64, 72, 1), (40, 320, 576, 8), (3000, 256, 512, 16), (6000, 512, 256, 1)]


@pytest.mark.parametrize("rows,K,N,E", SIZES)
def test_replays_equal_the_eager_calls(rows, K, N, E):
    calls, outs = everything(rows, K, N, E)

    def call():
        for c in calls.values():
            c()

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


def test_an_error_left_behind_is_not_the_operators():
    for rows, K, N, E in SIZES:
        calls, _ = everything(rows, K, N, E)
        reported, kept = run_after_an_error(calls)
        assert not reported and all(kept)


def test_calls_on_two_streams_at_once():
    """Two sets of buffers and workspaces, on a stream each, one after another without a wait between them."""
    sets = [everything(3000, 256, 512, 16, seed) for seed in (1, 2)]
    for calls, _ in sets:
        for c in calls.values():
            c()
    torch.cuda.synchronize()
    want = [[o.clone() for o in outs] for _, outs in sets]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _, outs in sets:
        for o in outs:
            o.fill_(7)
    torch.cuda.synchronize()
    for _ in range(5):
        for (calls, _), s in zip(sets, streams):
            with torch.cuda.stream(s):
                for c in calls.values():
                    c()
    torch.cuda.synchronize()
    for (_, outs), w in zip(sets, want):
        assert all(torch.equal(a, b) for a, b in zip(outs, w))
