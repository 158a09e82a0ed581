"""An error that some earlier call of the program left behind is not the operators': they run, report MOE_OK, and
leave it to whoever asks for it."""
import ctypes

import pytest

from paper_2607_19539_amd import binding as B

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


def calls():
    d, bf = dict(device="cuda"), torch.bfloat16
    T, H, E, k = 5000, 64, 8, 2
    x, w = torch.ones((T, H), dtype=bf, **d), torch.ones(H, dtype=bf, **d)
    rstd, dx, dw = torch.ones(T, **d), torch.empty_like(x), torch.empty(H, **d)
    q, s = torch.ones((T, H), dtype=torch.int8, **d), torch.ones(T, **d)
    cfg, logits = B.make_route_config(E, k), torch.zeros((T, E), **d)
    ids, gates, dl = torch.zeros((T, k), dtype=torch.int32, **d), torch.ones((T, k), **d), torch.empty((T, E), **d)
    off, row = torch.zeros(E + 1, dtype=torch.int32, **d), torch.zeros(T * k, dtype=torch.int32, **d)
    slot, few = torch.zeros((T, k), dtype=torch.int32, **d), torch.zeros((4, k), dtype=torch.int32, **d)
    few_row, few_slot = torch.zeros(4 * k, dtype=torch.int32, **d), torch.zeros((4, k), dtype=torch.int32, **d)
    w8, ws = torch.ones((1, 64, H), dtype=torch.int8, **d), torch.ones((1, 64), **d)
    y = torch.empty((T, 64), dtype=bf, **d)
    gws = torch.empty(B.load().moe_group_workspace(T * k, E), dtype=torch.uint8, **d)
    nws = torch.empty(B.load().moe_norm_backward_workspace(T, H), dtype=torch.uint8, **d)
    out = dict(
        norm=lambda: B.moe_norm(x, w, 1e-6, out=dx), norm_backward=lambda: B.moe_norm_backward(x, x, w, rstd, dx, dw, workspace=nws),
        q8_rows=lambda: B.moe_q8_rows(x, q, s), q8_restore=lambda: B.moe_q8_restore(q, s, dx),
        route=lambda: B.moe_route(cfg, logits, ids, gates), route_backward=lambda: B.moe_route_backward(cfg, logits, ids, gates, dl),
        group=lambda: B.moe_group(ids, E, off, row, slot, workspace=gws), group_few=lambda: B.moe_group(few, E, off, few_row, few_slot))
    for rows in (4, 200, 5000):
        out[f"q8_product_{rows}"] = lambda rows=rows: B.moe_q8_product(q[:rows], s[:rows], w8, ws, y[:rows])
        out[f"q8_gated_{rows}"] = lambda rows=rows: B.moe_q8_gated(q[:rows], s[:rows], w8, ws, w8, ws, y[:rows])
    return out


def run_after_an_error(todo):
    """The calls that report an error which an earlier call left behind, and whether each leaves it."""
    lib = B.load()
    hip = {n: getattr(lib, n) for n in ("hipSetDevice", "hipPeekAtLastError", "hipGetLastError")}  # of the runtime it is linked to
    for f in hip.values():
        f.restype = ctypes.c_int
    hip["hipSetDevice"].argtypes = [ctypes.c_int]
    for call in todo.values():
        call()
    torch.cuda.synchronize()
    reported, kept = [], []
    for name, call in todo.items():
        hip["hipGetLastError"]()
        left = hip["hipSetDevice"](9999)     # no such device: refused on the host, the device stays as it is
        assert left != 0 and hip["hipPeekAtLastError"]() == left
        try:
            call()
        except RuntimeError as e:
            reported.append((name, str(e)))
        kept.append(hip["hipPeekAtLastError"]() == left)
        hip["hipGetLastError"]()
    torch.cuda.synchronize()
    return reported, kept


def test_an_error_left_behind_is_not_the_operators():
    reported, kept = run_after_an_error(calls())
    assert not reported and all(kept)


def test_an_error_left_behind_is_not_the_combines():
    recv, gate = torch.ones((12, 64), dtype=torch.bfloat16, device="cuda"), torch.ones((4, 2), device="cuda")
    slot, out = torch.zeros((4, 2), dtype=torch.int32, device="cuda"), torch.empty((4, 64), dtype=torch.bfloat16, device="cuda")
    reported, kept = run_after_an_error(dict(combine=lambda: B.moe_combine(recv, slot, gate, out)))
    assert not reported and all(kept) and bool((out == 2).all())
