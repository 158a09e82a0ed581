"""Argument checks of the operators that train a layer: refused before the device is touched (no GPU)."""
import ctypes

import pytest

from paper_2607_19539_amd import binding as B
from tests.test_abi import _c_layout

P = 4096  # an aligned stand-in address; no call below reaches the device


def test_tensor_layout_matches_header(tmp_path):
    cls = B.moe_tensor_t
    fields = [f for f, _ in cls._fields_]
    size, offsets = _c_layout(tmp_path, "moe_tensor_t", fields)
    assert ctypes.sizeof(cls) == size
    assert [getattr(cls, f).offset for f in fields] == offsets


def refused(who, code):
    assert who in B.moe_stage_last_error(None)
    return code


def test_product_refusals():
    lib = B.load()

    def call(x=P, n=4, index=None, off=None, experts=1, w=P, rows=4, K=64, N=32, out=P):
        return lib.moe_product(x, n, index, off, experts, w, rows, K, N, out, None)

    assert call(rows=0, out=None) == B.MOE_OK
    for bad in (dict(experts=2), dict(experts=0), dict(n=3), dict(n=-1, index=P), dict(K=0), dict(N=-8), dict(rows=-1), dict(x=None),
                dict(w=None), dict(out=None)):
        assert call(**bad) == B.MOE_EINVAL, bad
    for bad in (dict(K=12), dict(N=20), dict(K=2 ** 20 + 8), dict(N=2 ** 20 + 8), dict(experts=1025, off=P), dict(index=P, n=2 ** 20, K=2048),
                dict(rows=2 ** 31, n=2 ** 31), dict(x=P + 8), dict(w=P + 8), dict(out=P + 8), dict(index=P + 2), dict(off=P + 2)):
        assert call(**bad) == B.MOE_EUNSUPPORTED, bad
    assert "moe_product" in B.moe_stage_last_error(None)


def test_product_dx_refusals():
    lib = B.load()

    def call(dy=P, off=None, experts=1, w=P, rows=4, K=64, N=32, dx=P):
        return lib.moe_product_dx(dy, off, experts, w, rows, K, N, dx, None)

    assert call(rows=0, dx=None) == B.MOE_OK
    for bad in (dict(experts=2), dict(experts=0), dict(K=0), dict(N=0), dict(rows=-1), dict(dy=None), dict(w=None), dict(dx=None)):
        assert call(**bad) == B.MOE_EINVAL, bad
    for bad in (dict(K=12), dict(N=20), dict(N=2 ** 20 + 8), dict(experts=1025, off=P), dict(rows=2 ** 31), dict(dy=P + 8), dict(w=P + 2),
                dict(dx=P + 4), dict(off=P + 1)):
        assert call(**bad) == B.MOE_EUNSUPPORTED, bad
    assert "moe_product_dx" in B.moe_stage_last_error(None)


def test_product_dw_refusals():
    lib = B.load()

    def call(dy=P, x=P, n=4, index=None, off=None, experts=1, rows=4, K=64, N=32, dw=P, kind=B.MOE_TYPE_F32, acc=0, ws=None, size=0):
        return lib.moe_product_dw(dy, x, n, index, off, experts, rows, K, N, dw, kind, acc, ws, size, None)

    assert call(rows=0, acc=1, dy=None, x=None) == B.MOE_OK
    for bad in (dict(experts=2), dict(n=3), dict(n=-1, index=P), dict(K=0), dict(rows=-1), dict(dy=None), dict(x=None), dict(dw=None),
                dict(kind=2), dict(acc=2), dict(rows=0, dw=None)):
        assert call(**bad) == B.MOE_EINVAL, bad
    for bad in (dict(K=12), dict(N=20), dict(experts=1025, off=P), dict(index=P, n=2 ** 20, K=2048), dict(acc=1, kind=B.MOE_TYPE_BF16),
                dict(dy=P + 8), dict(x=P + 8), dict(dw=P + 8), dict(ws=P + 8), dict(index=P + 2), dict(off=P + 2)):
        assert call(**bad) == B.MOE_EUNSUPPORTED, bad
    need = lib.moe_product_dw_workspace(32768, 1, 64, 32)
    assert need > 0 and lib.moe_product_dw_workspace(0, 1, 64, 32) == 0 and lib.moe_product_dw_workspace(4, 1, 64, 32) == 0
    many = dict(rows=32768, n=32768)
    assert call(**many) == B.MOE_ECAPACITY
    assert call(ws=P, size=need - 1, **many) == B.MOE_ECAPACITY
    assert "moe_product_dw" in B.moe_stage_last_error(None)


def test_gate_refusals():
    lib = B.load()

    def gate(gu=P, off=None, experts=0, rows=4, F=64, act=P):
        return lib.moe_gate(gu, off, experts, rows, F, act, None)

    def back(gu=P, dact=P, off=None, experts=0, rows=4, F=64, dgu=P, act=None):
        return lib.moe_gate_backward(gu, dact, off, experts, rows, F, dgu, act, None)

    for call, names in ((gate, ("gu", "act")), (back, ("gu", "dact", "dgu"))):
        assert call(rows=0, gu=None) == B.MOE_OK
        for bad in (dict(F=0), dict(rows=-1), dict(off=P), *({n: None} for n in names)):
            assert call(**bad) == B.MOE_EINVAL, bad
        for bad in (dict(F=12), dict(F=2 ** 19 + 8), dict(rows=2 ** 31), dict(off=P + 2, experts=1), *({n: P + 8} for n in names)):
            assert call(**bad) == B.MOE_EUNSUPPORTED, bad
    assert back(act=P + 4) == B.MOE_EUNSUPPORTED
    assert gate(rows=2 ** 31 - 1, F=4096) == B.MOE_EUNSUPPORTED       # more than one launch takes


def test_combine_backward_refusals():
    lib = B.load()

    def call(dout=P, recv=P, rows=4, H=64, slot=P, gate=P, T=4, k=2, drecv=P, dgate=P):
        return lib.moe_combine_backward(dout, recv, rows, H, slot, gate, T, k, drecv, dgate, None)

    assert call(T=0, dout=None) == B.MOE_OK
    for bad in (dict(H=0), dict(T=-1), dict(k=0), dict(rows=-1), dict(drecv=None, dgate=None), dict(dout=None), dict(recv=None),
                dict(slot=None), dict(gate=None)):
        assert call(**bad) == B.MOE_EINVAL, bad
    for bad in (dict(H=12), dict(H=65544), dict(k=65), dict(T=2 ** 31), dict(rows=2 ** 31), dict(dout=P + 8), dict(recv=P + 8),
                dict(drecv=P + 8), dict(slot=P + 2), dict(gate=P + 2), dict(dgate=P + 2), dict(T=2 ** 31 - 1, k=64)):
        assert call(**bad) == B.MOE_EUNSUPPORTED, bad
    assert "moe_combine_backward" in B.moe_stage_last_error(None)


def tensors(*entries):
    return (B.moe_tensor_t * max(len(entries), 1))(*[B.moe_tensor_t(*e) for e in entries]), len(entries)


def test_clip_refusals():
    lib = B.load()

    def squares(*entries, total=P, ws=P, size=1 << 20):
        return lib.moe_squares(*tensors(*entries), total, ws, size, None)

    def clip(*entries, total=P, max_norm=1.0, norm=None):
        return lib.moe_clip(*tensors(*entries), total, max_norm, norm, None)

    fine = (P, 2 * P, 64, 0, 0)
    assert lib.moe_squares_workspace(*tensors()) == 0 and lib.moe_squares_workspace(*tensors((P, P, 0, 0, 0))) == 0
    need = lib.moe_squares_workspace(*tensors(fine))
    assert need > 0 and lib.moe_squares_workspace(*tensors(*[fine] * 129)) == 2 * need
    for call in (squares, clip):
        for bad in ((P, P, -1, 0, 0), (None, P, 8, 0, 0), (P, P, 8, 2, 0), (P, P, 8, 0, 1)):
            assert call(fine, bad) == B.MOE_EINVAL, bad
        assert call((P + 2, P, 8, 0, 0)) == B.MOE_EUNSUPPORTED and call((P + 1, P, 8, 1, 0)) == B.MOE_EUNSUPPORTED
        assert call((P, P, 2 ** 60, 0, 0)) == B.MOE_EUNSUPPORTED
        assert call(fine, total=None) == B.MOE_EINVAL and call(fine, total=P + 4) == B.MOE_EUNSUPPORTED
    assert lib.moe_squares(None, 1, P, P, 1 << 20, None) == B.MOE_EINVAL and lib.moe_squares(None, -1, P, P, 1 << 20, None) == B.MOE_EINVAL
    assert squares(fine, ws=None) == B.MOE_ECAPACITY and squares(fine, size=need - 1) == B.MOE_ECAPACITY
    assert squares(fine, ws=P + 4) == B.MOE_EUNSUPPORTED
    assert clip((P, None, 8, 0, 0)) == B.MOE_EINVAL and clip((P, P + 2, 8, 0, 0)) == B.MOE_EUNSUPPORTED
    assert clip(fine, max_norm=-1.0) == B.MOE_EINVAL and clip(fine, max_norm=float("nan")) == B.MOE_EINVAL
    assert clip(fine, norm=P + 2) == B.MOE_EUNSUPPORTED
    # outs that overlap: the same tensor twice, an out in another's data, one that is shifted against its own data
    assert clip(fine, fine) == B.MOE_EINVAL
    assert clip((P, P, 64, 0, 0), (P + 252, P + 252, 64, 0, 0)) == B.MOE_EINVAL
    assert clip((P, 2 * P, 64, 0, 0), (2 * P + 128, 3 * P, 64, 0, 0)) == B.MOE_EINVAL
    assert clip((P, P + 4, 64, 0, 0)) == B.MOE_EINVAL
    assert "overlaps" in B.moe_stage_last_error(None)


def test_binding_checks_tensors():
    torch = pytest.importorskip("torch")
    x, w = torch.zeros((4, 64), dtype=torch.bfloat16), torch.zeros((2, 8, 64), dtype=torch.bfloat16)
    y = torch.zeros((4, 8), dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="device"):
        B.moe_product(x, w[:1], y)
    with pytest.raises(ValueError, match="expert_offsets"):
        B.moe_product(x, w, y)
    with pytest.raises(ValueError, match="at least"):
        B.moe_product(x[:2], w[:1], y)
    with pytest.raises(ValueError, match="three dimensions"):
        B.moe_product_dx(y, w[0], x)
    with pytest.raises(ValueError, match="two dimensions"):
        B.moe_product_dw(y[0], x, w)
    with pytest.raises(ValueError, match="as many gate"):
        B.moe_gate(x[:, :63], x)
    with pytest.raises(ValueError, match="device"):
        B.moe_gate_backward(x, y, x)
    with pytest.raises(ValueError, match="device"):
        B.moe_combine_backward(x, x, torch.zeros((4, 1), dtype=torch.int32), torch.zeros((4, 1)), drecv=x)
    for bad, out in (([x], None), ([1.5], None), ([x], [x, x])):
        with pytest.raises(ValueError, match="current device"):
            B.moe_squares(bad, torch.zeros(1, dtype=torch.float64))
        with pytest.raises(ValueError, match="current device"):
            B.moe_clip(bad, torch.zeros(1, dtype=torch.float64), 1.0, out=out)


@pytest.mark.parametrize("by_k", [False, True])
@pytest.mark.parametrize("rows,grouped,E,K,N", [
    (1048000, True, 1024, 16, 8), (1048560, False, 1, 16, 8), (1048561, False, 1, 16, 8), (2 ** 31 - 1, False, 1, 16, 8),
    (2 ** 31 - 1, True, 1024, 16, 8), (2 ** 30, False, 1, 128, 64), (8, True, 4, 16, 2 ** 20), (10 ** 6, False, 1, 8, 2 ** 20)])
def test_the_product_chosen_can_be_launched(rows, grouped, E, K, N, by_k):
    f = B.load()._ZN3moe12product_kindElbiiib
    f.argtypes, f.restype = [ctypes.c_int64, ctypes.c_bool] + [ctypes.c_int32] * 3 + [ctypes.c_bool], ctypes.c_int
    kind, ends = f(rows, grouped, E, K, N, by_k), E if grouped else 0
    if kind < 2:
        assert -(-rows // 16) + ends <= 65535 and -(-N // (64 if by_k else 16 << kind)) * 256 < 2 ** 32
    elif kind != 4:
        w, x = {2: (64, 64), 3: (128, 128), 5: (128, 64), 6: (128, 128)}[kind]
        assert (-(-rows // x) + ends) * -(-N // w) * 256 < 2 ** 32


@pytest.mark.parametrize("rows,E,K,N", [(1, 1024, 2 ** 13, 2 ** 13), (64, 1, 2 ** 18, 2 ** 18), (2 ** 31 - 1, 1, 2 ** 18, 2 ** 18), (1, 1, 2 ** 18, 2 ** 17)])
def test_the_way_to_dw_can_be_launched(rows, E, K, N):
    class DwPlan(ctypes.Structure):
        _fields_ = [("tile", ctypes.c_int), ("split", ctypes.c_int)]

    f = B.load()._ZN3moe15product_dw_planEliii
    f.argtypes, f.restype = [ctypes.c_int64] + [ctypes.c_int32] * 3, DwPlan
    p = f(rows, E, K, N)
    assert p.tile == 256 or E * p.split * -(-N // p.tile) * -(-K // p.tile) * 256 < 2 ** 32
