"""Argument checks of the operators around the stage: refused before the device is touched (no GPU)."""
import ctypes

import pytest

from paper_2607_19539_amd import binding as B
from tests.test_abi import _c_layout

P = 4096  # an aligned stand-in address; no call below reaches the device


def test_route_config_layout_matches_header(tmp_path):
    cls = B.moe_route_config_t
    fields = [f for f, _ in cls._fields_]
    size, offsets = _c_layout(tmp_path, "moe_route_config_t", fields)
    assert ctypes.sizeof(cls) == size
    assert [getattr(cls, f).offset for f in fields] == offsets


def norm(x=P, res=None, w=P, rows=4, hidden=64, eps=1e-6, sum_out=None, out=P, q=None, scale=None, rstd=None):
    return B.load().moe_norm(x, res, w, rows, hidden, eps, sum_out, out, q, scale, rstd, None)


def test_norm_refusals():
    assert norm(rows=0, x=None) == B.MOE_OK
    assert norm(hidden=0) == B.MOE_EINVAL
    assert norm(rows=-1) == B.MOE_EINVAL
    assert norm(hidden=12) == B.MOE_EUNSUPPORTED
    assert norm(hidden=65544) == B.MOE_EUNSUPPORTED
    assert norm(rows=2 ** 31) == B.MOE_EUNSUPPORTED
    assert norm(eps=-1.0) == B.MOE_EINVAL
    assert norm(eps=float("nan")) == B.MOE_EINVAL
    assert norm(out=None) == B.MOE_EINVAL             # no output
    assert norm(q=P) == B.MOE_EINVAL                  # no scale beside the 8-bit rows
    assert norm(scale=P) == B.MOE_EINVAL
    assert norm(x=None) == B.MOE_EINVAL
    assert norm(w=None) == B.MOE_EINVAL
    for k in ("x", "res", "w", "sum_out", "out"):
        assert norm(**{k: P + 8}) == B.MOE_EUNSUPPORTED, k
    assert norm(rstd=P + 2) == B.MOE_EUNSUPPORTED
    assert "moe_norm" in B.moe_stage_last_error(None)


def test_norm_backward_refusals():
    lib = B.load()

    def call(dy=P, h=P, w=P, rstd=P, dsum=None, rows=400, hidden=64, dx=P, dw=P, ws=P, n=1 << 30):
        return lib.moe_norm_backward(dy, h, w, rstd, dsum, rows, hidden, dx, dw, ws, n, None)

    need = lib.moe_norm_backward_workspace(400, 64)
    assert need > 0 and lib.moe_norm_backward_workspace(0, 64) == 0 and lib.moe_norm_backward_workspace(1, 64) == 0
    assert call(n=need - 1) == B.MOE_ECAPACITY
    assert call(ws=None) == B.MOE_ECAPACITY
    assert call(hidden=60) == B.MOE_EUNSUPPORTED
    assert call(dw=None) == B.MOE_EINVAL
    assert call(dx=None) == B.MOE_EINVAL
    assert call(h=None) == B.MOE_EINVAL
    assert call(dsum=P + 2) == B.MOE_EUNSUPPORTED
    assert call(ws=P + 4) == B.MOE_EUNSUPPORTED


def test_q8_row_refusals():
    lib = B.load()
    assert lib.moe_q8_rows(None, 0, 64, None, None, None) == B.MOE_OK
    assert lib.moe_q8_rows(P, 4, 4, P, P, None) == B.MOE_EUNSUPPORTED
    assert lib.moe_q8_rows(P, 4, 64, None, P, None) == B.MOE_EINVAL
    assert lib.moe_q8_rows(P, 4, 64, P + 8, P, None) == B.MOE_EUNSUPPORTED
    assert lib.moe_q8_restore(P, P, 4, 64, None, None) == B.MOE_EINVAL
    assert lib.moe_q8_restore(P, P, -4, 64, P, None) == B.MOE_EINVAL
    assert lib.moe_q8_restore(P, P + 1, 4, 64, P, None) == B.MOE_EUNSUPPORTED


ROUTE = dict(experts=64, k=4, groups=8, top_groups=2, group_best=2)


@pytest.mark.parametrize("change,code", [
    (dict(), B.MOE_OK), (dict(experts=0), B.MOE_EINVAL), (dict(k=0), B.MOE_EINVAL), (dict(k=65), B.MOE_EINVAL),
    (dict(groups=7), B.MOE_EINVAL), (dict(top_groups=9), B.MOE_EINVAL), (dict(top_groups=0), B.MOE_EINVAL),
    (dict(group_best=3), B.MOE_EINVAL), (dict(groups=64, top_groups=1), B.MOE_EINVAL), (dict(score=2), B.MOE_EINVAL),
    (dict(experts=2048), B.MOE_EUNSUPPORTED), (dict(experts=128, k=65), B.MOE_EUNSUPPORTED),
    (dict(experts=256, groups=128, top_groups=1), B.MOE_EUNSUPPORTED)])
def test_route_configurations(change, code):
    cfg = B.make_route_config(**{**ROUTE, **change})
    assert B.load().moe_route(ctypes.byref(cfg), P, 0, None, 0, P, P, None, None) == code  # no tokens
    assert B.load().moe_route_backward(ctypes.byref(cfg), P, 0, P, P, None, 0, P, None) == code


def test_route_refusals():
    lib, cfg = B.load(), B.make_route_config(**ROUTE)
    c = ctypes.byref(cfg)
    assert lib.moe_route(None, P, 0, None, 4, P, P, None, None) == B.MOE_EINVAL
    assert lib.moe_route(c, P, 2, None, 4, P, P, None, None) == B.MOE_EINVAL          # type
    assert lib.moe_route(c, None, 0, None, 4, P, P, None, None) == B.MOE_EINVAL
    assert lib.moe_route(c, P, 0, None, -1, P, P, None, None) == B.MOE_EINVAL
    assert lib.moe_route(c, P, 0, None, 4, None, P, None, None) == B.MOE_EINVAL
    assert lib.moe_route(c, P + 2, 0, None, 4, P, P, None, None) == B.MOE_EUNSUPPORTED
    assert lib.moe_route(c, P + 1, 1, None, 4, P, P, None, None) == B.MOE_EUNSUPPORTED
    assert lib.moe_route_backward(c, P, 0, P, None, None, 4, P, None) == B.MOE_EINVAL
    assert lib.moe_route_backward(c, P, 0, P, P, None, 4, P + 2, None) == B.MOE_EUNSUPPORTED
    assert "moe_route_backward" in B.moe_stage_last_error(None)
    cfg.renormalise = 2
    assert lib.moe_route(c, P, 0, None, 4, P, P, None, None) == B.MOE_EINVAL


def test_group_refusals():
    lib = B.load()

    def call(ids=P, tokens=4, k=2, experts=8, off=P, row=P, slot=P, ws=None, n=0):
        return lib.moe_group(ids, tokens, k, experts, off, row, slot, ws, n, None)

    assert call(k=0) == B.MOE_EINVAL
    assert call(tokens=-1) == B.MOE_EINVAL
    assert call(experts=0) == B.MOE_EINVAL
    assert call(experts=1025) == B.MOE_EUNSUPPORTED
    assert call(tokens=2 ** 30, k=2) == B.MOE_EUNSUPPORTED
    assert call(off=None) == B.MOE_EINVAL
    assert call(ids=None) == B.MOE_EINVAL
    assert call(slot=P + 2) == B.MOE_EUNSUPPORTED
    need = lib.moe_group_workspace(10 ** 6, 256)
    assert need > 0 and lib.moe_group_workspace(8, 8) == 0 and lib.moe_group_workspace(0, 8) == 0
    assert call(tokens=10 ** 6, k=1, experts=256) == B.MOE_ECAPACITY
    assert call(tokens=10 ** 6, k=1, experts=256, ws=P, n=need - 1) == B.MOE_ECAPACITY


@pytest.mark.parametrize("gated", [False, True])
def test_q8_product_refusals(gated):
    lib = B.load()

    def call(x=P, xs=P, n=4, index=None, off=None, experts=1, w=P, ws=P, w3=P, ws3=P, rows=4, K=64, N=32, out=P):
        if gated:
            return lib.moe_q8_gated(x, xs, n, index, off, experts, w, ws, w3, ws3, rows, K, N, out, None)
        return lib.moe_q8_product(x, xs, n, index, off, experts, w, ws, rows, K, N, out, None)

    assert call(rows=0, out=None) == B.MOE_OK
    assert call(experts=2) == B.MOE_EINVAL            # needs expert_offsets
    assert call(experts=0) == B.MOE_EINVAL
    assert call(n=3) == B.MOE_EINVAL                  # fewer rows than out
    assert call(K=0) == B.MOE_EINVAL
    assert call(K=24) == B.MOE_EUNSUPPORTED
    assert call(K=131072) == B.MOE_EUNSUPPORTED
    assert call(N=12) == B.MOE_EUNSUPPORTED
    assert call(experts=1025, off=P) == B.MOE_EUNSUPPORTED
    assert call(index=P, n=2 ** 20, K=4096) == B.MOE_EUNSUPPORTED   # gathered rows past 4 GiB
    for k in ("x", "xs", "w", "ws", "out") + (("w3", "ws3") if gated else ()):
        assert call(**{k: None}) == B.MOE_EINVAL, k
    for k in ("x", "w", "out") + (("w3",) if gated else ()):
        assert call(**{k: P + 8}) == B.MOE_EUNSUPPORTED, k
    assert call(xs=P + 2) == B.MOE_EUNSUPPORTED
    assert ("moe_q8_gated" if gated else "moe_q8_product") in B.moe_stage_last_error(None)


def test_more_rows_than_a_launch_takes():
    """A launch has fewer than 2^32 threads, of which a row or a token has a share."""
    lib, cfg = B.load(), B.make_route_config(8, 2)
    most = 2 ** 31 - 1
    assert lib.moe_q8_rows(P, most, 4096, P, P, None) == B.MOE_EUNSUPPORTED
    assert "rows" in B.moe_stage_last_error(None)
    assert norm(rows=most, hidden=65536) == B.MOE_EUNSUPPORTED
    assert lib.moe_q8_restore(P, P, most, 4096, P, None) == B.MOE_EUNSUPPORTED
    assert lib.moe_route(cfg, P, B.MOE_TYPE_F32, None, most, P, P, None, None) == B.MOE_EUNSUPPORTED


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("rows,grouped,E,K,N", [
    (1048000, True, 1024, 16, 8), (1048000, True, 8, 16, 8), (1048560, False, 1, 16, 8), (1048561, False, 1, 16, 8),
    (1040000, True, 1024, 128, 64), (2 ** 31 - 1, False, 1, 16, 8), (2 ** 31 - 1, True, 1024, 16, 8),
    (2 ** 30, False, 1, 128, 64)])
def test_the_product_chosen_can_be_launched(rows, grouped, E, K, N, gated):
    """No choice whose workgroups are more than a launch takes, at sizes where the estimates prefer the small ones."""
    f = B.load()._ZN3moe7q8_kindElbiiib
    f.argtypes, f.restype = [ctypes.c_int64, ctypes.c_bool] + [ctypes.c_int32] * 3 + [ctypes.c_bool], ctypes.c_int
    kind = f(rows, grouped, E, K, N, gated)
    ends = E if grouped else 0
    if kind < 2:
        assert -(-rows // 16) + ends <= 65535
    elif kind < 4:
        side = 64 if kind == 2 else 128
        cols = -(-N * (2 if gated else 1) // side)
        assert (-(-rows // side) + ends) * cols * 256 < 2 ** 32


def test_binding_checks_tensors():
    torch = pytest.importorskip("torch")
    x = torch.zeros((4, 64), dtype=torch.bfloat16)
    w = torch.zeros(64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="device"):
        B.moe_norm(x, w, 1e-6, out=x)
    with pytest.raises(ValueError, match="weight"):
        B._want("weight", w, (32,), B._BITS16)
    with pytest.raises(ValueError, match="got float"):
        B._opt("weight", 1.5, (64,), B._BITS16)
    assert B._opt("weight", None, (64,), B._BITS16) is None
    with pytest.raises(ValueError, match="two dimensions"):
        B.moe_norm(w, w, 1e-6, out=w)
    cfg = B.make_route_config(8, 2)
    with pytest.raises(ValueError, match="experts = 8"):
        B.moe_route(cfg, x, None, None)
    q = torch.zeros((4, 64), dtype=torch.int8)
    with pytest.raises(ValueError, match="expert_offsets"):
        B.moe_q8_product(q, w, torch.zeros((2, 8, 64), dtype=torch.int8), w, torch.zeros((4, 8), dtype=torch.bfloat16))
    with pytest.raises(ValueError, match="at least"):
        B.moe_q8_product(q, w, torch.zeros((1, 8, 64), dtype=torch.int8), w, torch.zeros((5, 8), dtype=torch.bfloat16))


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("rows,grouped,E,K,N", [
    (1, False, 1, 16, 2 ** 28 - 8), (1, False, 1, 16, 2 ** 28), (1, False, 1, 16, 2 ** 29), (1, False, 1, 128, 2 ** 30),
    (8, True, 4, 16, 2 ** 28), (1, False, 1, 16, 2 ** 31 - 512)])
def test_the_product_chosen_for_many_features_can_be_launched(rows, grouped, E, K, N, gated):
    """A workgroup for 16 or 32 features each, or for a tile's: a launch has fewer than 2^32 threads."""
    f = B.load()._ZN3moe7q8_kindElbiiib
    f.argtypes, f.restype = [ctypes.c_int64, ctypes.c_bool] + [ctypes.c_int32] * 3 + [ctypes.c_bool], ctypes.c_int
    kind, ends = f(rows, grouped, E, K, N, gated), E if grouped else 0
    if kind < 2:
        assert -(-N // (32 if kind == 1 and not gated else 16)) * 256 < 2 ** 32
    elif kind < 4:
        side = 64 if kind == 2 else 128
        assert (-(-rows // side) + ends) * -(-N * (2 if gated else 1) // side) * 256 < 2 ** 32


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("N", [2 ** 31 - 504, 2 ** 31 - 256, 2 ** 31 - 8])
def test_features_past_the_last_tile_have_a_32_bit_number(N, gated):
    lib = B.load()
    if gated:
        rc = lib.moe_q8_gated(P, P, 4, None, None, 1, P, P, P, P, 4, 64, N, P, None)
    else:
        rc = lib.moe_q8_product(P, P, 4, None, None, 1, P, P, 4, 64, N, P, None)
    assert rc == B.MOE_EUNSUPPORTED and "out_features" in B.moe_stage_last_error(None)
