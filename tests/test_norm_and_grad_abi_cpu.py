"""Refusals of the norms around a block and of the calls over many gradients: every call here ends on the host, before anything
is launched (the pointers are no addresses)."""
import ctypes

import pytest
import torch

OK, INVALID, UNSUPPORTED, WORKSPACE, DEVICE = range(5)
P = 0x1000
BAD = ctypes.c_size_t(-1).value


@pytest.fixture(scope="module")
def lib():
    import paper_2411_05288_amd as vp
    return vp.load_library()


def fwd(lib, **k):
    a = dict(x=P, y=P, gate=None, rows=0, w_post=None, b_post=None, w=P, b=None, N=8, h=8, dt=1, flags=0, scale=1.0, eps=1e-5, r=P,
             H=P, stats=P)
    a.update(k)
    return lib.vp_block_norm_fwd(*a.values(), None)


def bwd(lib, **k):
    a = dict(dH=P, dH_dt=0, dr=None, r=P, y=P, gate=None, rows=0, w_post=None, b_post=None, w=P, stats=P, N=8, h=8, dt=1, flags=0,
             scale=1.0, grad_dt=1, dx=P, dy=P, dgate=None, dw_post=None, db_post=None, dw=P, db=None, ws=P, wb=0)
    a.update(k)
    return lib.vp_block_norm_bwd(*a.values(), None)


@pytest.mark.parametrize("wrong", [
    dict(x=None), dict(H=None), dict(N=0), dict(h=0), dict(N=-1), dict(dt=2), dict(dt=-1), dict(flags=1), dict(flags=32),
    dict(rows=1), dict(gate=P), dict(gate=P, rows=3), dict(gate=P, rows=-1), dict(gate=P, rows=16), dict(w_post=P), dict(b_post=P),
    dict(y=None), dict(y=None, r=None, flags=8), dict(y=None, r=None, gate=P, rows=1), dict(eps=0.0), dict(eps=-1.0),
    dict(eps=float("nan")), dict(eps=float("inf")), dict(scale=float("nan")), dict(scale=float("inf")),
    *[{k: P + 8} for k in ("x", "y", "w", "b", "r", "H", "stats")], dict(gate=P + 2, rows=1), dict(w_post=P + 2, flags=8),
    dict(b_post=P + 4, flags=8)])
def test_forward_refuses(lib, wrong):
    assert fwd(lib, **wrong) == INVALID


def test_forward_size_limits(lib):
    assert fwd(lib, h=(1 << 20) + 1) == UNSUPPORTED
    assert fwd(lib, N=1 << 20, h=1 << 11) == UNSUPPORTED
    assert fwd(lib, N=1 << 31, h=1) == UNSUPPORTED


@pytest.mark.parametrize("wrong", [
    dict(dH=None), dict(r=None), dict(stats=None), dict(dx=None), dict(N=0), dict(h=-3), dict(dt=2), dict(dH_dt=2), dict(grad_dt=7),
    dict(dt=0, dH_dt=0, grad_dt=1), dict(dt=0, dH_dt=1, grad_dt=0), dict(flags=1), dict(rows=1), dict(gate=P), dict(gate=P, rows=3),
    dict(w_post=P), dict(b_post=P), dict(y=None), dict(dy=None), dict(y=None, dy=None, flags=8), dict(dgate=P), dict(dw_post=P),
    dict(db_post=P), dict(scale=float("inf")), *[{k: P + 8} for k in ("dH", "dr", "r", "y", "w", "stats", "dx", "dy", "dw", "db", "ws")],
    dict(gate=P, rows=1, dgate=P + 4), dict(flags=8, dw_post=P + 4), dict(flags=8, db_post=P + 4)])
def test_backward_refuses(lib, wrong):
    assert bwd(lib, **{"wb": 1 << 30, **wrong}) == INVALID


def test_backward_workspace_and_limits(lib):
    size = lib.vp_block_norm_bwd_workspace_bytes
    for N, h, rows, flags in ((8, 8, 0, 0), (8, 8, 4, 8), (1, 1, 0, 0), (4096, 8192, 1, 24)):
        need = size(N, h, rows, flags)
        assert 0 < need < BAD
        k = dict(N=N, h=h, rows=rows, gate=P if rows else None, flags=flags)
        assert bwd(lib, wb=need - 1, **k) == WORKSPACE and bwd(lib, ws=None, wb=1 << 40, **k) == WORKSPACE
    for wrong in ((0, 8, 0, 0), (8, 0, 0, 0), (8, 8, 3, 0), (8, 8, -1, 0), (8, 8, 0, 1), (1 << 20, 1 << 11, 0, 0), (1, (1 << 20) + 1, 0, 0)):
        assert size(*wrong) == BAD
    assert bwd(lib, h=(1 << 20) + 1, wb=1 << 40) == UNSUPPORTED
    # partial sums stay within some tens of MB at the sizes of the configurations, and do not grow with the rows of a gate
    assert size(4096, 8192, 4096, 8) <= 256 << 20 and size(1 << 15, 1 << 15, 0, 8) <= 256 << 20


def grads(n=2, ptr=P, count=8, dt=0):
    return ((ctypes.c_void_p * n)(*[ptr] * n), (ctypes.c_int64 * n)(*[count] * n), (ctypes.c_int32 * n)(*[dt] * n), n)


def test_gradient_calls_refuse(lib):
    wb = lib.vp_grad_workspace_bytes(2)
    assert 0 < wb < BAD and lib.vp_grad_workspace_bytes(0) > 0 and lib.vp_grad_workspace_bytes(-1) == BAD
    assert lib.vp_grad_workspace_bytes(100000) < 8 << 20
    calls = [lambda g, norm=P, ws=P, wb=wb, outs=None, most=1.0: lib.vp_grad_norm(*g, norm, ws, wb, None),
             lambda g, norm=P, ws=P, wb=wb, outs=None, most=1.0: lib.vp_grad_clip(*g, outs, most, norm, ws, wb, None),
             lambda g, norm=P, ws=P, wb=wb, outs=None, most=1.0: lib.vp_grad_scale(*g, outs, most, norm, ws, wb, None)]
    for k, call in enumerate(calls):
        assert call(grads(), norm=None) == INVALID and call(grads(), norm=P + 2) == INVALID
        assert call(grads(ptr=None)) == INVALID and call(grads(ptr=P + 2)) == INVALID and call(grads(ptr=P + 1, dt=1)) == INVALID
        assert call(grads(count=-1)) == INVALID and call(grads(dt=2)) == INVALID and call(grads(dt=-1)) == INVALID
        assert call((None, *grads()[1:])) == INVALID and call((*grads()[:3], -1)) == INVALID
        assert call((grads()[0], None, *grads()[2:])) == INVALID and call((*grads()[:2], None, 2)) == INVALID
        assert call(grads(), ws=P + 8) == INVALID
        assert call(grads(), ws=None) == WORKSPACE and call(grads(), wb=wb - 1) == WORKSPACE
        assert call(grads(n=1, count=(1 << 40) + 1)) == UNSUPPORTED and call(grads(count=1 << 62)) == UNSUPPORTED
        if k:
            for most in (-1.0, float("nan"), float("inf")):
                assert call(grads(), most=most) == INVALID
            outs = ctypes.c_void_p * 2
            assert call(grads(), outs=outs(P, None)) == INVALID and call(grads(), outs=outs(P, P + 2)) == INVALID
            assert call(grads(dt=1), outs=outs(P, P + 1)) == INVALID


def test_binding_refuses_wrong_tensors(lib):
    import paper_2411_05288_amd as vp
    x = torch.zeros(4, 8)
    with pytest.raises(vp.VPError, match="x must be"):
        vp.vp_block_norm_fwd(torch.zeros(8), None, x)
    with pytest.raises(vp.VPError, match="r must be"):
        vp.vp_block_norm_bwd(x, torch.zeros(8), None, x, dx=x)
    with pytest.raises(vp.VPError, match="gate must be"):
        vp.vp_block_norm_fwd(x, x, x, gate=torch.zeros(8))
    with pytest.raises(vp.VPError, match="dtype"):
        vp.vp_block_norm_fwd(x.half(), None, x.half())
    with pytest.raises(vp.VPError, match="GPU tensor"):
        vp.GradientArguments([x])
    with pytest.raises(vp.VPError, match="one tensor per gradient"):
        vp.GradientArguments([x], [])
    with pytest.raises(vp.VPError):
        vp.vp_block_norm_bwd_workspace_bytes(0, 8)
    with pytest.raises(vp.VPError):
        vp.vp_grad_workspace_bytes(-1)


def test_gradients_that_share_memory_are_found(monkeypatch):
    import paper_2411_05288_amd.binding as B
    monkeypatch.setattr(B, "_ptr", lambda t, *_: t.data_ptr())      # host tensors: only their addresses are looked at
    w = torch.zeros(1000)
    fine = [([w[:10], w[10:20]], None), ([w[10:20], w[:10], w[5:5]], None), ([w[:10]], [w[:10]]), ([w[:10], w[20:30]], [w[30:40], w[10:20]]),
            ([w[:10], w[:10]], [w[30:40], w[10:20]]), ([w[:10], w[20:30]], [w[:10], w[30:40]]), ([w[5:5]], [w[7:7]])]
    shared = [([w, w], None), ([w[:11], w[10:20]], None), ([w[:10], w[5:8]], None), ([w[:10], w[20:30]], [w[40:50], w[49:59]]),
              ([w[:10], w[20:30]], [w[40:50], w[9:19]]), ([w[:10]], [w[1:11]]), ([w[:10], w[20:30]], [w[20:30], w[:10]]),
              ([w[:100], w[200:210]], [w[300:400], w[40:50]]), ([w[:10], w[:10]], [w[:10], w[50:60]])]
    for grads, outs in fine:
        assert not B.GradientArguments(grads, outs).overlap, (grads, outs)
    for grads, outs in shared:
        assert B.GradientArguments(grads, outs).overlap


def test_plans_refuse(monkeypatch):
    import paper_2411_05288_amd as vp
    W = [torch.zeros(8, 8)]
    with pytest.raises(vp.VPError, match="either H"):
        vp.OutputLayerPlan(None, W, torch.zeros(4, dtype=torch.int64))
    plan = vp.BlockNormPlan(torch.zeros(4, 8), train=False)
    with pytest.raises(vp.VPError, match="train=False"):
        plan.backward(torch.zeros(4, 8))
