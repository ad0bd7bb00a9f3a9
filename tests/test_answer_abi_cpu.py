"""Refusals of the calls that answer (8-bit integers, verification of drafts): every call here ends on the host, before anything
is launched (the pointers are no addresses)."""
import ctypes

import pytest

OK, INVALID, UNSUPPORTED, WORKSPACE, DEVICE = range(5)
BAD = ctypes.c_size_t(-1).value
MB = 1 << 20
P = [k << 40 for k in range(1, 64)]      # addresses far from one another


@pytest.fixture(scope="module")
def lib():
    import paper_2411_05288_amd as vp
    return vp.load_library()


def array(kind, xs):
    return None if xs is None else (kind * len(xs))(*xs)


# ------------------------------------------------------------------------------------------------ vp_quantize_rows
def quantize(lib, **k):
    a = dict(x=P[0], N=8, h=100, dt=1, q=P[1], scales=P[2])
    a.update(k)
    return lib.vp_quantize_rows(*a.values(), None)


def test_row_stride(lib):
    assert [lib.vp_i8_row_stride(h) for h in (1, 127, 128, 129, 4096, 130944)] == [128, 128, 128, 256, 4096, 130944]
    assert [lib.vp_i8_row_stride(h) for h in (0, -1, 130945, 1 << 40)] == [-1] * 4


@pytest.mark.parametrize("wrong", [
    dict(x=None), dict(q=None), dict(scales=None), dict(N=0), dict(N=-1), dict(h=0), dict(h=-5), dict(dt=2), dict(dt=-1),
    dict(x=P[0] + 2), dict(q=P[1] + 8), dict(scales=P[2] + 2),
    dict(q=P[0]), dict(q=P[0] + 1584), dict(scales=P[0] + 1596), dict(scales=P[1] + 1020), dict(q=P[2])])
def test_quantize_refuses(lib, wrong):
    assert quantize(lib, **wrong) == INVALID


def test_quantize_size_limits(lib):
    assert quantize(lib, h=130945) == UNSUPPORTED
    assert quantize(lib, N=1 << 31, h=1) == UNSUPPORTED
    assert quantize(lib, N=1 << 24, h=1) == UNSUPPORTED      # rows of 128 bytes


# ------------------------------------------------------------------------------------------------ vp_output_fwd_i8_group
def product(lib, **k):
    a = dict(H=P[0], Hs=P[1], W=[P[2], P[3]], Ws=[P[4], P[5]], rows=[40, 30], offsets=[0, 40], p=2, labels=P[6], N=8, k=256, dt=1,
             flags=0, m=P[7], s=P[8], t=P[9], logits=None, ws=P[10], wb=MB)
    a.update(k)
    a["W"], a["Ws"], a["logits"] = (array(ctypes.c_void_p, a[n]) for n in ("W", "Ws", "logits"))
    a["rows"], a["offsets"] = (array(ctypes.c_int64, a[n]) for n in ("rows", "offsets"))
    return lib.vp_output_fwd_i8_group(*a.values(), None)


KEPT = dict(flags=1, logits=[P[11], P[12]])


@pytest.mark.parametrize("wrong", [
    *[{n: None} for n in ("H", "Hs", "W", "Ws", "rows", "offsets", "labels", "m", "s", "t")],
    dict(p=0), dict(N=0), dict(k=0), dict(k=-128), dict(k=100), dict(k=64), dict(dt=2), dict(flags=1), dict(flags=2), dict(flags=8),
    dict(logits=[P[11], P[12]]), {**KEPT, "logits": [P[11], None]}, dict(W=[P[2], None]), dict(Ws=[None, P[5]]),
    dict(rows=[40, 0]), dict(rows=[-1, 30]), dict(offsets=[0, -1]),
    dict(H=P[0] + 8), dict(Hs=P[1] + 2), dict(W=[P[2] + 8, P[3]]), dict(Ws=[P[4] + 1, P[5]]), dict(labels=P[6] + 4),
    dict(m=P[7] + 2), dict(s=P[8] + 1), dict(t=P[9] + 2), dict(ws=P[10] + 8), {**KEPT, "logits": [P[11] + 2, P[12]]},
    # shared memory: statistics with each other, the workspace or an input, logits with anything
    dict(s=P[7]), dict(t=P[8] + 60), dict(m=P[1]), dict(m=P[6] + 32), dict(ws=P[3]), dict(ws=P[9]), dict(s=P[5] + 116),
    {**KEPT, "logits": [P[11], P[11]]}, {**KEPT, "logits": [P[11], P[11] + 624]}, {**KEPT, "logits": [P[2], P[12]]},
    {**KEPT, "logits": [P[11], P[0]]}, {**KEPT, "logits": [P[11], P[7]]}, {**KEPT, "logits": [P[4], P[12]]},
    {**KEPT, "logits": [P[10], P[12]]}])
def test_product_refuses(lib, wrong):
    assert product(lib, **wrong) == INVALID


def test_product_size_limits_and_workspace(lib):
    size = lambda p, N, rows: lib.vp_output_i8_workspace_bytes(p, N, array(ctypes.c_int64, rows))      # noqa: E731
    need = size(2, 8, [40, 30])
    assert 0 < need < BAD
    assert product(lib, wb=need - 1) == WORKSPACE and product(lib, ws=None) == WORKSPACE
    assert product(lib, k=1 << 17) == UNSUPPORTED
    assert product(lib, N=1 << 24, wb=1 << 45) == UNSUPPORTED
    assert product(lib, rows=[40, (1 << 20) + 1]) == UNSUPPORTED
    assert product(lib, N=1 << 20, k=128, rows=[40, 1 << 11]) == UNSUPPORTED
    for wrong in ((0, 8, [40]), (1, 0, [40]), (1, -1, [40]), (1, 8, [0]), (2, 8, [40, -1]), (1, 8, [(1 << 20) + 1]), (1, 1 << 31, [1])):
        assert size(*wrong) == BAD
    assert lib.vp_output_i8_workspace_bytes(1, 8, None) == BAD
    # shards beyond one launch's share a workspace
    assert size(40, 8, [256] * 40) == size(16, 8, [256] * 16)


def test_single_shard_refuses(lib):
    a = dict(H=P[0], Hs=P[1], W=P[2], Ws=P[3], labels=P[4], N=8, k=256, Vs=40, offset=0, dt=1, flags=0, m=P[5], s=P[6], t=P[7],
             logits=None, ws=P[8], wb=MB)
    call = lambda **k: lib.vp_output_fwd_i8(*{**a, **k}.values(), None)      # noqa: E731
    for wrong in (dict(W=None), dict(Ws=None), dict(Vs=0), dict(offset=-1), dict(flags=1), dict(logits=P[9]), dict(k=130),
                  dict(m=P[6]), dict(flags=1, logits=P[2])):
        assert call(**wrong) == INVALID
    assert call(wb=0) == WORKSPACE and call(Vs=(1 << 20) + 1) == UNSUPPORTED


# ------------------------------------------------------------------------------------------------ vp_verify_drafts
def verify(lib, **k):
    a = dict(Y=[P[0], P[1]], rows=[40, 30], offsets=[0, 40], p=2, dt=1, m=P[2], s=P[3], Z=None, zm=None, zs=None, drafts=P[4],
             starts=P[5], u=P[6], N=8, sequences=3, accepted=P[7], tokens=P[8], ws=P[9], wb=MB)
    a.update(k)
    a["Y"], a["Z"] = (array(ctypes.c_void_p, a[n]) for n in ("Y", "Z"))
    a["rows"], a["offsets"] = (array(ctypes.c_int64, a[n]) for n in ("rows", "offsets"))
    return lib.vp_verify_drafts(*a.values(), None)


MODEL = dict(Z=[P[10], P[11]], zm=P[12], zs=P[13])


@pytest.mark.parametrize("wrong", [
    *[{n: None} for n in ("Y", "rows", "offsets", "m", "s", "drafts", "starts", "u", "accepted", "tokens")],
    dict(p=0), dict(dt=2), dict(N=0), dict(N=-4), dict(sequences=0), dict(sequences=-1), dict(Y=[P[0], None]),
    {**MODEL, "Z": None}, {**MODEL, "zm": None}, {**MODEL, "zs": None}, {**MODEL, "Z": [None, P[11]]}, dict(zm=P[12]),
    dict(rows=[0, 30]), dict(rows=[40, -1]), dict(offsets=[-1, 40]), dict(offsets=[0, (1 << 63) - 20]),
    dict(offsets=[0, 39]), dict(offsets=[29, 0]), dict(offsets=[7, 7]),
    dict(Y=[P[0] + 1, P[1]]), dict(dt=0, Y=[P[0] + 2, P[1]]), {**MODEL, "Z": [P[10], P[11] + 1]}, dict(m=P[2] + 2), dict(s=P[3] + 1),
    {**MODEL, "zm": P[12] + 2}, {**MODEL, "zs": P[13] + 2}, dict(drafts=P[4] + 4), dict(starts=P[5] + 4), dict(u=P[6] + 2),
    dict(accepted=P[7] + 2), dict(tokens=P[8] + 4), dict(ws=P[9] + 8),
    dict(tokens=P[4]), dict(accepted=P[6] + 28), dict(tokens=P[7] + 8), dict(ws=P[0]), dict(tokens=P[1] + 472), dict(accepted=P[9]),
    dict(tokens=P[5] + 24), {**MODEL, "accepted": P[13]}, {**MODEL, "tokens": P[11]}])
def test_verify_refuses(lib, wrong):
    assert verify(lib, **wrong) == INVALID


def test_verify_size_limits_and_workspace(lib):
    size = lib.vp_verify_workspace_bytes
    need = size(3, 70)
    assert 0 < need < BAD
    assert verify(lib, wb=need - 1) == WORKSPACE and verify(lib, ws=None) == WORKSPACE
    assert verify(lib, **MODEL, wb=need - 1) == WORKSPACE
    assert verify(lib, sequences=(1 << 23) + 1, wb=1 << 45) == UNSUPPORTED
    for wrong in ((0, 70), (-1, 70), (3, 0), (3, -1), (3, 1 << 31), ((1 << 23) + 1, 70)):
        assert size(*wrong) == BAD
    assert verify(lib, p=65, Y=[P[0]] * 65, rows=[1] * 65, offsets=list(range(65))) == UNSUPPORTED
    assert verify(lib, N=1 << 31) == UNSUPPORTED
    assert verify(lib, rows=[40, (1 << 20) + 1]) == UNSUPPORTED
    assert verify(lib, N=1 << 20, rows=[40, 1 << 11], wb=1 << 40) == UNSUPPORTED


@pytest.mark.parametrize("rows", [[1], [128], [129], [1000, 1], [4000] * 8, [16000] * 16, [300] * 17])
def test_a_workspace_suffices_for_fewer_tokens(lib, rows):
    """So one for the largest batch serves all of them, also where fewer tokens have narrower tiles."""
    sizes = [lib.vp_output_i8_workspace_bytes(len(rows), N, array(ctypes.c_int64, rows)) for N in range(1, 300)]
    assert sizes == sorted(sizes)
    sizes = [lib.vp_verify_workspace_bytes(n, sum(rows)) for n in range(1, 300)]
    assert sizes == sorted(sizes)


# ------------------------------------------------------------------------------------------------ vp_logits_stats
def statistics(lib, **k):
    a = dict(Y=[P[0], P[1]], rows=[40, 30], p=2, dt=1, N=8, m=P[2], s=P[3], ws=P[4], wb=MB)
    a.update(k)
    a["Y"], a["rows"] = array(ctypes.c_void_p, a["Y"]), array(ctypes.c_int64, a["rows"])
    return lib.vp_logits_stats(*a.values(), None)


@pytest.mark.parametrize("wrong", [
    *[{n: None} for n in ("Y", "rows", "m", "s")], dict(p=0), dict(p=-1), dict(dt=2), dict(N=0), dict(N=-1), dict(Y=[P[0], None]),
    dict(rows=[0, 30]), dict(rows=[40, -1]), dict(Y=[P[0] + 1, P[1]]), dict(dt=0, Y=[P[0], P[1] + 2]), dict(m=P[2] + 2), dict(s=P[3] + 1),
    dict(ws=P[4] + 8), dict(m=P[3]), dict(s=P[2] + 28), dict(m=P[4]), dict(s=P[0] + 636), dict(m=P[1]), dict(ws=P[1])])
def test_statistics_refuse(lib, wrong):
    assert statistics(lib, **wrong) == INVALID


def test_statistics_size_limits_and_workspace(lib):
    size = lambda p, N, rows: lib.vp_logits_stats_workspace_bytes(p, N, array(ctypes.c_int64, rows))      # noqa: E731
    need = size(2, 8, [40, 30])
    assert 0 < need < BAD
    assert statistics(lib, wb=need - 1) == WORKSPACE and statistics(lib, ws=None) == WORKSPACE
    assert statistics(lib, p=65, Y=[P[0]] * 65, rows=[1] * 65) == UNSUPPORTED
    assert statistics(lib, N=1 << 31) == UNSUPPORTED
    assert statistics(lib, rows=[40, (1 << 20) + 1]) == UNSUPPORTED
    assert statistics(lib, N=1 << 20, rows=[40, 1 << 11], wb=1 << 40) == UNSUPPORTED
    for wrong in ((0, 8, [40]), (65, 8, [40] * 65), (1, 0, [40]), (1, -1, [40]), (1, 8, [0]), (2, 8, [40, -1]), (1, 8, [(1 << 20) + 1]),
                  (1, 1 << 31, [1])):
        assert size(*wrong) == BAD
    assert lib.vp_logits_stats_workspace_bytes(1, 8, None) == BAD
    for rows in ([1], [2048], [2049, 1], [16000] * 16, [300] * 17):
        sizes = [size(len(rows), N, rows) for N in range(1, 300)]
        assert sizes == sorted(sizes)
