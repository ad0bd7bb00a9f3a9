"""Row maxima and sums of exponentials of logits as they are stored, against 64 bits."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def run(shards, stream=None, fill=0xFF):
    """(maximum, sum) of these shards' logits; nothing is written behind the workspace or the results."""
    import paper_2411_05288_amd as vp
    N, need = shards[0].shape[0], vp.vp_logits_stats_workspace_bytes(shards[0].shape[0], [t.shape[1] for t in shards])
    ws = torch.full((need + 256,), fill, dtype=torch.uint8, device="cuda")
    m, s = (torch.full((N + 8,), -7.0, device="cuda") for _ in range(2))
    if stream is not None:
        torch.cuda.synchronize()
    vp.vp_logits_stats(shards, m[:N], s[:N], ws[:need], stream)
    torch.cuda.synchronize()
    assert bool((ws[need:] == fill).all()) and bool((m[N:] == -7).all()) and bool((s[N:] == -7).all())
    return m[:N], s[:N]


def check(shards, got=None):
    """The maximum is exact.  A term exp(-d) of the sum is off by 2^-24 (half a step) of d for the difference, of d for its product with
    log2(e), of 0.23 d for that constant, and by 2 steps of its own; the sum takes 3 + 4 + 6 roundings one after the other within a
    wavefront, and the last one: together below 17."""
    Y = torch.cat([t.double() for t in shards], 1)
    m, s = run(shards) if got is None else got
    top = Y.amax(1)
    assert torch.equal(m.double(), top)
    d = torch.where(Y == -np.inf, 0.0, top[:, None] - Y)
    w = torch.where(Y == -np.inf, 0.0, torch.exp(-d))
    want = w.sum(1)
    bound = ((w * (2.3 * d + 4)).sum(1) / want + 17) * 2.0 ** -24
    assert bool(((s.double() - want).abs() <= bound * want).all())
    return m, s


def make(N, rows, dtype, seed=1, spread=3.0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return [(spread * torch.randn(N, n, generator=gen, device="cuda")).to(TYPES[dtype]) for n in rows]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N", [1, 3, 130])
@pytest.mark.parametrize("rows", [[1], [7], [8], [9], [511], [512], [513], [2047], [2048], [2049, 1], [300, 300, 301], [1] * 64,
                                  [2100] * 64, [16667] * 3, [8200, 5, 4097], [140000, 100]])
def test_sizes(rows, N, dtype):
    check(make(N, rows, dtype, seed=N + len(rows)))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("spread,shift", [(0.0, 0.0), (0.01, 5.0), (30.0, 0.0), (1.0, 1e4), (1.0, -1e4), (1e30, 0.0)])
def test_values(spread, shift, dtype):
    shards = make(40, [3000, 700], dtype, 2, spread)
    check([(t.float() + shift).to(t.dtype) for t in shards])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("value", [-np.inf, -1e30, "min"])
@pytest.mark.parametrize("rows", [[5], [3000, 700], [2048, 2048, 9]])
def test_ruled_out_tokens(rows, value, dtype):
    """Some tokens, all of a chunk or a shard, all but one, and all."""
    value = float(torch.finfo(TYPES[dtype]).min) if value == "min" else value
    V = sum(rows)
    Y = torch.cat(make(8, rows, dtype, 3), 1)
    Y[0, ::3] = value
    Y[1, :rows[0]] = value if len(rows) > 1 else Y[1, :rows[0]]
    Y[2, :-1] = value
    Y[3, 1:] = value
    Y[4, :V // 2] = value
    Y[5, V // 2:] = value
    Y[6] = value
    if value == -np.inf:
        m, s = run([t.contiguous() for t in Y.split(rows, 1)])
        assert m[6].item() == -np.inf and s[6].item() == 0.0
        Y[6] = 1.0
    check([t.contiguous() for t in Y.split(rows, 1)])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows", [[1], [40], [2048, 1], [2500, 600]])
def test_rows_that_hold_no_numbers(rows, dtype):
    """The sum is NaN where a NaN or +inf is, wherever it is and also where nothing else is; the other rows are as without."""
    V = sum(rows)
    clean = torch.cat(make(12, rows, dtype, 4), 1)
    Y = clean.clone()
    Y[0, 0], Y[1, V - 1], Y[2, V // 2] = np.nan, np.nan, np.inf
    Y[3] = np.nan
    Y[4] = np.inf
    Y[5, rows[0] - 1:] = np.nan
    Y[6] = -np.inf
    Y[6, V - 1] = np.nan
    Y[7, :] = -np.inf
    Y[7, 0] = np.inf
    m, s = run([t.contiguous() for t in Y.split(rows, 1)])
    assert bool(torch.isnan(s[:8]).all())
    wm, ws = run([t.contiguous() for t in clean.split(rows, 1)])
    assert torch.equal(m[8:], wm[8:]) and torch.equal(s[8:], ws[8:])


def test_rows_that_start_at_any_element():
    import paper_2411_05288_amd as vp
    for dtype in TYPES:
        for at in range(1, 9):
            flat = torch.cat([t.view(-1) for t in make(1, [9000], dtype, at)])
            shards = [flat[at:at + 5 * 777].view(5, 777), flat[4000 + at:4000 + at + 5 * 601].view(5, 601)]
            check(shards)
            m, s = torch.zeros(16, device="cuda")[at:at + 5], torch.zeros(16, device="cuda")[at + 1:at + 6]
            ws = torch.empty(vp.vp_logits_stats_workspace_bytes(9, [777, 601]), dtype=torch.uint8, device="cuda")      # (of more rows)
            vp.vp_logits_stats(shards, m, s, ws)
            torch.cuda.synchronize()
            check(shards, (m, s))


def test_many_short_rows():
    """More rows than workgroups of a launch, and than the launch that joins them has wavefronts."""
    N = (1 << 23) + 1001
    Y = torch.arange(2 * N, device="cuda", dtype=torch.float32).remainder_(97).view(N, 2).mul_(0.125)
    m, s = run([Y])
    assert torch.equal(m, Y.amax(1))
    want = torch.exp(Y.double() - m[:, None].double()).sum(1)
    assert bool(((s.double() - want).abs() <= 60 * 2.0 ** -24 * want).all())      # (d <= 12: 2.3 d + 4 + 17, and slack)


def test_rows_beyond_32_bits():
    N, V = 2047, 1 << 20
    Y = torch.zeros(N, V, dtype=torch.bfloat16, device="cuda")
    Y[N - 2:] = torch.randn(2, V, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda")
    m, s = run([Y])
    assert bool((m[:N - 2] == 0).all()) and bool((s[:N - 2] == V).all())
    check([Y[N - 2:]], (m[N - 2:], s[N - 2:]))


def test_results_repeat_on_another_stream_and_in_a_graph():
    import paper_2411_05288_amd as vp
    shards = make(37, [5000, 900], "bf16", 6)
    want = check(shards)
    stream = torch.cuda.Stream()
    for argument in (stream, stream.cuda_stream):
        for a, b in zip(run(shards, argument, fill=0x7F), want):
            assert torch.equal(a, b)
    ws = torch.empty(vp.vp_logits_stats_workspace_bytes(37, [5000, 900]), dtype=torch.uint8, device="cuda")
    m, s = torch.empty(37, device="cuda"), torch.empty(37, device="cuda")
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        vp.vp_logits_stats(shards, m, s, ws)
    torch.cuda.current_stream().wait_stream(stream)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        vp.vp_logits_stats(shards, m, s, ws)
    gen = torch.Generator(device="cuda").manual_seed(7)
    for _ in range(4):
        for t in shards:
            t.copy_(3 * torch.randn(t.shape, generator=gen, device="cuda"))
        want = run(shards)
        m.fill_(5)
        ws.fill_(0xFF)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(m, want[0]) and torch.equal(s, want[1])


def test_the_checks_in_python_lead_to_the_same_call(monkeypatch):
    import paper_2411_05288_amd.binding as B
    B.load_library()
    shards = make(9, [300, 77], "f32", 8)
    native = run(shards)
    assert B._HOST is not None
    monkeypatch.setattr(B, "_HOST", None)
    for a, b in zip(native, run(shards)):
        assert torch.equal(a, b)


def test_python_refusals():
    import paper_2411_05288_amd as vp
    z = lambda *s, dtype=torch.float32: torch.zeros(*s, dtype=dtype, device="cuda")      # noqa: E731
    good = dict(logits=[z(7, 30), z(7, 20)], global_max=z(7), global_sumexp=z(7), workspace=z(4096, dtype=torch.uint8))
    vp.vp_logits_stats(**good)
    for bad in (dict(logits=[]), dict(logits=[z(7, 30), z(6, 20)]), dict(logits=[z(7, 30), z(7, 20, dtype=torch.bfloat16)]),
                dict(logits=[z(7, 30, dtype=torch.float64)]), dict(logits=[z(7)]), dict(logits=[z(30, 7).t()]), dict(logits=[z(7, 0)]),
                dict(logits=[z(0, 7)], global_max=z(0), global_sumexp=z(0)), dict(logits=[torch.zeros(7, 30)]), dict(global_max=z(6)),
                dict(global_sumexp=z(7, dtype=torch.float64)), dict(global_max=good["global_sumexp"]), dict(workspace=None),
                dict(workspace=z(8, dtype=torch.uint8)), dict(logits=[z(7, 3)] * 65), dict(logits=[good["workspace"].view(torch.float32)[:70].view(7, 10)])):
        with pytest.raises(vp.VPError):
            vp.vp_logits_stats(**{**good, **bad})
    with pytest.raises(vp.VPError):
        vp.vp_logits_stats_workspace_bytes(0, [5])
