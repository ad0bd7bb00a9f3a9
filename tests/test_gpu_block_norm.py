"""The norms around a block (vp_block_norm_fwd, vp_block_norm_bwd) against their formulas in 64 bits, every output element
within a bound that follows from the roundings of a computation in 32 bits (norm_reference.py)."""
import itertools

import pytest
import torch

import norm_reference as ref

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
# lengths from one element to rows that no workgroup holds, odd ones, powers of two and their neighbours
SIZES = [(1, 1), (3, 7), (70, 8), (5, 63), (5, 64), (129, 65), (1, 128), (128, 256), (33, 511), (34, 1000), (17, 1001), (12, 1024),
         (64, 2050), (77, 200), (41, 129), (7, 4096), (301, 4096), (9, 4104), (6, 8192), (3, 8200), (5, 12288), (4, 16384), (3, 16391), (2, 32768),
         (2, 40001), (1, 70000), (1000, 40), (4099, 24)]


def guarded(shape, dtype, fill=7.0):
    """A tensor inside a larger one, and a check that what lies around it stays as it was."""
    n = 1
    for s in shape:
        n *= s
    pad = 64
    whole = torch.full((n + 2 * pad,), fill, dtype=dtype, device="cuda")
    inner = whole[pad:pad + n].view(shape)

    def untouched():
        return bool((whole[:pad] == fill).all()) and bool((whole[pad + n:] == fill).all())
    return inner, untouched


def inputs(N, h, dtype, post, gate, bias, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape, std=1.0, mean=0.0):
        return (torch.randn(*shape, generator=g, device="cuda") * std + mean).to(dtype)
    return {"x": normal(N, h, mean=0.3), "y": normal(N, h, std=2.0, mean=-0.4), "gate": normal(gate, h, std=0.5, mean=0.2) if gate else None,
            "w": normal(h, std=0.2, mean=1.0) if seed % 5 else None, "b": normal(h, std=0.3) if bias else None,
            "w_post": normal(h, std=0.2, mean=1.0) if post and seed % 7 else None, "b_post": normal(h, std=0.3) if post and bias else None}


def gates(N):
    """Rows of a gate: none, one, one for every token, and splits in between."""
    some = [g for g in range(2, N) if N % g == 0]
    return [0, 1, N] + some[:1] + some[-1:] + some[len(some) // 2:len(some) // 2 + 1]


def variants():
    out = []
    for k, (N, h) in enumerate(SIZES):
        for j, (dtype, post, center) in enumerate(itertools.product((BF16, F32), (True, False), (True, False))):
            gs = gates(N)
            out.append((N, h, dtype, post, center, gs[(k + j) % len(gs)], (k + j // 2) % 2 == 0, 10 * k + j))
    return out


@pytest.mark.parametrize("N,h,dtype,post,center,gate,bias,seed", variants())
def test_forward_and_backward(N, h, dtype, post, center, gate, bias, seed):
    import paper_2411_05288_amd as vp
    s = inputs(N, h, dtype, post, gate, bias, seed)
    scale, eps = (1.0, 0.37, -1.25)[seed % 3], (1e-5, 1e-6, 0.1)[seed % 3]
    opts = dict(gate=s["gate"], w_post=s["w_post"], b_post=s["b_post"], scale=scale, post=post, center=center)
    (H, H_ok), (r, r_ok), (stats, s_ok) = guarded((N, h), dtype), guarded((N, h), dtype), guarded((4, N), F32)
    vp.vp_block_norm_fwd(s["x"], s["y"], H, r=r, stats=stats, w=s["w"], b=s["b"], eps=eps, **opts)
    for name, (value, bound) in ref.forward(s["x"], s["y"], w=s["w"], b=s["b"], eps=eps, **opts).items():
        ref.check(name, {"r": r, "H": H, "stats": stats}[name], value, bound)
    assert H_ok() and r_ok() and s_ok()

    dH_type = (F32, dtype)[seed % 2]
    grad = (dtype, F32)[seed // 2 % 2]
    g = torch.Generator(device="cuda").manual_seed(seed + 1)
    dH = torch.randn(N, h, generator=g, device="cuda").to(dH_type)
    dr = torch.randn(N, h, generator=g, device="cuda").to(grad) if seed % 4 else None
    want = ["dx", "dy", "dw", "db"] + (["dgate"] if gate else []) + (["dw_post", "db_post"] if post else [])
    shapes = {"dx": ((N, h), grad), "dy": ((N, h), grad), "dgate": ((gate, h), F32)}
    out = {k: guarded(*shapes.get(k, ((h,), F32))) for k in want}
    ws = torch.full((vp.vp_block_norm_bwd_workspace_bytes(N, h, gate, post),), 0xFF, dtype=torch.uint8, device="cuda")
    vp.vp_block_norm_bwd(dH, r, s["y"], stats, dr=dr, w=s["w"], workspace=ws, **{k: t for k, (t, _) in out.items()}, **opts)
    expected = ref.backward(dH, r, s["y"], stats, dr=dr, w=s["w"], grad_dtype=grad, **opts)
    assert sorted(expected) == sorted(want)
    for name, (value, bound) in expected.items():
        ref.check(name, out[name][0], value, bound)
        assert out[name][1](), name
    # the same again: bit for bit
    again = {k: torch.empty_like(t) for k, (t, _) in out.items()}
    vp.vp_block_norm_bwd(dH, r, s["y"], stats, dr=dr, w=s["w"], workspace=ws, **again, **opts)
    for k, t in again.items():
        assert torch.equal(t, out[k][0]), k


@pytest.mark.parametrize("N,h,dtype,center", [(1, 4096, BF16, False), (5, 1001, F32, True), (130, 320, BF16, True), (2, 33333, BF16, False)])
def test_norm_alone(N, h, dtype, center):
    import paper_2411_05288_amd as vp
    s = inputs(N, h, dtype, False, 0, True, 3)
    H, stats = torch.empty_like(s["x"]), torch.empty(4, N, device="cuda")
    vp.vp_block_norm_fwd(s["x"], None, H, stats=stats, w=s["w"], b=s["b"], center=center)
    expected = ref.forward(s["x"], w=s["w"], b=s["b"], center=center)
    ref.check("H", H, *expected["H"])
    ref.check("stats", stats, *expected["stats"])
    bare = torch.empty_like(H)      # serving: nothing kept
    vp.vp_block_norm_fwd(s["x"], None, bare, w=s["w"], b=s["b"], center=center)
    assert torch.equal(bare, H)
    dH, dx, dw = torch.randn(N, h, device="cuda"), torch.empty(N, h, device="cuda"), torch.empty(h, device="cuda")
    ws = torch.full((vp.vp_block_norm_bwd_workspace_bytes(N, h),), 0xFF, dtype=torch.uint8, device="cuda")
    vp.vp_block_norm_bwd(dH, s["x"], None, stats, dx=dx, w=s["w"], dw=dw, center=center, workspace=ws)
    expected = ref.backward(dH, s["x"], None, stats, w=s["w"], center=center)
    ref.check("dx", dx, *expected["dx"])
    ref.check("dw", dw, *expected["dw"])


@pytest.mark.parametrize("N,h", [(9, 1000), (3, 4096), (2, 40000), (700, 77), (700, 205), (600, 1001), (300, 4099), (40, 9001), (20, 18437), (50, 5)])
def test_in_place(N, h):
    import paper_2411_05288_amd as vp
    s = inputs(N, h, BF16, True, 1, True, 4)
    opts = dict(gate=s["gate"], w_post=s["w_post"], b_post=s["b_post"], post=True, scale=0.5)
    H, r, stats = torch.empty_like(s["x"]), torch.empty_like(s["x"]), torch.empty(4, N, device="cuda")
    vp.vp_block_norm_fwd(s["x"], s["y"], H, r=r, stats=stats, w=s["w"], b=s["b"], **opts)
    x, y = s["x"].clone(), s["y"].clone()
    vp.vp_block_norm_fwd(x, y, y, r=x, w=s["w"], b=s["b"], **opts)
    assert torch.equal(x, r) and torch.equal(y, H)
    dH, dr = torch.randn(N, h, device="cuda").bfloat16(), torch.randn(N, h, device="cuda").bfloat16()
    ws = torch.empty(vp.vp_block_norm_bwd_workspace_bytes(N, h, 1, post=True), dtype=torch.uint8, device="cuda")

    def back(dr, dx):
        out = {"dx": dx, "dy": torch.empty_like(dx), "dgate": torch.empty(1, h, device="cuda"), "dw": torch.empty(h, device="cuda")}
        vp.vp_block_norm_bwd(dH, r, s["y"], stats, dr=dr, w=s["w"], workspace=ws, **out, **opts)
        return out
    apart = back(dr, torch.empty_like(dr))
    inside = back(dr, dr)
    for k in apart:
        assert torch.equal(apart[k], inside[k]), k


@pytest.mark.parametrize("N,h,gate", [(6, 96, 3), (4, 1000, 1)])
@pytest.mark.parametrize("center", [True, False])
def test_gradients_against_differences(N, h, gate, center):
    """Directional derivatives of <dH, H> + <dr, r> by central differences of the forward formulas in 64 bits."""
    import paper_2411_05288_amd as vp
    s = inputs(N, h, F32, True, gate, True, 11)
    leaves = ["x", "y", "gate", "w", "b", "w_post", "b_post"]
    opts = dict(scale=0.7, post=True, center=center)
    H, r, stats = torch.empty_like(s["x"]), torch.empty_like(s["x"]), torch.empty(4, N, device="cuda")
    vp.vp_block_norm_fwd(s["x"], s["y"], H, r=r, stats=stats, gate=s["gate"], w=s["w"], b=s["b"], w_post=s["w_post"],
                         b_post=s["b_post"], **opts)
    dH, dr = torch.randn(N, h, device="cuda"), torch.randn(N, h, device="cuda")
    names = {"x": "dx", "y": "dy", "gate": "dgate", "w": "dw", "b": "db", "w_post": "dw_post", "b_post": "db_post"}
    out = {names[k]: torch.empty_like(s[k]) for k in leaves}
    ws = torch.empty(vp.vp_block_norm_bwd_workspace_bytes(N, h, gate, post=True), dtype=torch.uint8, device="cuda")
    vp.vp_block_norm_bwd(dH, r, s["y"], stats, dr=dr, gate=s["gate"], w=s["w"], w_post=s["w_post"], b_post=s["b_post"],
                         workspace=ws, **out, **opts)
    expected = ref.backward(dH, r, s["y"], stats, dr=dr, gate=s["gate"], w=s["w"], w_post=s["w_post"], b_post=s["b_post"], **opts)
    p = {k: s[k].double() for k in leaves}

    def loss(q):      # the forward formulas, from inputs in 64 bits
        o = ref.forward(**{**q}, **opts)
        return float((o["H"][0] * dH.double()).sum() + (o["r"][0] * dr.double()).sum())
    ref.HALF.setdefault(torch.float64, 0.0)
    for k in leaves:
        way = torch.randn(p[k].shape, device="cuda", dtype=torch.float64)
        e = 1e-5
        # central differences: truncation of order e^2, rounding of order 1e-16 / e
        slope = (loss({**p, k: p[k] + e * way}) - loss({**p, k: p[k] - e * way})) / (2 * e)
        got = float((out[names[k]].double() * way).sum())
        # every element of the gradient is within its bound; r and the statistics that the kernel read are rounded to 32 bits
        # (a relative change of the gradient of some 2^-23 for each of six uses), and the differences are good to 1e-7
        value, bound = expected[names[k]]
        room = float((bound * way.abs()).sum()) + float((value * way).abs().sum()) * (6 * 2.0 ** -23 + 1e-7) + 1e-6
        assert abs(got - slope) <= room, (k, got, slope, room)


def test_nan_and_inf_stay_in_their_rows():
    import paper_2411_05288_amd as vp
    N, h = 8, 1000
    s = inputs(N, h, BF16, True, 0, False, 1)
    clean = {k: v.clone() for k, v in s.items() if v is not None}
    s["x"][2, 5], s["y"][4, 7], s["x"][6, 0] = float("nan"), float("inf"), float("-inf")
    outs = []
    for q in (clean, s):
        H, r, stats = torch.empty_like(s["x"]), torch.empty_like(s["x"]), torch.empty(4, N, device="cuda")
        vp.vp_block_norm_fwd(q["x"], q["y"], H, r=r, stats=stats, w=s["w"], w_post=s["w_post"], post=True)
        outs.append((H, r, stats))
    for row in range(N):
        same = [torch.equal(a[row], b[row]) for a, b in zip(outs[0][:2], outs[1][:2])] + [torch.equal(outs[0][2][:, row], outs[1][2][:, row])]
        assert all(same) if row not in (2, 4, 6) else not all(same), row
    assert bool(torch.isnan(outs[1][0][2]).any())


def test_zero_rows_and_gates():
    import paper_2411_05288_amd as vp
    N, h = 4, 640
    x = torch.zeros(N, h, device="cuda")
    H = torch.full_like(x, 7.0)
    stats = torch.empty(4, N, device="cuda")
    vp.vp_block_norm_fwd(x, None, H, stats=stats, eps=1e-6)
    assert bool((H == 0).all()) and torch.allclose(stats[3], torch.full((N,), 1e3, device="cuda"), rtol=1e-6)
    y = torch.randn(N, h, device="cuda")
    r = torch.empty_like(x)
    x = torch.randn(N, h, device="cuda")
    vp.vp_block_norm_fwd(x, y, H, r=r, gate=torch.zeros(1, h, device="cuda"), post=True)
    assert torch.equal(r, x)


def test_other_stream_and_graph():
    import paper_2411_05288_amd as vp
    N, h, G = 60, 1032, 5
    s = inputs(N, h, BF16, True, G, True, 2)
    plan = vp.BlockNormPlan(s["x"], s["y"], gate=s["gate"], w=s["w"], b=s["b"], w_post=s["w_post"], b_post=s["b_post"], scale=0.5,
                            post=True, center=True)
    dH, dr = torch.randn(N, h, device="cuda"), torch.randn(N, h, device="cuda").bfloat16()
    outs = [plan.r, plan.H, plan.stats, plan.dx, plan.dy] + plan.parameter_gradients()

    def step(stream=None):
        plan.forward(stream)
        plan.backward(dH, dr, stream)
    step()
    torch.cuda.synchronize()
    expected = [t.clone() for t in outs]
    side = torch.cuda.Stream()
    for stream in (side, side.cuda_stream):
        for t in outs:
            t.fill_(float("nan"))
        torch.cuda.synchronize()
        step(stream)
        side.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, expected))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(3):
        for t in outs + [plan.workspace]:
            t.fill_(float("nan") if t.is_floating_point() else 0xFF)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, expected))
        assert float(torch.arange(1000, device="cuda", dtype=torch.float32).sum()) == 499500.0


def test_gradients_that_are_not_wanted():
    import paper_2411_05288_amd as vp
    N, h = 50, 1200
    s = inputs(N, h, BF16, True, 10, True, 8)
    opts = dict(gate=s["gate"], w_post=s["w_post"], b_post=s["b_post"], post=True, center=True)
    H, r, stats = torch.empty_like(s["x"]), torch.empty_like(s["x"]), torch.empty(4, N, device="cuda")
    vp.vp_block_norm_fwd(s["x"], s["y"], H, r=r, stats=stats, w=s["w"], b=s["b"], **opts)
    dH = torch.randn(N, h, device="cuda")
    ws = torch.empty(vp.vp_block_norm_bwd_workspace_bytes(N, h, 10, post=True), dtype=torch.uint8, device="cuda")
    every = {"dgate": (10, h), "dw": (h,), "db": (h,), "dw_post": (h,), "db_post": (h,)}
    results = []
    for names in [list(every)] + [[k] for k in every] + [[]]:
        out = {k: torch.empty(every[k], device="cuda") for k in names}
        out["dx"], out["dy"] = torch.empty_like(r), torch.empty_like(r)
        ws.fill_(0xFF)
        vp.vp_block_norm_bwd(dH, r, s["y"], stats, w=s["w"], workspace=ws, **out, **opts)
        results.append(out)
        for k in out:
            assert torch.equal(out[k], results[0][k]), (names, k)


def test_wrong_tensors_are_refused_and_launch_nothing(monkeypatch):
    """The same by the native checks and by those in Python."""
    import paper_2411_05288_amd as vp
    import paper_2411_05288_amd.binding as B
    N, h = 6, 64
    s = inputs(N, h, BF16, True, 3, True, 1)
    wide = torch.zeros(N, 2 * h, dtype=BF16, device="cuda")
    stats, ws = torch.ones(4, N, device="cuda"), torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    f = torch.float32
    good = dict(x=s["x"], y=s["y"], H=torch.full_like(s["x"], 7.0), r=torch.full_like(s["x"], 7.0), stats=stats, gate=s["gate"], w=s["w"],
                b=s["b"], w_post=s["w_post"], b_post=s["b_post"], post=True)
    bad = [dict(x=s["x"].half()), dict(x=wide[:, :h]), dict(x=s["x"].cpu()), dict(x=s["x"][0]), dict(y=s["y"][:5]), dict(y=s["y"].float()),
           dict(y=wide[:, ::2]), dict(H=None), dict(H=good["H"].float()), dict(H=good["H"].cpu()), dict(r=wide), dict(stats=stats[:3]),
           dict(stats=stats.double()), dict(gate=s["gate"][0]), dict(gate=s["gate"][:, :32]), dict(gate=torch.zeros(4, h, dtype=BF16, device="cuda")),
           dict(w=s["w"].float()), dict(w=s["w"][:63]), dict(b=s["b"].cpu()), dict(w_post=s["w_post"][None]), dict(b_post=wide[0, ::2]),
           dict(post=False), dict(eps=0.0), dict(eps=float("nan")), dict(scale=float("inf")), dict(y=None), dict(x=wide.view(-1)[1:1 + N * h].view(N, h))]
    back = dict(dH=torch.zeros(N, h, device="cuda"), r=s["x"], y=s["y"], stats=stats, dx=torch.full((N, h), 7.0, device="cuda"),
                dy=torch.full((N, h), 7.0, device="cuda"), gate=s["gate"], w=s["w"], w_post=s["w_post"], b_post=s["b_post"], post=True,
                dw=torch.full((h,), 7.0, device="cuda"), workspace=ws)
    worse = [dict(dH=back["dH"][:5]), dict(dH=back["dH"].double()), dict(dH=back["dH"].cpu()), dict(r=wide), dict(dx=back["dx"].half()), dict(dy=None),
             dict(dx=back["dx"].bfloat16()), dict(dr=torch.zeros(N, h, dtype=BF16, device="cuda")), dict(dw=back["dw"].bfloat16()),
             dict(db=torch.zeros(63, device="cuda")), dict(dgate=torch.zeros(2, h, device="cuda")), dict(dgate=torch.zeros(h, device="cuda")),
             dict(workspace=None), dict(workspace=ws[:64]), dict(workspace=ws.cpu()), dict(workspace=ws[8:]), dict(stats=None), dict(post=False),
             dict(y=None), dict(gate=None, dgate=torch.zeros(3, h, device="cuda"))]
    B.load_library()
    for host in (B._HOST, None):
        monkeypatch.setattr(B, "_HOST", host)
        for wrong in bad:
            with pytest.raises(vp.VPError):
                vp.vp_block_norm_fwd(**{**good, **wrong})
        for wrong in worse:
            with pytest.raises(vp.VPError):
                vp.vp_block_norm_bwd(**{**back, **wrong})
        torch.cuda.synchronize()
        for t in (good["H"], good["r"], back["dx"], back["dy"], back["dw"]):
            assert bool((t == 7).all())
        assert bool((stats == 1).all())
        # both ways give the same
        out = [torch.empty_like(s["x"]), torch.empty_like(s["x"]), torch.empty_like(stats)]
        vp.vp_block_norm_fwd(**{**good, "H": out[0], "r": out[1], "stats": out[2]})
        if host is not None:
            first = out
        assert all(torch.equal(a, b) for a, b in zip(out, first))
    with pytest.raises(TypeError):
        vp.vp_grad_clip([back["dx"]], None, back["dw"][:1], ws)


def test_bf16_as_bit_patterns():
    import paper_2411_05288_amd as vp
    s = inputs(5, 200, BF16, False, 0, False, 6)
    a, b = torch.empty_like(s["x"]), torch.empty_like(s["x"])
    vp.vp_block_norm_fwd(s["x"], None, a, w=s["w"])
    vp.vp_block_norm_fwd(s["x"].view(torch.int16), None, b, w=s["w"])
    assert torch.equal(a, b)


def test_offsets_beyond_32_bits():
    """The rows at both ends of tensors of more than 2^32 bytes."""
    import paper_2411_05288_amd as vp
    N, h = 262149, 4100
    g = torch.Generator(device="cuda").manual_seed(1)
    x, y = (torch.randn(N, h, generator=g, device="cuda") for _ in range(2))
    assert x.numel() * 4 > 1 << 32
    H, r, stats = torch.empty_like(x), torch.empty_like(x), torch.empty(4, N, device="cuda")
    vp.vp_block_norm_fwd(x, y, H, r=r, stats=stats, post=True, center=True)
    ends = torch.tensor([0, 1, N // 2, N - 2, N - 1], device="cuda")
    for name, (value, bound) in ref.forward(x[ends], y[ends], post=True, center=True).items():
        ref.check(name, {"r": r[ends], "H": H[ends], "stats": stats[:, ends]}[name], value, bound)
    dr = x      # (any values)
    dx, dy = torch.empty_like(x), torch.empty_like(x)
    ws = torch.empty(vp.vp_block_norm_bwd_workspace_bytes(N, h, post=True), dtype=torch.uint8, device="cuda")
    vp.vp_block_norm_bwd(H, r, y, stats, dr=dr, dx=dx, dy=dy, post=True, center=True, workspace=ws)
    expected = ref.backward(H[ends], r[ends], y[ends], stats[:, ends], dr=dr[ends], post=True, center=True)
    ref.check("dx", dx[ends], *expected["dx"])
    ref.check("dy", dy[ends], *expected["dy"])


@pytest.mark.parametrize("N,h", [(1500, 264), (40, 9000), (300, 5)])
def test_two_streams_at_once(N, h):
    """Calls that overlap, each with buffers and a workspace of its own."""
    import paper_2411_05288_amd as vp
    s = inputs(N, h, BF16, True, 1, True, 9)
    plans = [vp.BlockNormPlan(s["x"], s["y"], gate=s["gate"], w=s["w"], b=s["b"], w_post=s["w_post"], b_post=s["b_post"], post=True) for _ in range(3)]
    dH = torch.randn(N, h, device="cuda")
    streams = [torch.cuda.Stream() for _ in plans]
    torch.cuda.synchronize()
    for _ in range(4):
        for plan, stream in zip(plans, streams):
            plan.forward(stream)
            plan.backward(dH, stream=stream)
    torch.cuda.synchronize()
    for plan in plans[1:]:
        for a, b in zip([plan.r, plan.H, plan.stats, plan.dx, plan.dy] + plan.parameter_gradients(),
                        [plans[0].r, plans[0].H, plans[0].stats, plans[0].dx, plans[0].dy] + plans[0].parameter_gradients()):
            assert torch.equal(a, b)


TYPES = [(F32, F32, F32), (BF16, F32, F32), (BF16, F32, BF16), (BF16, BF16, F32), (BF16, BF16, BF16)]


@pytest.mark.parametrize("dtype,dH_type,grad", TYPES)
@pytest.mark.parametrize("post,bias", list(itertools.product((False, True), repeat=2)))
@pytest.mark.parametrize("N,h,gate", [(N, h, gate) for N, h in ((612, 90), (612, 250), (36, 1043), (612, 520), (36, 8203), (36, 4), (12, 260), (12, 18437), (12, 33000))
                                      for gate in (0, 1, 4, 12, 36, 612) if not gate or N % gate == 0])
def test_every_backward_kernel(N, h, post, gate, bias, dtype, dH_type, grad):
    """All types and parts at rows of lanes, wavefronts and a workgroup, two vectors per thread, and lengths below a vector; a
    gate per channel, per token, and with rows that lie within and across what a group of threads sums."""
    import paper_2411_05288_amd as vp
    seed = h + 2 * gate + bias
    s = inputs(N, h, dtype, post, gate, bias, seed)
    opts = dict(gate=s["gate"], w_post=s["w_post"], b_post=s["b_post"], scale=0.75, post=post, center=bias)
    H, r, stats = torch.empty_like(s["x"]), torch.empty_like(s["x"]), torch.empty(4, N, device="cuda")
    vp.vp_block_norm_fwd(s["x"], s["y"], H, r=r, stats=stats, w=s["w"], b=s["b"], **opts)
    dH, dr = torch.randn(N, h, device="cuda").to(dH_type), torch.randn(N, h, device="cuda").to(grad)
    shapes = {"dx": ((N, h), grad), "dy": ((N, h), grad), "dgate": ((gate, h), F32)}
    want = ["dx", "dy", "dw"] + (["db"] if bias else []) + (["dgate"] if gate else [])
    want += (["dw_post"] + (["db_post"] if bias else [])) if post else []
    out = {k: guarded(*shapes.get(k, ((h,), F32))) for k in want}
    size = vp.vp_block_norm_bwd_workspace_bytes(N, h, gate, post)
    ws, ws_ok = guarded((size,), torch.uint8, 0xFF)
    vp.vp_block_norm_bwd(dH, r, s["y"], stats, dr=dr, w=s["w"], workspace=ws, **{k: t for k, (t, _) in out.items()}, **opts)
    expected = ref.backward(dH, r, s["y"], stats, dr=dr, w=s["w"], grad_dtype=grad, **opts)
    for name in want:
        ref.check(name, out[name][0], *expected[name])
        assert out[name][1](), name
    assert ws_ok()


@pytest.mark.parametrize("N,h,dtype", [(9, 1000, F32), (700, 77, BF16), (700, 205, BF16), (300, 4099, BF16), (40, 9001, F32), (20, 18437, BF16),
                                       (2, 40000, F32), (50, 5, BF16)])
@pytest.mark.parametrize("center", [False, True])
def test_norm_alone_in_place(N, h, dtype, center):
    import paper_2411_05288_amd as vp
    s = inputs(N, h, dtype, False, 0, True, 3)
    H, stats = torch.empty_like(s["x"]), torch.empty(4, N, device="cuda")
    vp.vp_block_norm_fwd(s["x"], None, H, stats=stats, w=s["w"], b=s["b"], center=center)
    x = s["x"].clone()
    vp.vp_block_norm_fwd(x, None, x, w=s["w"], b=s["b"], center=center)
    assert torch.equal(x, H)


def test_outputs_that_share_memory_are_refused():
    import paper_2411_05288_amd as vp
    N, h = 6, 64
    s = inputs(N, h, BF16, True, 3, True, 1)
    opts = dict(gate=s["gate"], w_post=s["w_post"], b_post=s["b_post"], post=True)
    kept = {k: v.clone() for k, v in s.items()}
    H, r, stats = torch.empty_like(s["x"]), torch.empty_like(s["x"]), torch.ones(4, N, device="cuda")
    for wrong in (dict(H=s["x"]), dict(r=s["y"]), dict(r=H), dict(H=s["y"], r=s["y"]), dict(x=s["y"], H=s["y"])):
        with pytest.raises(vp.VPError, match="vp_block_norm_fwd failed: VP_ERR_INVALID_ARG"):
            vp.vp_block_norm_fwd(**{**dict(x=s["x"], y=s["y"], H=H, r=r, stats=stats, w=s["w"], b=s["b"]), **opts, **wrong})
    whole = torch.ones(1 << 18, device="cuda")
    dH, dr, ws = whole[:N * h].view(N, h), torch.ones(N, h, device="cuda"), torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    dx, dy, dw = torch.empty_like(dH), torch.empty_like(dH), torch.empty(h, device="cuda")
    for wrong in (dict(dx=dH), dict(dy=dr), dict(dy=dx), dict(dw=dx[0]), dict(dw=dH[1]), dict(dw_post=dw), dict(workspace=whole.view(torch.uint8)),
                  dict(dgate=dr[:3]), dict(dgate=dx[2:5])):
        with pytest.raises(vp.VPError, match="vp_block_norm_bwd failed: VP_ERR_INVALID_ARG"):
            vp.vp_block_norm_bwd(**{**dict(dH=dH, r=s["x"], y=s["y"], stats=stats, dx=dx, dy=dy, dr=dr, w=s["w"], dw=dw, workspace=ws), **opts, **wrong})
    torch.cuda.synchronize()
    assert all(torch.equal(v, kept[k]) for k, v in s.items())
    assert all(bool((t == 1).all()) for t in (dH, dr, stats))


def test_a_gate_without_rows_is_refused(monkeypatch):
    """The same by the native checks and by those in Python."""
    import paper_2411_05288_amd as vp
    import paper_2411_05288_amd.binding as B
    N, h = 4, 64
    x, y, gate = torch.ones(N, h, device="cuda"), torch.ones(N, h, device="cuda"), torch.empty(0, h, device="cuda")
    H, stats, dx, dy = torch.full_like(x, 7.0), torch.ones(4, N, device="cuda"), torch.full_like(x, 7.0), torch.full_like(x, 7.0)
    ws = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    B.load_library()
    for host in (B._HOST, None):
        monkeypatch.setattr(B, "_HOST", host)
        with pytest.raises(vp.VPError, match="gate must be"):
            vp.vp_block_norm_fwd(x, y, H, gate=gate)
        with pytest.raises(vp.VPError, match="gate must be"):
            vp.vp_block_norm_bwd(x, x, y, stats, dx=dx, dy=dy, gate=gate, workspace=ws)
        with pytest.raises(vp.VPError, match="gate must be"):
            vp.BlockNormPlan(x, y, gate=gate).forward()
    torch.cuda.synchronize()
    assert all(bool((t == 7).all()) for t in (H, dx, dy))


@pytest.mark.parametrize("N,large", [(N, at) for N in (96, 128, 256) for at in (0, 1, 37)])
def test_sums_over_few_tokens_lose_little(N, large):
    """Up to 256 tokens of 256 columns: at most 7 additions in a row for the tokens of a slice (256 / 32 of them), then 5 levels of a
    tree over 32 slices, so 12 roundings relative to the sum of absolute values.  Slices of N / 32 beside a value of which that is
    half a step are lost one by one where they are added to it in a row."""
    import paper_2411_05288_amd as vp
    h = 256
    dH = torch.ones(N, h, device="cuda")
    value = 2.0 ** (26 if N <= 128 else 27)
    dH[large] = value
    x, stats = torch.full((N, h), 0.5, device="cuda"), torch.ones(4, N, device="cuda")
    stats[2] = 0.0      # rh = x
    ws = torch.full((vp.vp_block_norm_bwd_workspace_bytes(N, h),), 0xFF, dtype=torch.uint8, device="cuda")
    dw, db, dx = torch.empty(h, device="cuda"), torch.empty(h, device="cuda"), torch.empty_like(x)
    vp.vp_block_norm_bwd(dH, x, None, stats, dx=dx, dw=dw, db=db, workspace=ws)
    for got, exact in ((db, value + N - 1), (dw, (value + N - 1) / 2)):
        off = float((got.double() - exact).abs().max())
        assert off <= 12 * ref.U * exact, off
