"""The norm of many gradients together and clipping by it (vp_grad_norm, vp_grad_clip, vp_grad_scale) against sums in 64 bits."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
HALF = {F32: 2.0 ** -24, BF16: 2.0 ** -8}


def lists():
    """(name, [(elements, type, elements that it starts behind an aligned address)])"""
    chunk = 32768
    yield "none", []
    yield "one", [(1, F32, 0)]
    yield "empty tensors", [(0, F32, 0), (0, BF16, 0)]
    yield "empty ones between", [(0, F32, 0), (5, F32, 0), (0, BF16, 0), (0, F32, 0), (9, BF16, 0), (0, F32, 0)]
    yield "odd starts", [(n, t, k) for n in (1, 3, 4, 8, 17, 1000, 8192, 20011) for t in (F32, BF16) for k in (1, 2, 3)]
    yield "around a chunk", [(chunk // s + d, t, 0) for t, s in ((F32, 4), (BF16, 2)) for d in (-9, -8, -4, -1, 0, 1, 7, 8)]
    yield "as many as the arguments hold", [(k % 37 + 1, (F32, BF16)[k % 2], 0) for k in range(120)]
    yield "one more", [(k % 37 + 1, (F32, BF16)[k % 2], k % 3) for k in range(121)]
    yield "many", [(k * k % 4001, (F32, BF16)[k % 3 == 0], k % 2) for k in range(700)]
    yield "more chunks than workgroups", [(20000003, F32, 0), (7, BF16, 1), (30000001, BF16, 3)]


def make(spec, seed=0, std=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    out = []
    for n, t, k in spec:
        whole = torch.full((n + k + 64,), 7.0, dtype=t, device="cuda")
        whole[k:k + n] = (torch.randn(n, generator=g, device="cuda") * std).to(t)
        out.append((whole, whole[k:k + n]))
    return out


def exact_norm(grads):
    return math.sqrt(math.fsum(float(g.double().square().sum()) for g in grads))


def check_clipped(got, grad, factor):
    # norm to half a step, the quotient, the product: three roundings to 32 bits, and the last one to the type
    value = grad.double() * factor
    bound = value.abs() * (4 * 2.0 ** -24 + (HALF[grad.dtype] if grad.dtype == BF16 else 0)) + 1e-44 + (5e-41 if grad.dtype == BF16 else 0)
    assert bool(((got.double() - value).abs() <= bound).all())


@pytest.mark.parametrize("name,spec", list(lists()), ids=[n for n, _ in lists()])
@pytest.mark.parametrize("max_norm", [0.25, 1e9, 0.0])
def test_norm_clip_and_scale(name, spec, max_norm):
    import paper_2411_05288_amd as vp
    both = make(spec, seed=len(spec))
    grads = [g for _, g in both]
    before = [g.clone() for g in grads]
    expected = exact_norm(grads)
    norm = torch.full((1,), 7.0, device="cuda")
    ws = torch.full((vp.vp_grad_workspace_bytes(len(grads)),), 0xFF, dtype=torch.uint8, device="cuda")
    vp.vp_grad_norm(grads, norm, ws)
    # the sum in 64 bits, its root rounded to 32
    assert abs(float(norm) - expected) <= expected * (2.0 ** -24 + 1e-12)
    first = norm.clone()
    factor = max_norm / expected if expected > max_norm else 1.0
    # into other tensors
    outs = make(spec, seed=99)
    ws.fill_(0xFF)
    norm.fill_(7.0)
    vp.vp_grad_clip(grads, max_norm, norm, ws, outs=[o for _, o in outs])
    assert torch.equal(norm, first)
    for (whole, o), (n, t, k), g, b in zip(outs, spec, grads, before):
        assert torch.equal(g, b)
        check_clipped(o, g, factor)
        assert bool((whole[:k] == 7).all()) and bool((whole[k + n:] == 7).all())
    # in place, and by a norm that is known
    for known in (False, True):
        here = make(spec, seed=len(spec))
        if known:
            vp.vp_grad_scale([g for _, g in here], max_norm, norm, ws)
        else:
            vp.vp_grad_clip([g for _, g in here], max_norm, norm, ws)
        assert torch.equal(norm, first)
        for (whole, g), (_, o), (n, t, k) in zip(here, outs, spec):
            assert torch.equal(g, o)
            assert bool((whole[:k] == 7).all()) and bool((whole[k + n:] == 7).all())


def test_repeated_and_in_another_order():
    """The norm does not depend on how often it is taken, and the tensors' order changes it by a rounding at most."""
    import paper_2411_05288_amd as vp
    grads = [g for _, g in make([(50000, F32, 0), (70001, BF16, 1), (3, F32, 2)], seed=5)]
    ws = torch.empty(vp.vp_grad_workspace_bytes(3), dtype=torch.uint8, device="cuda")
    norms = []
    for order in (grads, grads, grads[::-1]):
        norm = torch.empty(1, device="cuda")
        vp.vp_grad_norm(order, norm, ws)
        norms.append(norm)
    assert torch.equal(norms[0], norms[1])
    assert abs(float(norms[0]) - float(norms[2])) <= 2.0 ** -23 * float(norms[0])


@pytest.mark.parametrize("value", [1e-30, 1e30, 3e38])
def test_squares_beyond_the_range_of_32_bits(value):
    import paper_2411_05288_amd as vp
    n = 1000
    g = torch.full((n,), value, device="cuda")
    norm, ws = torch.empty(1, device="cuda"), torch.empty(vp.vp_grad_workspace_bytes(1), dtype=torch.uint8, device="cuda")
    vp.vp_grad_clip([g], 1.0, norm, ws)
    expected = float(torch.tensor(value)) * math.sqrt(n)
    if expected > 3.4028235e38:      # the norm is beyond 32 bits: it says so, and the gradients stay
        assert math.isinf(float(norm)) and bool((g == value).all())
    else:
        assert abs(float(norm) - expected) <= 2.0 ** -23 * expected
        assert bool(torch.isfinite(g).all()) and abs(float(g[0]) - min(float(torch.tensor(value)), 1 / math.sqrt(n))) <= 1e-6 / math.sqrt(n)


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("where", [0, 12345, 39999])
def test_a_norm_that_is_not_finite_leaves_the_gradients(bad, where):
    import paper_2411_05288_amd as vp
    for dtype in (F32, BF16):
        grads = [torch.randn(40000, device="cuda").to(dtype), torch.randn(33, device="cuda")]
        grads[0][where] = bad
        before = [g.clone() for g in grads]
        outs = [torch.empty_like(g) for g in grads]
        plan, copy = vp.GradientClipPlan(grads), vp.GradientClipPlan(grads, outs)
        plan.clip(1.0)
        copy.clip(1.0)
        assert not math.isfinite(float(plan.norm)) and (math.isnan(bad) == math.isnan(float(plan.norm)))
        for g, b, o in zip(grads, before, outs):
            assert torch.equal(g.view(torch.int16 if g.dtype == BF16 else torch.int32), b.view(torch.int16 if g.dtype == BF16 else torch.int32))
            assert torch.equal(torch.isnan(o), torch.isnan(b)) and torch.equal(o[~torch.isnan(o)], b[~torch.isnan(b)])


def test_plan_on_another_stream_and_in_a_graph():
    import paper_2411_05288_amd as vp
    spec = [(k * 977 % 50021, (F32, BF16)[k % 2], k % 2) for k in range(150)]
    grads, outs = [g for _, g in make(spec, seed=1)], [o for _, o in make(spec, seed=2)]
    plan = vp.GradientClipPlan(grads, outs)
    plan.clip(0.5)
    torch.cuda.synchronize()
    expected, norm = [o.clone() for o in outs], plan.norm.clone()
    side = torch.cuda.Stream()

    def clear():
        for o in outs:
            o.fill_(9.0)
        plan.norm.fill_(9.0)
        plan.workspace.fill_(0xFF)
        torch.cuda.synchronize()
    clear()
    plan.clip(0.5, stream=side)
    side.synchronize()
    assert torch.equal(plan.norm, norm) and all(torch.equal(a, b) for a, b in zip(outs, expected))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        plan.clip(0.5)
    # the calls' host arrays are gone from the plan when the graph is replayed
    plan.arguments.ptrs = plan.arguments.counts = plan.arguments.out_ptrs = None
    for _ in range(3):
        clear()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(plan.norm, norm) and all(torch.equal(a, b) for a, b in zip(outs, expected))
        assert float(torch.arange(1000, device="cuda", dtype=torch.float32).sum()) == 499500.0


def test_shared_memory_is_refused():
    import paper_2411_05288_amd as vp
    whole = torch.randn(1000, device="cuda")
    norm, ws = torch.empty(1, device="cuda"), torch.empty(vp.vp_grad_workspace_bytes(8), dtype=torch.uint8, device="cuda")
    before = whole.clone()
    a, b = whole[:600], whole[500:]
    for grads, outs in (([whole, whole], None), ([a, b], None), ([whole[:10], whole[20:30]], [whole[40:50], whole[45:55]]),
                        ([whole[:10], whole[20:30]], [whole[40:50], whole[5:15]]), ([whole[:10]], [whole[1:11]]),
                        ([whole[:10], whole[20:30]], [whole[20:30], whole[:10]])):
        with pytest.raises(vp.VPError, match="shares memory"):
            vp.vp_grad_clip(grads, 0.1, norm, ws, outs=outs)
    torch.cuda.synchronize()
    assert torch.equal(whole, before)
    vp.vp_grad_norm([whole, whole], norm, ws)      # reading a tensor twice is no conflict
    assert abs(float(norm) - math.sqrt(2) * float(whole.double().norm())) <= 1e-6 * float(norm)
    vp.vp_grad_clip([whole[:10], whole[20:30]], 0.1, norm, ws, outs=[whole[:10], whole[20:30]])      # in place by outs


def test_training_step_from_norm_to_clipping():
    """The last block's norms, the sharded output layer, their gradients, the input layer's, and clipping over all of them."""
    import norm_reference as ref
    import paper_2411_05288_amd as vp
    N, h, V, p = 96, 256, 1000, 4
    g = torch.Generator(device="cuda").manual_seed(3)

    def normal(*shape, std=1.0, mean=0.0):
        return torch.randn(*shape, generator=g, device="cuda") * std + mean
    x, y, w, wp = normal(N, h), normal(N, h), normal(h, std=0.1, mean=1.0), normal(h, std=0.1, mean=1.0)
    Ws = [normal(V // p, h, std=0.05) for _ in range(p)]
    ids = torch.randint(0, V, (N,), generator=g, device="cuda")
    labels = torch.randint(0, V, (N,), generator=g, device="cuda")
    norm = vp.BlockNormPlan(x, y, w=w, w_post=wp, post=True)
    plan = vp.OutputLayerPlan(None, Ws, labels, norm=norm)
    plan.step()
    embed = vp.EmbeddingPlan([torch.zeros(V // p, h, device="cuda") for _ in range(p)], ids, norm.dx)
    embed.backward()
    # the same in 64 bits, by automatic differentiation of the formulas
    leaves = [t.double().requires_grad_() for t in (x, y, w, wp)] + [W.double().requires_grad_() for W in Ws]
    X, Y, W1, WP = leaves[:4]

    def rms(v):
        return v / (v.square().mean(1, keepdim=True) + norm.eps).sqrt()
    logits = rms(X + rms(Y) * WP) * W1 @ torch.cat(leaves[4:]).t()
    loss = (torch.logsumexp(logits, 1) - logits.gather(1, labels[:, None])[:, 0]).mean()
    loss.backward()
    table = torch.zeros(V, h, device="cuda", dtype=torch.float64).index_add_(0, ids, X.grad)
    # the products of the fp32 path keep 1e-5 of a tensor's largest element, and so does what is made of them
    assert abs(float(plan.loss) - float(loss.detach())) <= 1e-5 * float(loss.detach())
    grads = [*plan.dW, norm.dw, norm.dw_post, *embed.dtable]
    expected = [*[t.grad for t in leaves[4:]], W1.grad, WP.grad, *table.split(V // p)]
    for name, got, value in [("dx", norm.dx, X.grad), ("dy", norm.dy, Y.grad)] + [(str(k), a, b) for k, (a, b) in enumerate(zip(grads, expected))]:
        assert float((got.double() - value).abs().max()) <= 2e-5 * float(value.abs().max()), name
    before = [t.clone() for t in grads]
    total = exact_norm(before)
    got = plan.clip_gradients(total / 3, embed.dtable)
    assert abs(float(got) - total) <= 2.0 ** -23 * total
    for a, b in zip(grads, before):
        check_clipped(a, b, 1 / 3)
    plan.step()      # the next step writes the same gradients again, and the same plan clips them
    first = plan.clip_plan
    embed.dtable[0].mul_(3.0)
    plan.clip_gradients(total / 3, embed.dtable)
    assert plan.clip_plan is first


def test_a_tensor_of_more_than_32_bits_of_bytes():
    import paper_2411_05288_amd as vp
    n = (1 << 30) + 5000
    big, small = torch.full((n,), 0.5, device="cuda"), torch.full((3,), 2.0, device="cuda")
    big[-1], big[1 << 30] = 3.0, -4.0
    norm, ws = torch.empty(1, device="cuda"), torch.empty(vp.vp_grad_workspace_bytes(2), dtype=torch.uint8, device="cuda")
    vp.vp_grad_clip([big, small], 1.0, norm, ws)
    expected = math.sqrt((n - 2) * 0.25 + 9 + 16 + 12)
    assert abs(float(norm) - expected) <= 2.0 ** -23 * expected
    f = 1 / expected
    for at, value in ((0, 0.5), (12345678, 0.5), (1 << 30, -4.0), (n - 2, 0.5), (n - 1, 3.0)):
        assert abs(float(big[at]) - value * f) <= 4 * 2.0 ** -24 * abs(value * f)
    assert int((big != big[0]).sum()) == 2 and abs(float(small[2]) - 2 * f) <= 8 * 2.0 ** -24 * f


@pytest.mark.parametrize("algorithm", [1, 2])
def test_step_with_norm_and_clipping_in_a_graph(algorithm):
    """bf16, layer norms with a gate per sequence: the whole step and the clipping, eager and replayed, bit for bit."""
    import paper_2411_05288_amd as vp
    N, h, V, p = 240, 512, 1536, 3
    g = torch.Generator(device="cuda").manual_seed(4)

    def normal(*shape, std=1.0, mean=0.0):
        return (torch.randn(*shape, generator=g, device="cuda") * std + mean).bfloat16()
    norm = vp.BlockNormPlan(normal(N, h), normal(N, h), gate=normal(4, h), w=normal(h, mean=1.0, std=0.1), b=normal(h), post=True,
                            w_post=normal(h, mean=1.0, std=0.1), b_post=normal(h), center=True, scale=0.5)
    labels = torch.randint(0, V, (N,), generator=g, device="cuda")
    plan = vp.OutputLayerPlan(None, [normal(V // p, h, std=0.05) for _ in range(p)], labels, norm=norm, algorithm=algorithm)
    other = normal(1001)
    kept = other.clone()

    def step():
        other.copy_(kept)
        plan.step()
        return plan.clip_gradients(0.01, [other])
    total = step()
    torch.cuda.synchronize()
    outs = [plan.loss, norm.H, norm.r, norm.dx, norm.dy, total, other, *norm.parameter_gradients(), *plan.dW]
    expected = [t.clone() for t in outs]
    assert float(total) > 0.01 and all(bool(torch.isfinite(t).all()) for t in outs)
    clipped = exact_norm([other, *norm.parameter_gradients(), *plan.dW])
    assert abs(clipped - 0.01) <= 0.01 * 2.0 ** -8      # (the bf16 one rounds its elements by half a step at most)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(3):
        for t in outs + [plan.workspace, norm.workspace, plan.clip_plan.workspace]:
            t.fill_(float("nan") if t.is_floating_point() else 0xFF)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, expected))
        assert float(torch.arange(1000, device="cuda", dtype=torch.float32).sum()) == 499500.0


def test_plan_scales_by_a_norm_over_several_devices():
    """What a program with its gradients on several devices does: norms joined outside, every device scales by the whole."""
    import paper_2411_05288_amd as vp
    parts = [[g for _, g in make([(5000, F32, 0), (333, BF16, 1)], seed=s)] for s in (1, 2)]
    before = [[g.clone() for g in part] for part in parts]
    plans = [vp.GradientClipPlan(part) for part in parts]
    for plan in plans:
        plan.compute_norm()
    whole = torch.stack([plan.norm.double() ** 2 for plan in plans]).sum(0).sqrt().float()
    expected = exact_norm([g for part in before for g in part])
    assert abs(float(whole) - expected) <= 2.0 ** -22 * expected
    for plan in plans:
        plan.scale(2.0, whole)
    for part, old in zip(parts, before):
        for g, b in zip(part, old):      # the joined norm has two roundings more
            value = b.double() * (2.0 / expected)
            assert bool(((g.double() - value).abs() <= value.abs() * (8 * 2.0 ** -24 + (HALF[BF16] if g.dtype == BF16 else 0))).all())
    plans[0].compute_norm()
    mine = float(plans[0].norm)
    plans[0].scale(mine / 4)
    assert abs(exact_norm(parts[0]) - mine / 4) <= mine * 2.0 ** -8


def test_plan_notices_gradients_that_moved():
    import paper_2411_05288_amd as vp
    W = [torch.randn(64, 32, device="cuda")]
    plan = vp.OutputLayerPlan(torch.randn(16, 32, device="cuda"), W, torch.zeros(16, dtype=torch.int64, device="cuda"))
    plan.step()
    other = torch.randn(100, device="cuda")
    plan.clip_gradients(1e-3, [other])
    first = plan.clip_plan
    plan.clip_gradients(1e-3, [other])
    assert plan.clip_plan is first
    other.data = torch.randn(100, device="cuda")      # the same tensor, other memory
    total = plan.clip_gradients(1e-4, [other])
    assert plan.clip_plan is not first and float(total) > 1
    assert abs(exact_norm([other, *plan.dW]) - 1e-4) <= 1e-9


def test_evaluation_with_a_norm_that_keeps_nothing():
    import paper_2411_05288_amd as vp
    N, h, V = 5, 256, 640
    x, y = torch.randn(N, h, device="cuda").bfloat16(), torch.randn(N, h, device="cuda").bfloat16()
    W = [torch.randn(V // 2, h, device="cuda").bfloat16() for _ in range(2)]
    labels = torch.arange(N, device="cuda")
    losses = []
    for train in (True, False):
        norm = vp.BlockNormPlan(x, y, post=True, train=train)
        plan = vp.OutputLayerPlan(None, W, labels, save_logits=False, norm=norm)
        plan.forward()
        losses.append(plan.loss.clone())
    assert torch.equal(*losses) and norm.stats is None
    with pytest.raises(vp.VPError, match="train=False"):
        plan.backward()


def test_a_captured_clipping_outlives_calls_with_other_gradients():
    import paper_2411_05288_amd as vp
    g = torch.Generator(device="cuda").manual_seed(6)
    plan = vp.OutputLayerPlan(torch.randn(16, 32, generator=g, device="cuda"), [torch.randn(64, 32, generator=g, device="cuda")],
                              torch.zeros(16, dtype=torch.int64, device="cuda"))
    few = [torch.randn(100, generator=g, device="cuda") for _ in range(3)]
    many = [torch.randn(50, generator=g, device="cuda") for _ in range(200)]
    kept = [t.clone() for t in few]

    def step():
        for t, k in zip(few, kept):
            t.copy_(k)
        plan.step()
        return plan.clip_gradients(0.1, few)
    total = step().clone()
    expected = [t.clone() for t in few + plan.dW]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(3):
        other = plan.clip_gradients(1e9, many)      # a larger list, another plan and workspace
        assert float(other) > float(total)
        junk = [torch.full((1 << 14,), float("nan"), device="cuda") for _ in range(20)]      # what was freed is written by others
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(plan.clip_norm, total)
        assert all(torch.equal(a, b) for a, b in zip(few + plan.dW, expected))
        assert all(bool(torch.isnan(t).all()) for t in junk)


def test_plan_notices_gradients_that_changed_where_they_are():
    """A shorter view or another type at the same address: what lies behind is not touched, and the list is made anew."""
    import paper_2411_05288_amd as vp
    plan = vp.OutputLayerPlan(torch.randn(16, 32, device="cuda"), [torch.randn(64, 32, device="cuda")],
                              torch.zeros(16, dtype=torch.int64, device="cuda"))
    plan.step()
    whole = torch.full((400,), 3.0, device="cuda")
    other = whole[:300]
    kept = vp.GradientClipPlan([other])
    plan.clip_gradients(1e6, [other])
    first = plan.clip_plan
    other.data = other.data[:100]
    total = plan.clip_gradients(1e-3, [other])
    assert plan.clip_plan is not first and abs(exact_norm([other, *plan.dW]) - 1e-3) <= 1e-8 and float(total) > 30
    assert bool((whole[100:] == 3).all())
    other.data = other.data.view(BF16)[:100]
    with pytest.raises(vp.VPError, match="since the arguments were made"):
        kept.clip(1e-3)
    with pytest.raises(vp.VPError, match="since the arguments were made"):
        kept.compute_norm()
    other.fill_(2.0)
    total = plan.clip_gradients(1.0, [other])
    assert plan.clip_plan.arguments.dts[-1] == vp.VP_BF16 and abs(float(total) - 20) <= 1e-4      # 10 * 2 and what is left of dW
    assert bool((whole[100:] == 3).all())


def long_lists():
    """(name, numbers of elements) around the 160 tensors that the kernel arguments hold, full batches of a table, and the 2048 of
    whose first chunks a workgroup holds every one (above that every second, every third)."""
    for n in (159, 160, 161, 319, 320, 321, 480, 481):
        yield "%d" % n, [k * 13 % 61 for k in range(n)]
    for n in (2047, 2048, 2049, 4096, 4097, 5000):
        yield "%d" % n, [k * 29 % 97 for k in range(n)]
    # tensors without elements where every second one is looked up, at the ends of what lies between, and at both ends of the list
    yield "empty ones that are looked up", [0 if k % 2 == 0 else k % 50 + 1 for k in range(4000)]
    yield "empty ones between", [0 if k % 2 else k % 50 + 1 for k in range(4000)]
    yield "empty runs", [0 if k // 5 % 3 else k % 50 + 1 for k in range(5001)]
    yield "empty ends", [0] * 1000 + [7] * 2000 + [0] * 1000
    yield "one of many", [0] * 3000 + [33] + [0] * 1999
    yield "none of many", [0] * 2500
    # tensors of several chunks among small ones
    yield "large ones between", [30011 if k % 500 == 17 else k % 9 for k in range(4500)]


@pytest.mark.parametrize("name,counts", list(long_lists()), ids=[n for n, _ in long_lists()])
@pytest.mark.parametrize("mixed", [False, True])
def test_long_lists(name, counts, mixed):
    """Views of one buffer per type, in place and into the views of another; every element of the buffers is looked at, those between
    the tensors too."""
    import paper_2411_05288_amd as vp
    types = [BF16 if mixed and k % 3 == 1 else F32 for k in range(len(counts))]
    gap = 3      # elements between two tensors
    size = {t: sum(n + gap for n, u in zip(counts, types) if u == t) + gap for t in (F32, BF16)}
    g = torch.Generator(device="cuda").manual_seed(len(counts))
    whole = {t: torch.randn(n, generator=g, device="cuda").to(t) for t, n in size.items()}
    inside = {t: torch.zeros(n, dtype=torch.bool) for t, n in size.items()}
    at, spans = dict.fromkeys(size, gap), []
    for n, t in zip(counts, types):
        spans.append((t, at[t], n))
        inside[t][at[t]:at[t] + n] = True
        at[t] += n + gap
    inside = {t: m.cuda() for t, m in inside.items()}

    def views(buffers):
        return [buffers[t][a:a + n] for t, a, n in spans]
    expected = math.sqrt(math.fsum(float(whole[t].double()[inside[t]].square().sum()) for t in whole))
    most = expected / 3 if expected else 1.0
    norm, ws = torch.full((1,), 7.0, device="cuda"), torch.full((vp.vp_grad_workspace_bytes(len(counts)),), 0xFF, dtype=torch.uint8, device="cuda")
    vp.vp_grad_norm(views(whole), norm, ws)
    assert abs(float(norm) - expected) <= expected * (2.0 ** -24 + 1e-12)
    outs, here, known = ({t: b.clone() for t, b in whole.items()} for _ in range(3))
    for buffers, call in ((outs, lambda b: vp.vp_grad_clip(views(whole), most, norm, ws, outs=views(b))),
                          (here, lambda b: vp.vp_grad_clip(views(b), most, norm, ws)),
                          (known, lambda b: vp.vp_grad_scale(views(b), most, norm, ws))):
        ws.fill_(0xFF)
        call(buffers)
        for t, b in buffers.items():
            assert torch.equal(b[~inside[t]], whole[t][~inside[t]])
            if expected:
                check_clipped(b[inside[t]], whole[t][inside[t]], 1 / 3)


@pytest.mark.parametrize("as_number", [False, True])
def test_clipping_on_another_stream_takes_its_memory_there(as_number):
    """What a call on a stream allocates belongs to that stream: memory freed by work that is still running on the current one may
    not be written from another."""
    import paper_2411_05288_amd as vp
    plan = vp.OutputLayerPlan(torch.randn(16, 32, device="cuda"), [torch.randn(64, 32, device="cuda")],
                              torch.zeros(16, dtype=torch.int64, device="cuda"))
    plan.step()
    torch.cuda.synchronize()
    before = [t.clone() for t in plan.dW]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    total = plan.clip_gradients(1e-3, stream=side.cuda_stream if as_number else side)
    side.synchronize()
    expected = exact_norm(before)
    assert abs(float(total) - expected) <= 2.0 ** -23 * expected
    check_clipped(plan.dW[0], before[0], 1e-3 / expected)
    for t in (plan.clip_norm, plan.clip_workspaces[-1]):
        (segment,) = [s for s in torch.cuda.memory_snapshot() if s["address"] <= t.data_ptr() < s["address"] + s["total_size"]]
        assert segment["stream"] == side.cuda_stream
