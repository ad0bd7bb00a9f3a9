"""The operators that answer, together as they are used: a norm, hidden states and weights in 8-bit integers, logits and statistics of
the shards, drafted tokens verified against them."""
import numpy as np
import pytest
import torch

import answer_reference as ref

pytestmark = pytest.mark.gpu


def weights(rows, h, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return [(torch.randn(n, h, generator=gen, device="cuda") * 0.05).to(torch.bfloat16) for n in rows]


class Model:
    """The end of a model: a norm and the output layer in integers."""

    def __init__(self, N, h, rows, seed, vocab_size=None, logits_dtype=None, labels=None):
        import paper_2411_05288_amd as vp
        self.x = torch.randn(N, h, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda").to(torch.bfloat16)
        self.W = weights(rows, h, seed + 1)
        self.norm = vp.BlockNormPlan(self.x, w=torch.ones(h, dtype=torch.bfloat16, device="cuda"), train=False)
        self.plan = vp.OutputLayerI8Plan(None, [vp.quantize_rows(w) for w in self.W], labels, norm=self.norm,
                                         vocab_size=vocab_size, logits_dtype=logits_dtype)

    def reference(self):
        """Logits and statistics in 64 bits of the plan's own normed states."""
        qH, sH = ref.quantize_rows_fast(self.norm.H.double().cpu().numpy())
        V = self.plan.vocab_size
        qW, sW = ref.quantize_rows_fast(torch.cat(self.W)[:V].double().cpu().numpy())
        Y = ref.logits(qH, sH, qW, sW)
        return Y, Y.max(1), np.exp(Y - Y.max(1, keepdims=True)).sum(1)


def inputs(counts, V, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    starts = torch.tensor(np.concatenate([[0], np.cumsum([c + 1 for c in counts])]), device="cuda")
    N = int(starts[-1])
    return starts, torch.randint(0, V, (N,), generator=gen, device="cuda"), torch.rand(N, generator=gen, device="cuda")


def check(verify, order):
    """The verification against the definition, on the logits and statistics that the plans left."""
    host = lambda t: None if t is None else t.cpu().numpy()      # noqa: E731
    joined = lambda ts: None if ts is None else torch.cat([t.double() for t in ts], 1).cpu().numpy()      # noqa: E731
    t, d = verify.target, verify.draft
    a, tokens, margins = ref.verify(joined(verify.logits), host(t.global_max), host(t.global_sumexp), host(verify.drafts),
                                    host(verify.starts), host(verify.uniforms), np.full(t.N, -5), order, joined(verify.draft_logits),
                                    None if d is None else host(d.global_max), None if d is None else host(d.global_sumexp))
    assert (margins > 1e-12).all()
    np.testing.assert_array_equal(host(verify.accepted), a)
    np.testing.assert_array_equal(host(verify.tokens), tokens)


@pytest.mark.parametrize("logits_dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,vocab_size", [([300, 300, 300], 900), ([300, 300, 300], 501), ([300, 300, 300], 300), ([700], 650)])
def test_a_step_of_an_answer(rows, vocab_size, logits_dtype):
    import paper_2411_05288_amd as vp
    counts = [3, 0, 5, 1]
    N, h = sum(counts) + len(counts), 200
    labels = torch.randint(0, vocab_size, (N,), generator=torch.Generator(device="cuda").manual_seed(1), device="cuda")
    target, draft = (Model(N, h, rows, s, vocab_size, logits_dtype, labels) for s in (1, 5))
    starts, _, uniforms = inputs(counts, vocab_size, 3)
    draft.plan.forward()
    drafts = torch.cat(draft.plan.logits, 1).float().argmax(1)
    verify = vp.DraftVerifyPlan(target.plan, starts, drafts, uniforms, draft=draft.plan)
    target.plan.forward()
    verify.forward()
    torch.cuda.synchronize()
    check(verify, np.arange(vocab_size))
    for model in (target, draft):
        Y, m, s = model.reference()
        p = model.plan
        A = np.abs(Y).max()
        # (bounds of the logits, the statistics of a shard and their sum as in the tests of the product)
        assert np.abs(p.global_max.cpu().numpy() - m).max() <= 4 * 2.0 ** -24 * A
        loss = np.log(s) + m - Y[np.arange(N), labels.cpu().numpy()]
        tol = 2.0 ** -24 * (48 * A + 400)
        assert np.abs(p.loss_rows.cpu().numpy() - loss).max() <= tol + 2.0 ** -22 * np.abs(loss).max()
        assert abs(p.loss.item() - loss.mean()) <= tol + 2.0 ** -21 * np.abs(loss).max()


def test_a_plan_without_labels_and_one_token():
    import paper_2411_05288_amd as vp
    W = [vp.quantize_rows(w) for w in weights([500, 400], 129, 3)]
    H = torch.randn(1, 129, generator=torch.Generator(device="cuda").manual_seed(2), device="cuda")
    plan = vp.OutputLayerI8Plan(H, W)
    assert plan.logits[0].dtype == torch.float32
    starts, drafts, uniforms = inputs([0], 900, 1)
    verify = vp.DraftVerifyPlan(plan, starts, drafts, uniforms)
    plan.forward()
    verify.forward()
    torch.cuda.synchronize()
    check(verify, np.arange(900))


@pytest.mark.parametrize("algorithm", [1, 2])
def test_verification_over_the_trained_layers_logits(algorithm):
    """The logits and statistics of OutputLayerPlan, with shards of padding behind the vocabulary."""
    import paper_2411_05288_amd as vp
    counts, rows, h, V = [2, 4, 0, 3], [128, 128, 128, 128], 64, 300
    N = sum(counts) + len(counts)
    gen = torch.Generator(device="cuda").manual_seed(4)
    plans = []
    for seed in (1, 2):
        H = torch.randn(N, h, generator=gen, device="cuda").to(torch.bfloat16)
        plans.append(vp.OutputLayerPlan(H, weights(rows, h, seed), torch.zeros(N, dtype=torch.int64, device="cuda"), vocab_size=V,
                                        algorithm=algorithm))
        plans[-1].forward()
    starts, drafts, uniforms = inputs(counts, V, 9)
    verify = vp.DraftVerifyPlan(plans[0], starts, drafts, uniforms, draft=plans[1])
    verify.forward()
    torch.cuda.synchronize()
    check(verify, np.arange(V))


def test_refusals_of_the_plans():
    import paper_2411_05288_amd as vp
    W = [vp.quantize_rows(w) for w in weights([64, 64], 100, 1)]
    H = torch.zeros(3, 100, device="cuda")
    starts, drafts, uniforms = inputs([2], 128, 1)
    for bad in (dict(H=None), dict(H=torch.zeros(100, device="cuda")), dict(H=torch.zeros(3, 200, device="cuda")), dict(vocab_size=0),
                dict(vocab_size=129), dict(W_shards=[(W[0][0], W[1][1][:5])]), dict(W_shards=[(W[0][0].view(-1), W[0][1])])):
        with pytest.raises(vp.VPError):
            vp.OutputLayerI8Plan(**{**dict(H=H, W_shards=W), **bad})
    alone, plan = vp.OutputLayerI8Plan(H, W, save_logits=False), vp.OutputLayerI8Plan(H, W)
    other = vp.OutputLayerI8Plan(H, W[:1])
    for a, k in (((alone,), {}), ((plan,), dict(draft=alone)), ((plan,), dict(draft=other))):
        with pytest.raises(vp.VPError):
            vp.DraftVerifyPlan(*a, starts, drafts, uniforms, **k)
    for wrong in (starts[0], starts[:1], starts[:0]):
        with pytest.raises(vp.VPError):
            vp.DraftVerifyPlan(plan, wrong, drafts, uniforms)
    with pytest.raises(vp.VPError):
        vp.quantize_rows(torch.zeros(4, device="cuda"))
    assert vp.OutputLayerI8Plan(H, iter(W)).vocab_size == 128


def step_of(target, draft, verify):
    draft.plan.forward()
    target.plan.forward()
    verify.forward()


def test_a_step_in_a_graph_and_on_another_stream():
    """Captured once and replayed with other inputs in the same buffers, with the program's own work in between; two graphs of two
    plans replayed in turn; the same through a stream argument."""
    import paper_2411_05288_amd as vp
    counts, rows, h = [3, 0, 5, 1, 2], [300, 400], 256
    N = sum(counts) + len(counts)
    runs = []
    for seed in (1, 20):
        target, draft = Model(N, h, rows, seed), Model(N, h, rows, seed + 5)
        starts, drafts, uniforms = inputs(counts, 700, seed)
        verify = vp.DraftVerifyPlan(target.plan, starts, drafts, uniforms, draft=draft.plan)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step_of(target, draft, verify)
        torch.cuda.current_stream().wait_stream(side)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step_of(target, draft, verify)
        runs.append((target, draft, verify, graph))
    gen = torch.Generator(device="cuda").manual_seed(99)
    for turn in range(4):
        want = []
        for target, draft, verify, graph in runs:
            target.x.copy_(torch.randn(N, h, generator=gen, device="cuda"))
            draft.x.copy_(target.x.float() + 0.3 * torch.randn(N, h, generator=gen, device="cuda"))
            verify.uniforms.copy_(torch.rand(N, generator=gen, device="cuda"))
            verify.drafts.copy_(torch.randint(0, 700, (N,), generator=gen, device="cuda"))
            step_of(target, draft, verify)
            torch.cuda.synchronize()
            check(verify, np.arange(700))
            want.append([t.clone() for t in (verify.accepted, verify.tokens, target.plan.loss_rows, *target.plan.logits)])
            verify.tokens.fill_(-9)
            target.plan.workspace.fill_(0xFF)
            verify.workspace.fill_(0xFF)
        for _, _, _, graph in runs:
            graph.replay()
        torch.cuda.synchronize()
        assert float(torch.arange(1000, device="cuda", dtype=torch.float32).sum()) == 499500.0
        for (target, _, verify, _), w in zip(runs, want):
            for a, b in zip((verify.accepted, verify.tokens, target.plan.loss_rows, *target.plan.logits), w):
                assert torch.equal(a, b)
        stream = torch.cuda.Stream()
        stream.wait_stream(torch.cuda.current_stream())
        for argument in (stream, stream.cuda_stream):
            for (target, draft, verify, _), w in zip(runs, want):
                verify.tokens.fill_(-9)
                stream.wait_stream(torch.cuda.current_stream())
                for p in (draft.plan, target.plan, verify):
                    p.forward(argument)
                stream.synchronize()
                assert torch.equal(verify.tokens, w[1]) and torch.equal(verify.accepted, w[0])


def test_rows_become_integers_on_another_stream():
    import paper_2411_05288_amd as vp
    w = weights([700], 300, 1)[0]
    a = vp.quantize_rows(w)
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    b = vp.quantize_rows(w, stream)
    c = vp.quantize_rows(w, stream.cuda_stream)
    stream.synchronize()
    for t in (b, c):
        assert torch.equal(a[0], t[0]) and torch.equal(a[1], t[1])


def sum_bound(Y, m):
    """Bound of the relative error of fp32 sums of exp(y - m) over the rows of Y.  The difference d, its product with log2(e), that
    constant and the exponential are off by 2^-24 (half a step) of d, d, 0.23 d and 2 steps of the term: 2.3 d 2^-24 + 2^-22.  Sums: 16
    roundings one after the other at most, and the last one."""
    with np.errstate(invalid="ignore"):
        d = np.where(Y == -np.inf, 0.0, m[:, None] - Y)
        w = np.where(Y == -np.inf, 0.0, np.exp(Y - m[:, None]))
    return ((w * (2.3 * d + 4)).sum(1) / w.sum(1) + 17) * 2.0 ** -24


def check_normalised(verify):
    """What the verification calls probabilities are, as softmax of the logits that it reads: their sums are 1."""
    for side, logits in ((verify.target, verify.logits), (verify.draft, verify.draft_logits)):
        if side is not None:
            Y = torch.cat([y.double() for y in logits], 1).cpu().numpy()
            m, s = (t.double().cpu().numpy() for t in (side.global_max, side.global_sumexp))
            total = np.exp(Y - m[:, None]).sum(1) / s
            assert (np.abs(total - 1) <= 1.01 * sum_bound(Y, m)).all()


class Peaked:
    """A plan whose rows all are the same, with leading logits of this size."""

    def __init__(self, kind, N, rows, seed, size, dtype=torch.bfloat16):
        import paper_2411_05288_amd as vp
        h, W = 128, weights(rows, 128, seed)
        x = torch.randn(h, generator=torch.Generator(device="cuda").manual_seed(seed + 50), device="cuda")
        x = x * (size / (torch.cat(W).float() @ x).max())
        H = x.to(dtype).expand(N, h).contiguous()
        if kind == "i8":
            self.plan = vp.OutputLayerI8Plan(H, [vp.quantize_rows(w) for w in W])
        else:
            self.plan = vp.OutputLayerPlan(H, [w.to(dtype) for w in W], torch.zeros(N, dtype=torch.int64, device="cuda"), algorithm=kind)

    def probabilities(self):
        Y = torch.cat([y[0].double() for y in self.plan.logits]).cpu().numpy()
        return np.exp(Y - Y.max()) / np.exp(Y - Y.max()).sum()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("size", [3.0, 20.0, 40.0])
@pytest.mark.parametrize("kind", ["i8", 1, 2])
def test_statistics_are_those_of_the_kept_logits(kind, size, dtype):
    """The layers' own statistics are taken before the logits are rounded to bf16."""
    import paper_2411_05288_amd as vp
    counts, rows = [3, 0, 2, 8, 1], [200, 133, 300]
    starts, drafts, uniforms = inputs(counts, sum(rows), 5)
    target, draft = (Peaked(kind, int(starts[-1]), rows, s, size, dtype) for s in (1, 2))
    verify = vp.DraftVerifyPlan(target.plan, starts, drafts, uniforms, draft=draft.plan)
    for model in (draft, target):
        model.plan.forward()
    own = [(p.global_max.clone(), p.global_sumexp.clone(), p.loss_rows.clone()) for p in (target.plan, draft.plan)]
    verify.forward()
    check_normalised(verify)
    check(verify, np.arange(sum(rows)))
    for p, kept in zip((target.plan, draft.plan), own):      # (what a backward pass or the loss takes stays)
        assert all(torch.equal(a, b) for a, b in zip((p.global_max, p.global_sumexp, p.loss_rows), kept))


@pytest.mark.parametrize("model", [True, False])
@pytest.mark.parametrize("change", ["none", "mask", "mask_low", "temperature"])
@pytest.mark.parametrize("kind", ["i8", 1])
def test_tokens_follow_the_kept_logits(kind, change, model):
    """Whatever the drafts are, the first token of a sequence is distributed as softmax of the target's kept logits says, also where
    the program rules tokens out (with -inf, or a constant far below) or divides by a temperature.  Of S sequences a token's count
    is within 6 deviations and 12 of S p (Bernstein's inequality: below 2e-8 for a token; the seeds are fixed)."""
    import paper_2411_05288_amd as vp
    S, rows = 10000, [100, 57]
    V, N = sum(rows), 2 * S
    target, draft = (Peaked(kind, N, rows, s, 20.0) for s in (1, 2))
    rng = np.random.default_rng(7)
    for m in (target, draft):
        m.plan.forward()
    top = int(target.probabilities().argmax())
    for y, at in zip(target.plan.logits, target.plan.offsets):
        if change.startswith("mask"):
            out = [j - at for j in {top, *range(0, V, 3)} if 0 <= j - at < y.shape[1]]
            y[:, out] = -np.inf if change == "mask" else -1e30
        elif change == "temperature":
            y.div_(0.7)
    p, q = target.probabilities(), draft.probabilities()
    if model:
        drawn = rng.choice(V, N, p=q)
    else:
        drawn = np.full(N, int(p.argmax()))
    verify = vp.DraftVerifyPlan(target.plan, torch.arange(0, N + 1, 2, device="cuda"), torch.from_numpy(drawn).cuda(),
                                torch.from_numpy(rng.random(N).astype(np.float32)).cuda(), draft=draft.plan if model else None)
    verify.forward()
    torch.cuda.synchronize()
    check_normalised(verify)
    within = lambda n, S, p: (np.abs(n - S * p) <= 6 * np.sqrt(S * p * (1 - p)) + 12).all()      # noqa: E731
    first = np.bincount(verify.tokens[0::2].cpu().numpy(), minlength=V)
    assert within(first, S, p) and not first[p == 0].any()
    accepted = verify.accepted.cpu().numpy()
    assert within(accepted.sum(), S, np.minimum(p, q).sum() if model else p.max())
    behind = verify.tokens[1::2].cpu().numpy()[accepted == 1]
    assert within(np.bincount(behind, minlength=V), len(behind), p)
    assert (verify.tokens[1::2].cpu().numpy()[accepted == 0] == -1).all()


@pytest.mark.parametrize("dtype,h", [(torch.float32, 101), (torch.bfloat16, 101), (torch.bfloat16, 130)])
def test_rows_of_a_shard_cut_anywhere_become_integers(dtype, h):
    """Shards that are views of a whole matrix, of uneven sizes: they begin at any element."""
    import paper_2411_05288_amd as vp
    W = (torch.randn(501, h, generator=torch.Generator(device="cuda").manual_seed(3), device="cuda")).to(dtype)
    q, scales = vp.quantize_rows(W)
    stream = torch.cuda.Stream()
    for at in (1, 2, 3, 7, 167, 334):
        for argument in (None, stream):
            stream.wait_stream(torch.cuda.current_stream())
            a, b = vp.quantize_rows(W[at:], argument)
            torch.cuda.current_stream().wait_stream(stream)
            assert torch.equal(a, q[at:]) and torch.equal(b, scales[at:])
