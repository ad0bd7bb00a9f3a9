"""Verification of drafted tokens and the draw of the next one, against the definition in 64 bits."""
import math

import numpy as np
import pytest
import torch

import answer_reference as ref

pytestmark = pytest.mark.gpu
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
UNTOUCHED = -77


class Case:
    """Sequences with these numbers of drafts (None: a sequence without rows) over shards of these sizes."""

    def __init__(self, counts, rows, dtype="f32", model=True, seed=1, spread=2.0, behind=0, offsets=None, sure=0.6):
        rng = np.random.default_rng(seed)
        self.counts, self.rows, self.dtype = counts, rows, dtype
        self.starts = np.concatenate([[0], np.cumsum([0 if c is None else c + 1 for c in counts])]).astype(np.int64)
        N, V = int(self.starts[-1]) + behind, sum(rows)
        N = max(N, 1)
        self.N, self.V = N, V
        self.offsets = np.cumsum([0] + rows[:-1]).tolist() if offsets is None else offsets
        self.order = np.concatenate([np.arange(n) + at for n, at in zip(rows, self.offsets)])
        held = lambda a: torch.from_numpy(a).to(TYPES[dtype]).double().numpy()      # noqa: E731
        Y = rng.normal(0, spread, (N, V))
        Z = Y + rng.normal(0, 0.5, (N, V))
        self.Z = held(Z) if model else None
        # drafts: of the draft model, or tokens that the target gives about this probability
        drawn = (Z + rng.gumbel(size=(N, V))).argmax(1)
        if not model and sure is not None:
            others = np.log(np.exp(Y).sum(1) - np.exp(Y[np.arange(N), drawn]) + 1e-30)
            Y[np.arange(N), drawn] = others + math.log(sure / (1 - sure))
        self.Y = held(Y)
        self.drafts = self.order[drawn].astype(np.int64)
        self.uniforms = rng.random(N).astype(np.float32)
        self.tokens = np.full(N, UNTOUCHED, np.int64)
        self.stats()

    def stats(self):
        of = lambda Y: (None, None) if Y is None else self.stats_of(Y)      # noqa: E731
        (self.m, self.s), (self.zm, self.zs) = of(self.Y), of(self.Z)

    @staticmethod
    def stats_of(Y):
        m = Y.max(1).astype(np.float32)
        with np.errstate(invalid="ignore"):
            return m, np.exp(Y - m[:, None].astype(np.float64)).sum(1).astype(np.float32)

    def inputs(self):
        dev = lambda a: None if a is None else torch.from_numpy(a).cuda()      # noqa: E731

        def shards(Y):
            if Y is None:
                return None
            return [torch.from_numpy(y.copy()).to(TYPES[self.dtype]).cuda() for y in np.split(Y, np.cumsum(self.rows)[:-1], 1)]
        return dict(logits=shards(self.Y), shard_offsets=self.offsets, global_max=dev(self.m), global_sumexp=dev(self.s),
                    drafts=dev(self.drafts), starts=dev(self.starts), uniforms=dev(self.uniforms),
                    accepted=torch.full((len(self.starts) - 1,), UNTOUCHED, dtype=torch.int32, device="cuda"),
                    tokens=dev(self.tokens), draft_logits=shards(self.Z), draft_max=dev(self.zm), draft_sumexp=dev(self.zs))

    def run(self):
        import paper_2411_05288_amd as vp
        a = self.inputs()
        need = vp.vp_verify_workspace_bytes(len(self.starts) - 1, self.V)
        ws = torch.full((need + 256,), 0xFF, dtype=torch.uint8, device="cuda")
        vp.vp_verify_drafts(workspace=ws[:need], **a)
        torch.cuda.synchronize()
        assert bool((ws[need:] == 0xFF).all())
        return a["accepted"].cpu().numpy(), a["tokens"].cpu().numpy()

    def want(self):
        return ref.verify(self.Y, self.m, self.s, self.drafts, self.starts, self.uniforms, self.tokens, self.order, self.Z, self.zm,
                          self.zs)

    def check(self):
        """Equal, where no border between two tokens is within 1e-12 of a draw (sums of V terms in 64 bits are off by V 1e-16 at
        most, and here V is below 3000 in all but a few tests)."""
        accepted, tokens = self.run()
        a, t, margins = self.want()
        np.testing.assert_array_equal(accepted, a)
        assert (margins > 1e-12).all()
        np.testing.assert_array_equal(tokens, t)
        return a, t


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("model", [True, False])
@pytest.mark.parametrize("rows", [[1], [2], [7], [8], [64], [255, 2], [1000], [300, 300, 301], [13] * 24, [1] * 64, [2048], [2049, 1],
                                  [4095, 4097, 100]])
def test_vocabularies(rows, model, dtype):
    Case([0, 1, 2, 3, 4, 5, 0, 7, 2, 2] * 3, rows, dtype, model, seed=len(rows) + rows[0]).check()


@pytest.mark.parametrize("model", [True, False])
@pytest.mark.parametrize("counts", [[0], [1], [0] * 50, [63], [64], [65], [128], [129, 1], [200, 0, 300], list(range(40)), [1] * 300])
def test_numbers_of_drafts(counts, model):
    # (a draft without a model is accepted with probability 0.98, so that long runs of them are)
    Case(counts, [50, 60], "f32", model, seed=len(counts), sure=0.98).check()


@pytest.mark.parametrize("u", [0.0, 1e-30, 0.5, 1 - 2.0 ** -24])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_the_ends_of_the_random_numbers(u, dtype):
    """At 0 every draft of positive probability is accepted, and the first possible token is drawn; near 1 the last one."""
    c = Case([0, 1, 3, 0], [300, 211], dtype, seed=4)
    c.uniforms[:] = u
    c.Y[:, :3] = -np.inf
    c.Y[:, -2:] = -np.inf
    c.stats()
    a, t = c.check()
    if u == 0:
        assert a.tolist() == [0, 1, 3, 0] and (t[c.starts[1:] - 1] == 3).all()
    if u > 0.9:
        assert t[0] == 508


def test_sequences_without_rows_and_rows_behind():
    c = Case([None, 2, None, None, 0, 3, None], [100], "bf16", behind=5)
    a, t = c.check()
    assert (t[-5:] == UNTOUCHED).all() and a[0] == a[2] == a[3] == a[6] == 0


def test_starts_outside_are_taken_as_the_bounds():
    c = Case([2, 3, 1], [100])
    c.starts = np.array([-5, 3, 7, 1 << 40], np.int64)
    c.check()
    c.starts = np.array([3, 3, 2, 9], np.int64)      # (not ascending: an empty sequence; the next begins at 2)
    c.check()
    c.starts = np.array([-9, -1, 0, 0], np.int64)
    a, t = c.check()
    assert not a.any() and (t == UNTOUCHED).all()


def test_drafts_that_no_shard_owns():
    for model in (True, False):
        c = Case([3, 3, 3, 3], [40, 50], model=model, offsets=[100, 400])
        c.drafts[[0, 4, 8, 12]] = [-1, 140, 99, 1 << 62]
        a, t = c.check()
        assert not a.any()


def test_shards_with_gaps_and_out_of_order():
    c = Case([4] * 20, [40, 50, 60], "bf16", offsets=[1000, 10, 300])
    a, t = c.check()
    assert a.any() and set(t[t >= 0]) <= set(c.order.tolist())


def test_masked_tokens():
    """Of each model on its own: a draft that the target rules out is rejected, one that the draft model rules out is accepted if
    the target does not."""
    rng = np.random.default_rng(6)
    c = Case([4] * 40, [200, 133], "f32")
    c.Y[rng.random(c.Y.shape) < 0.4] = -np.inf
    c.Z[rng.random(c.Z.shape) < 0.4] = -np.inf
    c.stats()
    a, t = c.check()
    for b in range(40):
        i = c.starts[b]
        for e in range(a[b] + 1):
            assert c.Y[i + e, t[i + e]] > -np.inf
    c.drafts[:] = np.where(c.Z.min(1) == -np.inf, np.argmin(c.Z, 1), 0)
    c.check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [5, 300, 5000])
def test_rows_without_a_possible_token(V, dtype):
    c = Case([0, 0, 0, 1, 1, 0, 2, 0], [V], dtype, seed=8)
    at = c.starts[:-1]
    c.Y[at[0]] = -np.inf
    c.Y[at[1], V // 2] = np.nan
    c.Y[at[2], V - 1] = np.inf
    c.Y[at[3]] = -np.inf
    c.Z[at[4]] = np.nan
    c.stats()
    a, t = c.check()
    assert [t[i] for i in at[[0, 1, 2, 3, 4]]] == [-1] * 5 and not a[:5].any()
    assert t[at[5]] >= 0 and t[at[7]] >= 0


def test_statistics_without_a_number():
    c = Case([1, 1, 1, 1, 1], [300])
    c.m[0], c.s[2], c.zm[4], c.s[6], c.s[8] = np.nan, np.nan, np.nan, 0.0, np.inf
    a, t = c.check()
    assert t[0] == t[2] == t[4] == -1


LARGE = [-1e30, "min", 3e38, 1e12, -2.0 ** 34, 2.0 ** 34, -2.0 ** 33, 2.0 ** 33, 2.0 ** 28, -2.0 ** 28, 2.0 ** 27, -2.0 ** 27]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("model", [True, False])
@pytest.mark.parametrize("value", LARGE)
def test_rows_of_large_logits(value, model, dtype):
    """Rows whose largest logit has no number of its type within hundreds of it, as a constant far below all others leaves one where
    it rules out every token but those of -inf: only the tokens that have it can be drawn, and none behind a shard's end."""
    value = float(torch.finfo(TYPES[dtype]).min) if value == "min" else float(torch.tensor(value, dtype=TYPES[dtype]))
    c = Case([0, 1, 2, 0, 3] * 8, [300, 77, 513], dtype, model, seed=21)
    rng = np.random.default_rng(22)
    lower = float(torch.tensor(value - abs(value) / 4, dtype=TYPES[dtype]))
    for Y in (c.Y,) if c.Z is None else (c.Y, c.Z):
        Y[:] = np.where(rng.random(Y.shape) < 0.5, -np.inf, lower)
        Y[1::2] = -np.inf
        has = rng.random(Y.shape) < np.repeat([0.5, 0.02], [300, 590])
        has[np.arange(c.N), rng.integers(0, c.V, c.N)] = True      # (a token at least)
        Y[has] = value
    alone = c.starts[2]      # one token of the whole vocabulary, the last of the second shard
    c.Y[alone] = -np.inf
    c.Y[alone, 376] = value
    c.uniforms[::7] = 0.0
    c.stats()
    accepted, t = c.run()
    a, want, margins = c.want()
    for i, token in enumerate(t):
        assert token == -1 or (0 <= token < c.V and c.Y[i, token] == value)
    np.testing.assert_array_equal(accepted, a)
    assert (margins[c.uniforms[c.starts[1:] - 1] > 0] > 1e-12).all()      # (at 0 the first possible token is meant)
    np.testing.assert_array_equal(t, want)


@pytest.mark.parametrize("value", [v for v in LARGE if v not in (-1e30, "min", 3e38)])
def test_neighbours_of_large_logits(value):
    """Logits a few steps of their type below a large one keep their weights."""
    c = Case([0, 1, 2, 3] * 10, [300, 77], "f32", seed=23)
    rng = np.random.default_rng(24)
    for Y in (c.Y, c.Z):
        near = np.full(Y.shape, np.float32(value))
        for k in range(1, 41):
            step = np.nextafter(near, np.float32(-np.inf))
            near = np.where(rng.random(Y.shape) < 0.9, step, near)
        Y[:] = near
    c.stats()
    c.check()


def test_nothing_is_left_of_the_difference():
    """p nowhere above q, as roundings of the statistics can leave it: the token is drawn from p."""
    c = Case([1] * 30, [3000, 2000], seed=10)
    c.Z = c.Y.copy()
    c.stats()
    c.zs = (c.s * 0.5).astype(np.float32)
    c.uniforms[c.starts[:-1]] = 0.75
    a, t = c.check()
    assert not a.any() and len(set(t[c.starts[:-1]])) > 10
    one = Case([1], [1])      # (a vocabulary of one token, rejected)
    one.zs = one.zs * np.float32(0.5)
    one.uniforms[:] = 0.9
    a, t = one.check()
    assert a[0] == 0 and t.tolist() == [0, -1]


def test_nothing_is_read_of_the_last_rows_of_the_draft_model():
    c, d = Case([2, 0, 3], [300]), Case([2, 0, 3], [300])
    d.Z[d.starts[1:] - 1] = np.nan
    d.zm[d.starts[1:] - 1] = np.nan
    d.drafts[d.starts[1:] - 1] = 1 << 50
    np.testing.assert_array_equal(c.check()[1], d.check()[1])


@pytest.mark.parametrize("V,rows", [(128256, [16032] * 8), (256000, [16000] * 16), (50001, [16667] * 3)])
def test_large_vocabularies(V, rows):
    """(Sums of 256000 terms in 64 bits are off by less than 1e-10 of the whole, and the shares of the tokens are 4e-6.)"""
    c = Case([3, 0, 2, 4], rows, "bf16", seed=V)
    accepted, tokens = c.run()
    a, t, margins = c.want()
    np.testing.assert_array_equal(accepted, a)
    assert (margins > 1e-10).all()
    np.testing.assert_array_equal(tokens, t)


def test_rows_beyond_32_bits():
    import paper_2411_05288_amd as vp
    N, V = 2047, 1 << 20
    gen = torch.Generator(device="cuda").manual_seed(1)
    Y = torch.zeros(N, V, dtype=torch.bfloat16, device="cuda")
    Y[N - 2:] = torch.randn(2, V, generator=gen, device="cuda")
    m, s = torch.zeros(N, device="cuda"), torch.full((N,), float(V), device="cuda")
    m[N - 2:] = Y[N - 2:].float().amax(1)
    s[N - 2:] = torch.exp(Y[N - 2:].double() - m[N - 2:, None].double()).sum(1).float()
    drafts = torch.full((N,), V - 1, device="cuda")
    starts = torch.tensor([0, N - 2, N], device="cuda")
    u = torch.full((N,), 0.75, device="cuda")
    accepted, tokens = torch.zeros(2, dtype=torch.int32, device="cuda"), torch.zeros(N, dtype=torch.int64, device="cuda")
    ws = torch.empty(vp.vp_verify_workspace_bytes(2, V), dtype=torch.uint8, device="cuda")
    vp.vp_verify_drafts([Y], [0], m, s, drafts, starts, u, accepted, tokens, ws)
    torch.cuda.synchronize()
    a, t, margins = ref.verify(Y[N - 2:].double().cpu().numpy(), m[N - 2:].cpu().numpy(), s[N - 2:].cpu().numpy(),
                               np.full(2, V - 1), [0, 2], u[N - 2:].cpu().numpy(), np.zeros(2, np.int64), np.arange(V))
    assert accepted[1].item() == a[0] == 0 and margins[0] > 1e-9
    assert tokens[N - 2:].tolist() == t.tolist()
    assert accepted[0].item() == 0 and tokens[0].item() == int(0.75 * (V - 1)) and tokens[1].item() == -1


@pytest.mark.parametrize("model", [True, False])
def test_tokens_are_distributed_as_the_target_says(model):
    """Whatever the draft model is, the first token of a sequence is distributed as p.  Of S = 40000 sequences a token's count is
    within 5 deviations sqrt(S p (1 - p)) of S p (8 tokens: 1 in 200000 runs would not be; the seed is fixed)."""
    S = 40000
    c = Case([1] * S, [5, 3], "f32", model, seed=12, sure=None)
    rng = np.random.default_rng(13)
    c.Y[:] = rng.normal(0, 1, 8).astype(np.float32)
    if model:
        c.Z[:] = rng.normal(0, 1, 8).astype(np.float32)
        q = np.exp(c.Z[0]) / np.exp(c.Z[0]).sum()
        c.drafts[:] = rng.choice(8, c.N, p=q)
    else:
        c.drafts[:] = 3
    c.stats()
    accepted, tokens = c.run()
    p = np.exp(c.Y[0]) / np.exp(c.Y[0]).sum()
    first = np.bincount(tokens[c.starts[:-1]], minlength=8)
    assert (np.abs(first - S * p) <= 5 * np.sqrt(S * p * (1 - p))).all()
    share = np.minimum(p, q).sum() if model else p[3]
    assert abs(accepted.sum() - S * share) <= 5 * math.sqrt(S * share * (1 - share))
    behind = tokens[c.starts[:-1] + 1][accepted == 1]
    n = len(behind)
    assert (np.abs(np.bincount(behind, minlength=8) - n * p) <= 5 * np.sqrt(n * p * (1 - p))).all()


def test_logits_that_start_at_any_element():
    import paper_2411_05288_amd as vp
    c = Case([2, 3, 0], [77, 31], "bf16")
    a, need = c.inputs(), vp.vp_verify_workspace_bytes(3, 108)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    for name in ("logits", "draft_logits"):
        flat = torch.zeros(4000, dtype=torch.bfloat16, device="cuda")
        at, views = 1, []
        for t in a[name]:
            views.append(flat[at:at + t.numel()].view_as(t))
            views[-1].copy_(t)
            at += t.numel()
        a[name] = views
    vp.vp_verify_drafts(workspace=ws, **a)
    np.testing.assert_array_equal(a["tokens"].cpu().numpy(), c.want()[1])


@pytest.mark.parametrize("model", [True, False])
def test_the_checks_in_python_lead_to_the_same_call(model, monkeypatch):
    import paper_2411_05288_amd.binding as B
    B.load_library()
    c = Case([2, 0, 5, 1], [300, 77], "bf16", model)
    native = c.check()
    assert B._HOST is not None
    monkeypatch.setattr(B, "_HOST", None)
    for a, b in zip(native, c.run()):
        np.testing.assert_array_equal(a, b)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("model", [True, False])
def test_many_sequences_of_a_large_vocabulary(model, dtype):
    """More segments than wavefronts on the chip: the token is checked by its place in the running sum of 64 bits."""
    import paper_2411_05288_amd as vp
    S, rows = 700, [6500, 6501]
    N, V = 2 * S, sum(rows)
    gen = torch.Generator(device="cuda").manual_seed(3)
    Y = [(2 * torch.randn(N, n, generator=gen, device="cuda")).to(TYPES[dtype]) for n in rows]
    Z = [(y.float() + 0.5 * torch.randn(N, y.shape[1], generator=gen, device="cuda")).to(TYPES[dtype]) for y in Y] if model else None

    def stats(shards):
        m = torch.cat(shards, 1).float().amax(1)
        return m, torch.exp(torch.cat(shards, 1).double() - m[:, None].double()).sum(1).float()
    (m, s), (zm, zs) = stats(Y), stats(Z) if model else (None, None)
    drafts = torch.randint(0, V, (N,), generator=gen, device="cuda")
    starts = torch.arange(0, N + 1, 2, device="cuda")
    u = torch.rand(N, generator=gen, device="cuda")
    accepted, tokens = torch.empty(S, dtype=torch.int32, device="cuda"), torch.empty(N, dtype=torch.int64, device="cuda")
    ws = torch.full((vp.vp_verify_workspace_bytes(S, V),), 0xFF, dtype=torch.uint8, device="cuda")
    vp.vp_verify_drafts(Y, [0, rows[0]], m, s, drafts, starts, u, accepted, tokens, ws, draft_logits=Z, draft_max=zm, draft_sumexp=zs)
    first = torch.arange(0, N, 2, device="cuda")
    p = torch.exp(torch.cat(Y, 1).double() - m[:, None].double()) / s[:, None].double()
    q = torch.exp(torch.cat(Z, 1).double() - zm[:, None].double()) / zs[:, None].double() if model else torch.nn.functional.one_hot(drafts, V).double()
    d = drafts[first]
    ok = u[first].double() * q[first, d] < p[first, d]
    assert torch.equal(accepted, ok.int())
    w = torch.where(ok[:, None], p[first + 1], (p[first] - q[first]).clamp(min=0))
    c = w.cumsum(1)
    token = tokens[torch.where(ok, first + 1, first)]
    target = u[first + 1].double() * c[:, -1]
    upto = c.gather(1, token[:, None])[:, 0]
    before = upto - w.gather(1, token[:, None])[:, 0]
    # sums of 13001 terms in 64 bits: off by less than 1e-11 of the whole
    assert bool((before <= target + 1e-11 * c[:, -1]).all()) and bool((upto >= target - 1e-11 * c[:, -1]).all())
    assert bool((w.gather(1, token[:, None]) > 0).all())
    assert bool((tokens[first[ok]] == d[ok]).all()) and bool((tokens[first[~ok] + 1] == -1).all())


def test_python_refusals():
    import paper_2411_05288_amd as vp
    c = Case([2, 3], [77, 31], "bf16")
    good = {**c.inputs(), "workspace": torch.empty(1 << 16, dtype=torch.uint8, device="cuda")}
    vp.vp_verify_drafts(**good)
    z = lambda *s, dtype=torch.float32: torch.zeros(*s, dtype=dtype, device="cuda")      # noqa: E731
    for bad in (dict(logits=[]), dict(logits=[z(7, 77), z(7, 31)]), dict(logits=good["logits"][:1]), dict(shard_offsets=[0]),
                dict(shard_offsets=[0, 76]), dict(global_max=z(6)), dict(global_sumexp=z(7, dtype=torch.float64)), dict(drafts=z(7)),
                dict(drafts=z(8, dtype=torch.int64)), dict(starts=z(3)), dict(starts=z(1, dtype=torch.int64)),
                dict(starts=z(3, 1, dtype=torch.int64)), dict(uniforms=z(6)), dict(accepted=z(2, dtype=torch.int64)),
                dict(accepted=z(3, dtype=torch.int32)), dict(tokens=z(7, dtype=torch.int32)), dict(draft_logits=None),
                dict(draft_max=None), dict(draft_logits=good["draft_logits"][:1]), dict(workspace=z(16, dtype=torch.uint8)),
                dict(tokens=good["drafts"]), dict(logits=[z(7), z(7)])):
        with pytest.raises(vp.VPError):
            vp.vp_verify_drafts(**{**good, **bad})
