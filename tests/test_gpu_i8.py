"""Rows in 8-bit integers and the output layer's logits and statistics from them, against exact integers and 64 bits."""
import math

import numpy as np
import pytest
import torch

import answer_reference as ref

pytestmark = pytest.mark.gpu
U = 2.0 ** -24      # half a step of fp32, relative
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def poisoned(*shape, dtype):
    """A GPU tensor between two bands of 256 bytes of 0xA5, which it is itself full of: (tensor, check that the bands are whole)."""
    n = int(np.prod(shape)) * torch.empty((), dtype=dtype).element_size()
    raw = torch.full((n + 512 + 15,), 0xA5, dtype=torch.uint8, device="cuda")
    t = raw[256:256 + n].view(dtype).reshape(shape)
    return t, lambda: bool((raw[:256] == 0xA5).all()) and bool((raw[256 + n:] == 0xA5).all())


def quantize(x):
    import paper_2411_05288_amd as vp
    N, h = x.shape
    stride = vp.vp_i8_row_stride(h)
    q, q_whole = poisoned(N, stride, dtype=torch.int8)
    s, s_whole = poisoned(N, dtype=torch.float32)
    vp.vp_quantize_rows(x, q, s)
    torch.cuda.synchronize()
    assert q_whole() and s_whole()
    q = q.cpu().numpy()
    assert not q[:, h:].any()
    return q[:, :h].astype(np.int64), s.cpu().numpy()


def same(got, want):
    np.testing.assert_array_equal(got[0], want[0])
    np.testing.assert_array_equal(got[1].view(np.uint32) & 0x7fffffff if np.isnan(want[1]).any() else got[1],
                                  want[1].view(np.uint32) & 0x7fffffff if np.isnan(want[1]).any() else want[1])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N,h", [(1, 1), (1, 7), (3, 8), (2, 16), (5, 127), (4, 128), (3, 129), (9, 200), (300, 256), (65, 333), (2, 1001),
                                 (33, 1024), (7, 2048), (5, 2050), (4, 4096), (2, 5000), (3, 8192), (2, 16384), (2, 16391), (1, 32768),
                                 (1, 40001), (1, 130944), (2000, 8)])
def test_rows(N, h, dtype):
    gen = torch.Generator().manual_seed(N * 1000 + h)
    x = (torch.randn(N, h, generator=gen) * torch.exp(torch.randn(N, 1, generator=gen))).to(TYPES[dtype])
    same(quantize(x.cuda()), ref.quantize_rows_fast(x.double().numpy()))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("largest", [127.0, 254.0, 63.5, 1.9921875, 127 * 2.0 ** -20, 127 * 2.0 ** 100, 127 * 2.0 ** -126])
def test_halves_go_to_even(largest, dtype):
    """127 x / largest = k + 1/2 for every k, of both signs, and with fp32 the numbers beside them."""
    halves = torch.tensor([(k + 0.5) * (largest / 127) for k in range(127)], dtype=torch.float64).float()
    if dtype == "bf16":
        halves = halves.to(torch.bfloat16).float()
    beside = torch.cat([halves, torch.nextafter(halves, torch.zeros(())), torch.nextafter(halves, torch.tensor(math.inf))])
    row = torch.cat([torch.tensor([largest]), halves if dtype == "bf16" else beside])
    x = torch.stack([row, -row]).to(TYPES[dtype])
    x = x.clamp(-largest, largest)
    same(quantize(x.cuda()), ref.quantize_rows(x.double().numpy()))


@pytest.mark.parametrize("h", [5, 64, 700, 5000, 40000])
def test_numbers_of_all_sizes(h):
    """Subnormal rows, the largest numbers, zeros of both signs, and rows that are not finite, which change no other row."""
    gen = torch.Generator().manual_seed(h)
    x = torch.randn(10, h, generator=gen)
    x[0] *= 1e-40
    x[1] = 0
    x[1, 0] = -0.0
    x[2] = torch.sign(x[2]) * torch.finfo(torch.float32).max
    x[3, h // 2] = math.inf
    x[4, h - 1] = -math.inf
    x[5, 0] = math.nan
    x[6] = 2.0 ** -149 * (x[6] > 0)
    x[6, 0] = 2.0 ** -149
    x[7] *= 1e-30
    x[7, 1] = 1e30
    x[8] *= 3e37
    same(quantize(x.cuda()), ref.quantize_rows(x.double().numpy()))
    finite = torch.isfinite(x.to(torch.bfloat16)).all(1) | (torch.arange(10) == 3)
    y = x.to(torch.bfloat16)[finite]
    same(quantize(y.cuda()), ref.quantize_rows(y.double().numpy()))


def test_rows_far_into_a_large_matrix():
    """Elements beyond 2^31 bytes."""
    N, h = 16000, 131000 - 56
    x = torch.zeros(N, h, dtype=torch.bfloat16, device="cuda")
    gen = torch.Generator(device="cuda").manual_seed(3)
    some = [0, 8196, 16383 - 400, N - 1]
    for i in some:
        x[i] = torch.randn(h, generator=gen, device="cuda")
    import paper_2411_05288_amd as vp
    q, s = vp.quantize_rows(x)
    torch.cuda.synchronize()
    for i in some:
        want = ref.quantize_rows_fast(x[i:i + 1].double().cpu().numpy())
        np.testing.assert_array_equal(q[i].cpu().numpy().astype(np.int64), want[0][0])
        assert s[i].item() == want[1][0]
    assert not q[1].any() and s[1].item() == 0


# ------------------------------------------------------------------------------------------------ the product
class Product:
    """A call and what it should give.  Values y = fl(fl(float(sum) t) s) or in another order: three roundings, at most 4 U off
    relative to y (2 to the -8 more where they are kept in bf16).  The sum of exponentials is compared with the one of the exact
    logits around the maximum that the call gave: with A the row's largest |y|, the exponents of a term are off by at most
    (4 + 4) U A for the logits, 8 U A for the arguments' roundings (each at most 2 A in size) and as much again where a tile's sum
    joins others, the exponentials by 4 U each, the sum of a tile's 256 terms by 256 U, that of the tiles by 4 U for each."""

    def __init__(self, N, k, rows, dtype, seed=1, keep=True, q=None, single=False, offsets=None):
        rng = np.random.default_rng(seed)
        self.N, self.k, self.rows, self.dtype, self.keep = N, k, rows, dtype, keep
        V = sum(rows)
        self.H = rng.integers(-127, 128, (N, k)).astype(np.int8) if q is None else np.full((N, k), q, np.int8)
        self.W = rng.integers(-127, 128, (V, k)).astype(np.int8) if q is None else np.full((V, k), q, np.int8)
        # (logits of a size that a model has, whatever k is; outputs that hold infinities come with the extremes)
        self.sH = (rng.uniform(0.5, 2, N) * 4 / (5400 * math.sqrt(k))).astype(np.float32)
        self.sW = rng.uniform(0.5, 2, V).astype(np.float32)
        self.offsets = np.cumsum([0] + rows[:-1]).tolist() if offsets is None else offsets
        self.labels = rng.integers(-3, V + 3, N)
        self.single = single

    def run(self, stream=None):
        import paper_2411_05288_amd as vp
        dev = lambda a: torch.from_numpy(a).cuda()      # noqa: E731
        p, N, rows = len(self.rows), self.N, self.rows
        cuts = np.cumsum(rows)[:-1]
        W, sW = [dev(w) for w in np.split(self.W, cuts)], [dev(t) for t in np.split(self.sW, cuts)]
        stats = [poisoned(p, N, dtype=torch.float32) for _ in range(3)]
        logits = [poisoned(N, n, dtype=TYPES[self.dtype]) for n in rows] if self.keep else None
        need = vp.vp_output_i8_workspace_bytes(N, rows)
        ws, ws_whole = poisoned(need, dtype=torch.uint8)
        ws.fill_(0xFF)
        m, s, t = (a for a, _ in stats)
        Y = None if logits is None else [a for a, _ in logits]
        H, sH, labels = dev(self.H), dev(self.sH), dev(self.labels)
        if self.single:
            vp.vp_output_fwd_i8(H, sH, W[0], sW[0], labels, self.offsets[0], m[0], s[0], t[0], Y and Y[0], ws)
        else:
            vp.vp_output_fwd_i8_group(H, sH, W, sW, labels, self.offsets, m, s, t, Y, ws)
        torch.cuda.synchronize()
        assert ws_whole() and all(whole() for _, whole in stats + (logits or []))
        return m, s, t, Y

    def check(self, out):
        m, s, t = (a.cpu().numpy().astype(np.float64) for a in out[:3])
        want = ref.logits(self.H, self.sH, self.W, self.sW)
        for r, (n, at) in enumerate(zip(self.rows, np.cumsum([0] + self.rows))):
            y = want[:, at:at + n]
            A = np.abs(y).max(1)
            assert (np.abs(m[r] - y.max(1)) <= 4 * U * A).all()
            sums = np.exp(y - m[r][:, None]).sum(1)
            assert (np.abs(s[r] / sums - 1) <= U * (24 * A + 12 + 256 + 4 * -(-n // 256))).all()
            local = self.labels - self.offsets[r]
            own = (local >= 0) & (local < n)
            target = np.where(own, y[np.arange(self.N), np.clip(local, 0, n - 1)], 0)
            assert (np.abs(t[r] - target) <= 4 * U * np.abs(target)).all()
            if out[3] is not None:
                got = out[3][r].double().cpu().numpy()
                assert (np.abs(got - y) <= (4 * U + (2.0 ** -8 if self.dtype == "bf16" else 0)) * np.abs(y)).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N", [1, 2, 17, 31, 32, 33, 64, 65, 100, 128, 129, 192, 200, 257, 300])
@pytest.mark.parametrize("k,rows", [(128, [256]), (256, [300, 5]), (384, [1, 255, 257]), (640, [513, 1000])])
def test_product(N, k, rows, dtype):
    case = Product(N, k, rows, dtype, seed=N + k)
    case.check(case.run())


@pytest.mark.parametrize("k", [128 * i for i in (1, 2, 3, 4, 5, 6, 7, 9, 10, 11, 16, 32, 64)])
@pytest.mark.parametrize("N", [1, 40, 150, 400])
def test_lengths_of_the_sum(N, k):
    case = Product(N, k, [270], "f32", seed=k)
    case.check(case.run())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N", [1, 64, 65, 96, 97, 128, 129, 192, 193, 256, 300, 513])
@pytest.mark.parametrize("k,rows", [(2048, [300, 5]), (2176, [300, 5]), (2304, [1, 255, 257]), (4096, [513, 1000])])
def test_long_sums(N, k, rows, dtype):
    """On both sides of every choice between the kernels: sums of 2048, 64 and 128 tokens, tiles of 64 to 256 tokens."""
    case = Product(N, k, rows, dtype, seed=N + k)
    case.check(case.run())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N,k,rows", [(300, 128, [25000, 26001]), (300, 128, [25600, 25600]), (300, 2304, [20001, 20002]),
                                      (2200, 128, [3000, 3001]), (2200, 2304, [3001]), (40, 256, [70001]), (100, 2304, [70001])])
def test_more_tiles_than_compute_units(N, k, rows, dtype):
    case = Product(N, k, rows, dtype, seed=k)
    case.check(case.run())


@pytest.mark.parametrize("N,k,rows", [(1, 128, [1]), (3, 128, [7] * 20), (5, 256, [64] * 16), (40, 256, [300] * 17), (300, 128, [100] * 40)])
def test_many_shards(N, k, rows):
    case = Product(N, k, rows, "bf16", seed=5)
    case.check(case.run())


@pytest.mark.parametrize("N", [1, 40, 300])
def test_statistics_alone(N):
    kept, alone = Product(N, 256, [300, 700], "f32"), Product(N, 256, [300, 700], "f32", keep=False)
    a, b = kept.run(), alone.run()
    alone.check(b)
    for x, y in zip(a[:3], b[:3]):
        assert torch.equal(x, y)


@pytest.mark.parametrize("N", [1, 33, 300])
def test_single_calls_equal_the_group(N):
    rows = [300, 31, 512]
    group = Product(N, 384, rows, "bf16", seed=9)
    m, s, t, Y = group.run()
    for r, at in enumerate(group.offsets):
        one = Product(N, 384, [rows[r]], "bf16", single=True, offsets=[at])
        one.H, one.sH, one.labels = group.H, group.sH, group.labels
        one.W, one.sW = group.W[at:at + rows[r]], group.sW[at:at + rows[r]]
        a = one.run()
        for x, y in zip(a[:3], (m, s, t)):
            assert torch.equal(x[0], y[r])
        assert torch.equal(a[3][0], Y[r])


@pytest.mark.parametrize("N", [1, 70, 260])
@pytest.mark.parametrize("q,k", [(127, 130944), (-127, 4096), (-128, 130944)])
def test_the_largest_sums(N, q, k):
    case = Product(N, k, [270], "f32", q=q)
    case.sH[:] = 2.0 ** -30
    case.check(case.run())


@pytest.mark.parametrize("N", [3, 100, 300])
def test_tokens_and_columns_without_a_number(N):
    """Scales of zero give logits of zero, a NaN its token's or column's logits, and no other's."""
    clean, case = Product(N, 256, [300, 400], "f32", seed=3), Product(N, 256, [300, 400], "f32", seed=3)
    for c in (clean, case):
        c.sH[0] = 0
        c.sW[5] = 0
    case.sH[1] = np.nan
    a, b = clean.run(), case.run()
    clean.check(a)
    others = [i for i in range(N) if i != 1]
    for x, y in zip(a[:3], b[:3]):
        assert torch.equal(x[:, others], y[:, others])
    for x, y in zip(a[3], b[3]):
        assert torch.equal(x[others], y[others]) and bool(torch.isnan(y[1]).all())
        assert not x[0].any()
    case.sH[1] = clean.sH[1]
    case.sW[7] = np.nan
    b = case.run()
    assert bool(torch.isnan(b[3][0][:, 7].cpu()[1:]).all())
    columns = [j for j in range(300) if j != 7]
    assert torch.equal(a[3][0][:, columns], b[3][0][:, columns]) and torch.equal(a[3][1], b[3][1])
    assert torch.equal(a[0][1], b[0][1])


@pytest.mark.parametrize("dtype,N", [("bf16", 2047), ("f32", 1030)])
def test_outputs_beyond_32_bits(dtype, N):
    import paper_2411_05288_amd as vp
    Vs, k = 1 << 20, 128
    gen = torch.Generator(device="cuda").manual_seed(7)
    H = torch.randint(-127, 128, (N, k), generator=gen, device="cuda", dtype=torch.int8)
    W = torch.randint(-127, 128, (Vs, k), generator=gen, device="cuda", dtype=torch.int8)
    sH, sW = torch.rand(N, generator=gen, device="cuda") * 1e-5, torch.rand(Vs, generator=gen, device="cuda")
    Y = torch.zeros(N, Vs, dtype=TYPES[dtype], device="cuda")
    m, s, t = (torch.zeros(N, device="cuda") for _ in range(3))
    ws = torch.empty(vp.vp_output_i8_workspace_bytes(N, [Vs]), dtype=torch.uint8, device="cuda")
    vp.vp_output_fwd_i8(H, sH, W, sW, torch.full((N,), Vs - 1, device="cuda"), 0, m, s, t, Y, ws)
    torch.cuda.synchronize()
    some = torch.tensor([0, 1, N // 2, N - 1], device="cuda")
    want = torch.mm(H[some].double(), W.double().t().contiguous()) * sH[some, None].double() * sW.double()      # (whole sums)
    bound = (4 * U + (2.0 ** -8 if dtype == "bf16" else 0)) * want.abs()
    assert bool(((Y[some].double() - want).abs() <= bound).all())
    assert bool(((t[some].double() - want[:, -1]).abs() <= 4 * U * want[:, -1].abs()).all())
    assert bool(((m[some].double() - want.amax(1)).abs() <= 4 * U * want.abs().amax(1)).all())


def test_repeats_bit_for_bit():
    case = Product(70, 512, [1000, 1000], "bf16", seed=2)
    a, b = case.run(), case.run()
    assert all(torch.equal(x, y) for x, y in zip((*a[:3], *a[3]), (*b[:3], *b[3])))


@pytest.mark.parametrize("N", [1, 40, 100])
def test_the_checks_in_python_lead_to_the_same_calls(N, monkeypatch):
    import paper_2411_05288_amd.binding as B
    B.load_library()
    case = Product(N, 256, [300, 77], "bf16", seed=4)
    x = torch.randn(N, 200, generator=torch.Generator().manual_seed(1)).cuda()
    native, rows = case.run(), quantize(x)
    assert B._HOST is not None
    monkeypatch.setattr(B, "_HOST", None)
    python, same_rows = case.run(), quantize(x)
    assert all(torch.equal(a, b) for a, b in zip((*native[:3], *native[3]), (*python[:3], *python[3])))
    assert (rows[0] == same_rows[0]).all() and (rows[1] == same_rows[1]).all()


def test_python_refusals():
    import paper_2411_05288_amd as vp
    z = lambda *s, dtype=torch.float32: torch.zeros(*s, dtype=dtype, device="cuda")      # noqa: E731
    i8 = lambda *s: z(*s, dtype=torch.int8)      # noqa: E731
    for bad in (dict(x=z(4)), dict(q=i8(4, 100)), dict(q=z(4, 128)), dict(scales=z(3)), dict(scales=z(4, dtype=torch.float64)),
                dict(x=z(100, 4).t()), dict(x=torch.zeros(4, 100)), dict(x=z(4, 100, dtype=torch.float16))):
        with pytest.raises(vp.VPError):
            vp.vp_quantize_rows(**{**dict(x=z(4, 100), q=i8(4, 128), scales=z(4)), **bad})
    good = dict(H=i8(4, 128), H_scales=z(4), W_shards=[i8(30, 128), i8(20, 128)], W_scales=[z(30), z(20)],
                labels=z(4, dtype=torch.int64), shard_offsets=[0, 30], local_max=z(2, 4), local_sumexp=z(2, 4), local_target=z(2, 4),
                logits_out=[z(4, 30), z(4, 20)], workspace=z(1 << 16, dtype=torch.uint8))
    vp.vp_output_fwd_i8_group(**good)
    for bad in (dict(H=i8(4, 256)), dict(H=z(4, 128)), dict(H_scales=z(5)), dict(W_shards=[i8(30, 128)]), dict(W_scales=[z(30)]),
                dict(W_scales=[z(30), z(21)]), dict(shard_offsets=[0]), dict(labels=z(4)), dict(local_max=z(1, 4)),
                dict(logits_out=[z(4, 30)]), dict(logits_out=[z(4, 30), z(4, 21)]), dict(workspace=None),
                dict(logits_out=[z(4, 30), z(4, 20, dtype=torch.bfloat16)]), dict(H=i8(128, 4).t()), dict(H=i8(128)),
                dict(logits_out=[]), dict(logits_out=[z(4, 30, dtype=torch.float16), z(4, 20, dtype=torch.float16)]),
                dict(W_shards=[], W_scales=[], shard_offsets=[], logits_out=None), dict(local_max=good["local_sumexp"])):
        with pytest.raises(vp.VPError):
            vp.vp_output_fwd_i8_group(**{**good, **bad})


@pytest.mark.parametrize("N,k", [(3, 128), (40, 256), (100, 2304), (300, 256), (300, 2304), (600, 2304)])
@pytest.mark.parametrize("rows,nan", [([300, 1, 400], [300]), ([300, 400], list(range(300, 700))), ([300, 31], list(range(300, 331))),
                                      ([600], list(range(128, 256))), ([600], list(range(256, 512))), ([600], list(range(512, 600))),
                                      ([600], [599]), ([600], list(range(600))), ([33], [32]), ([129], [128]), ([257, 40], [256])])
def test_sums_with_a_nan(rows, nan, N, k):
    """A NaN makes the sums NaN that it is part of, also where a tile, a wavefront's part of one or a shard holds nothing else; the
    other shards' statistics and, with a token's NaN, the other tokens' stay."""
    import paper_2411_05288_amd as vp
    clean, case, token = (Product(N, k, rows, "bf16", seed=8) for _ in range(3))
    case.sW[nan] = np.nan
    token.sH[N - 1] = np.nan
    a, b, c = clean.run(), case.run(), token.run()
    clean.check(a)
    shard_of = np.repeat(np.arange(len(rows)), rows)
    hit = sorted(set(shard_of[nan].tolist()))
    rest = [r for r in range(len(rows)) if r not in hit]
    for x, y in zip(a[:3], b[:3]):
        assert torch.equal(x[rest], y[rest])
    for x, y in zip(a[:3], c[:3]):
        assert torch.equal(x[:, :-1], y[:, :-1])
    assert bool(torch.isnan(b[1][hit]).all()) and bool(torch.isnan(c[1][:, -1]).all())
    for stats, tokens in ((b, slice(None)), (c, slice(N - 1, N))):
        m, s, loss = (torch.zeros(N, device="cuda") for _ in range(3))
        vp.vp_combine_stats(*stats[:3], m, s, loss, torch.zeros(1, device="cuda"))
        assert bool(torch.isnan(s[tokens]).all()) and bool(torch.isnan(loss[tokens]).all())
        if stats is c:
            assert bool(torch.isfinite(loss[:-1]).all())
