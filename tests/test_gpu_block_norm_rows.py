"""The backward pass of the norms around a block where every group of threads takes several rows, one after the other: sums over
tokens in small whole numbers, which fp32 adds up without rounding (a row that is lost, doubled or added to another row of the
gate changes them), and gradients of activations against the formulas."""
import pytest
import torch

import norm_reference as ref

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
# Rows of 16 and 32 lanes, of one, three, eight and sixteen wavefronts, of two and four vectors per thread, and below and above what
# one pass takes; N is a multiple of 7, 3 and 10.
SIZES = [(50400, 24), (25200, 200), (12600, 264), (5040, 1043), (1680, 4096), (840, 8192), (840, 8203), (840, 18437), (1680, 5), (420, 33000)]


def rows_in_a_row(N, h):
    """How many rows a group of threads takes: the workspace without post norm and gate is two partial matrices of a row for every
    workgroup, and a workgroup has at most 1024 threads in groups of 16, 32 or whole wavefronts that hold a row."""
    import paper_2411_05288_amd as vp
    one_pass = 8 <= h <= 32768
    size = vp.vp_block_norm_bwd_workspace_bytes(N, h) - (0 if one_pass else (N * 16 + 255) // 256 * 256)
    parts = size // (2 * ((h + 3) // 4 * 4) * 4)
    vectors = -(-h // 8)
    threads = 16 if h <= 128 else 32 if h <= 256 else -(-(vectors if h <= 8192 else -(-vectors // (2 if h <= 16384 else 4))) // 64) * 64
    return N / (parts * (1024 // threads if one_pass else 1))


def gates(N):
    """No gate, one row, a row for every token; rows of 7 and 3 tokens, which begin and end within what a group of threads takes
    (four rows), and ten rows that many groups share."""
    return [0, 1, N, N // 7, N // 3, 10]


def whole(g, shape, most, dtype):
    return torch.randint(-most, most + 1, shape, generator=g, device="cuda").to(dtype)


def rows_of(v, gate):
    """Sums over the tokens of every row of the gate."""
    return v.reshape(gate, -1, v.shape[1]).sum(1)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("N,h", SIZES)
def test_sums_over_tokens_in_whole_numbers(N, h, dtype):
    """With rho2 = 0, dx is dr; with rho1 = 1 and m1 = 0, yh is y.  The largest sums, of 2 * 2 * 3 * 3 per token and of 2 * 8 * 3, stay
    below 2^24."""
    import paper_2411_05288_amd as vp
    assert rows_in_a_row(N, h) >= 3
    assert 48 * N < 1 << 24
    g = torch.Generator(device="cuda").manual_seed(N + h)
    dH, r, y, dr = (whole(g, (N, h), 3, t) for t in (F32, dtype, dtype, dtype))
    w, w_post, b_post = (whole(g, (h,), 2, dtype) for _ in range(3))
    stats = torch.zeros(4, N, device="cuda")
    stats[1], stats[3] = 1.0, 1.0
    still = stats.clone()
    still[3] = 0.0
    D, R, Y, DR = (t.double() for t in (dH, r, y, dr))
    dw, db = (D * R).sum(0), D.sum(0)
    for G in gates(N):
        gate = whole(g, (G, h), 2, dtype) if G else None
        d = 2 * DR if gate is None else 2 * DR * ref.gate_rows(gate, N)
        for post in (False, True):
            u = Y * w_post.double() + b_post.double() if post else Y
            exact = {"dgate": rows_of(2 * u * DR, G)} if G else {}
            exact.update({"dw_post": (d * Y).sum(0), "db_post": d.sum(0)} if post else {})
            ws = torch.full((vp.vp_block_norm_bwd_workspace_bytes(N, h, G, post),), 0xFF, dtype=torch.uint8, device="cuda")
            opts = dict(gate=gate, w=w, w_post=w_post if post else None, b_post=b_post if post else None, scale=2.0, post=post, workspace=ws)
            for every in (True, False):      # all kinds of sums, or those of RMS norms without biases
                def call(stats, names):
                    names = [k for k in names if every or not k.startswith("db")]
                    out = {k: torch.full((G, h) if k == "dgate" else (h,), float("nan"), device="cuda") for k in names}
                    dx, dy = torch.empty_like(dr), torch.empty_like(dr)
                    ws.fill_(0xFF)
                    vp.vp_block_norm_bwd(dH, r, y, stats, dr=dr, dx=dx, dy=dy, **out, **opts)
                    return dx, dy, out
                _, _, out = call(stats, ["dw", "db"])
                assert torch.equal(out["dw"].double(), dw) and (not every or torch.equal(out["db"].double(), db)), (G, post, every)
                dx, dy, out = call(still, ["db", *exact])
                assert torch.equal(dx, dr) and (not every or torch.equal(out.pop("db").double(), db)), (G, post, every)
                for k, t in out.items():
                    assert torch.equal(t.double(), exact[k]), (G, post, every, k)
                if not post:
                    assert torch.equal(dy.double(), d.to(dtype).double()), (G, every)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("N,h", SIZES)
def test_gradients_of_activations(N, h, dtype):
    """The rows that a group takes after its first one, whose values come while the sums of the one before are formed."""
    import paper_2411_05288_amd as vp
    g = torch.Generator(device="cuda").manual_seed(N + h + 1)

    def normal(*shape, mean=0.0, std=1.0, dtype=dtype):
        return (torch.randn(*shape, generator=g, device="cuda") * std + mean).to(dtype)
    x, y, dH, dr = normal(N, h, mean=0.2), normal(N, h, std=2.0), normal(N, h, dtype=F32), normal(N, h)
    w, w_post, b_post = normal(h, mean=1.0, std=0.2), normal(h, mean=1.0, std=0.2), normal(h, std=0.3)
    for k, G in enumerate(gates(N)):
        post, center = k % 2 == 0, k % 3 == 0
        opts = dict(gate=normal(G, h, mean=0.5) if G else None, w_post=w_post if post else None, b_post=b_post if post else None, scale=0.5, post=post,
                    center=center)
        H, r, stats = torch.empty_like(x), torch.empty_like(x), torch.empty(4, N, device="cuda")
        vp.vp_block_norm_fwd(x, y, H, r=r, stats=stats, w=w, **opts)
        ws = torch.full((vp.vp_block_norm_bwd_workspace_bytes(N, h, G, post),), 0xFF, dtype=torch.uint8, device="cuda")
        dx, dy, dw = torch.empty_like(x), torch.empty_like(x), torch.empty(h, device="cuda")
        vp.vp_block_norm_bwd(dH, r, y, stats, dr=dr, w=w, dx=dx, dy=dy, dw=dw, workspace=ws, **opts)
        expected = ref.backward(dH, r, y, stats, dr=dr, w=w, grad_dtype=dtype, **opts)
        for name, t in (("dx", dx), ("dy", dy), ("dw", dw)):
            ref.check(name, t, *expected[name])


@pytest.mark.parametrize("value", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("N,h", [(50400, 24), (12600, 264), (5040, 1043), (840, 8203), (840, 18437), (1680, 5)])
def test_what_is_not_finite_stays_in_its_row_and_columns(N, h, value):
    """Of dH: its row of dx and dy, its column of dw, and its token's row of dgate; everything else as without it, bit for bit."""
    import paper_2411_05288_amd as vp
    g = torch.Generator(device="cuda").manual_seed(h)
    x, y, dH = (torch.randn(N, h, generator=g, device="cuda").to(t) for t in (BF16, BF16, F32))
    gate = torch.randn(N // 7, h, generator=g, device="cuda").bfloat16()
    H, r, stats = torch.empty_like(x), torch.empty_like(x), torch.empty(4, N, device="cuda")
    vp.vp_block_norm_fwd(x, y, H, r=r, stats=stats, gate=gate, post=True, center=True)
    ws = torch.empty(vp.vp_block_norm_bwd_workspace_bytes(N, h, N // 7, post=True), dtype=torch.uint8, device="cuda")

    def back(dH):
        out = {"dx": torch.empty_like(x), "dy": torch.empty_like(x), "dgate": torch.empty(N // 7, h, device="cuda"), "dw": torch.empty(h, device="cuda")}
        ws.fill_(0xFF)
        vp.vp_block_norm_bwd(dH, r, y, stats, gate=gate, post=True, center=True, workspace=ws, **out)
        return out
    clean = back(dH)
    for row, column in ((0, 0), (N // 2 + 1, h - 1), (N - 1, h // 2)):
        bad = dH.clone()
        bad[row, column] = value
        got = back(bad)
        assert not torch.isfinite(got["dw"][column]) and not torch.isfinite(got["dx"][row, column])
        hit = {"dx": row, "dy": row, "dgate": row // 7, "dw": column}
        for k, at in hit.items():
            left = torch.ones(got[k].shape[0], dtype=torch.bool, device="cuda")
            left[at] = False
            assert torch.equal(got[k][left], clean[k][left]), (k, row, column)


@pytest.mark.parametrize("N,h,dtype", [(50400, 24, BF16), (5040, 1043, F32), (840, 8203, BF16), (420, 33000, F32)])
@pytest.mark.parametrize("center", [False, True])
def test_all_gradients_of_the_norm_alone(N, h, dtype, center):
    import paper_2411_05288_amd as vp
    g = torch.Generator(device="cuda").manual_seed(h)
    x, dH, dr = (torch.randn(N, h, generator=g, device="cuda").to(t) for t in (dtype, F32, F32))
    w, stats = torch.rand(h, generator=g, device="cuda").to(dtype) + 0.5, torch.empty(4, N, device="cuda")
    vp.vp_block_norm_fwd(x, None, torch.empty_like(x), stats=stats, w=w, center=center)
    ws = torch.full((vp.vp_block_norm_bwd_workspace_bytes(N, h),), 0xFF, dtype=torch.uint8, device="cuda")
    out = {"dx": torch.empty(N, h, device="cuda"), "dw": torch.empty(h, device="cuda"), "db": torch.empty(h, device="cuda")}
    vp.vp_block_norm_bwd(dH, x, None, stats, dr=dr, w=w, center=center, workspace=ws, **out)
    for name, (value, bound) in ref.backward(dH, x, None, stats, dr=dr, w=w, center=center).items():
        ref.check(name, out[name], value, bound)
