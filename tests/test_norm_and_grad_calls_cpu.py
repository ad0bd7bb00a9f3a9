"""What the Python calls of the norms around a block and of the calls over many gradients do before and after the library's
function, on the host: a stub stands in for the library."""
import pytest
import torch

DEVICE = 4      # VP_ERR_DEVICE


class Library:
    """Counts the calls of its functions; every one succeeds."""

    def __init__(self):
        self.calls = []

    def vp_status_string(self, status):
        return b"status %d" % status

    def __getattr__(self, name):
        def call(*args):
            self.calls.append((name, args))
            return 0
        return call


@pytest.fixture
def library(monkeypatch):
    import paper_2411_05288_amd.binding as B
    lib = Library()
    monkeypatch.setattr(B, "load_library", lambda: lib)
    monkeypatch.setattr(B, "_ptr", lambda t, *_: None if t is None else t.data_ptr())      # host tensors stand for the GPU's
    monkeypatch.setattr(B, "_on_current_device", lambda ts: None)
    monkeypatch.setattr(B, "_stream", lambda s: 0)
    monkeypatch.setattr(B, "_ADDRESS", {"vp_block_norm_fwd": 1, "vp_block_norm_bwd": 2})
    return lib


@pytest.mark.parametrize("status", [1, 2, 3, DEVICE])
def test_a_norm_call_that_failed_is_not_made_again(library, monkeypatch, status):
    """A device error may come after the kernels were launched: in place, a second call would work on what the first left."""
    import paper_2411_05288_amd as vp
    import paper_2411_05288_amd.binding as B

    class Host:
        def block_norm_fwd(self, *a):
            return status
        block_norm_bwd = block_norm_fwd
    monkeypatch.setattr(B, "_HOST", Host())
    x, y, stats = torch.zeros(4, 8), torch.zeros(4, 8), torch.zeros(4, 4)
    with pytest.raises(vp.VPError, match="vp_block_norm_fwd failed: status %d" % status):
        vp.vp_block_norm_fwd(x, y, y, r=x, stats=stats)
    with pytest.raises(vp.VPError, match="vp_block_norm_bwd failed: status %d" % status):
        vp.vp_block_norm_bwd(x, x, None, stats, dx=y, workspace=torch.zeros(1 << 16, dtype=torch.uint8))
    assert library.calls == []


def test_a_norm_call_that_was_not_made_is_made_with_the_checks_in_python(library, monkeypatch):
    import paper_2411_05288_amd as vp
    import paper_2411_05288_amd.binding as B

    class Host:
        def block_norm_fwd(self, *a):
            return None
        block_norm_bwd = block_norm_fwd
    monkeypatch.setattr(B, "_HOST", Host())
    x, y, stats = torch.zeros(4, 8), torch.zeros(4, 8), torch.zeros(4, 4)
    vp.vp_block_norm_fwd(x, None, y, stats=stats)
    vp.vp_block_norm_bwd(x, x, None, stats, dx=y, workspace=torch.zeros(1 << 16, dtype=torch.uint8))
    assert [name for name, _ in library.calls] == ["vp_block_norm_fwd", "vp_block_norm_bwd"]


def changes():
    """(name, what a program may do to a tensor of 100 fp32 elements that the arguments of a call were made of)"""
    def moved(t):
        t.data = t.data.clone()

    def shorter(t):      # the same address: the old number of elements would reach into what lies behind
        t.data = t.data[:50]

    def longer(t):
        t.data = t.data.as_strided((120,), (1,))

    def resized(t):
        t.resize_(99)

    def other_type(t):
        t.data = t.data.view(torch.bfloat16)[:100]

    def strided(t):
        t.data = t.data.view(10, 10).t()

    def freed(t):
        t.untyped_storage().resize_(0)
    return [moved, shorter, longer, resized, other_type, strided, freed]


@pytest.mark.parametrize("native", [True, False])
@pytest.mark.parametrize("change", changes(), ids=lambda f: f.__name__)
@pytest.mark.parametrize("of_outs", [False, True])
def test_tensors_that_changed_are_not_written(library, monkeypatch, native, change, of_outs):
    """The arguments hold addresses and numbers of elements: what no longer fits them is refused before anything is called."""
    import paper_2411_05288_amd as vp
    import paper_2411_05288_amd.binding as B
    host = B._load_host(B.host_path()) if native else None
    if native and host is None:
        pytest.skip("_vphost.so is not built for this PyTorch")
    monkeypatch.setattr(B, "_HOST", host)
    ws, norm = torch.zeros(1 << 16, dtype=torch.uint8), torch.zeros(1)
    grads = [torch.zeros(300), torch.zeros(400)[:100], torch.zeros(0)]
    outs = [torch.zeros(300), torch.zeros(400)[:100], torch.zeros(0)]
    plan = vp.GradientClipPlan(grads, outs, norm=norm, workspace=ws)
    calls = [plan.compute_norm, lambda: plan.clip(1.0), lambda: plan.scale(1.0)]
    for call in calls:
        call()
    assert plan.covers(grads) and [name for name, _ in library.calls] == ["vp_grad_norm", "vp_grad_clip", "vp_grad_scale"]
    library.calls.clear()
    change((outs if of_outs else grads)[1])
    assert not plan.covers(grads)
    for call in calls[1 if of_outs else 0:]:
        with pytest.raises(vp.VPError, match="since the arguments were made"):
            call()
    assert library.calls == []
    vp.GradientClipPlan(grads[:1], outs[:1], norm=norm, workspace=ws).clip(1.0)      # the others are as they were
    assert len(library.calls) == 1


@pytest.mark.parametrize("change", changes()[:3], ids=lambda f: f.__name__)
def test_clip_gradients_of_a_changed_tensor(library, monkeypatch, change):
    """The kept list of gradients is made anew for a gradient that is another one at the same address."""
    import paper_2411_05288_amd as vp
    W, other = [torch.zeros(16, 8)], torch.zeros(400)[:100]
    monkeypatch.setattr(vp.OutputLayerPlan, "__init__", lambda self: None)
    plan = vp.OutputLayerPlan()
    plan.dW, plan.norm, plan.dH = W, None, torch.zeros(4, 8)
    plan.clip_plan, plan.clip_norm, plan.clip_workspaces = None, None, []
    monkeypatch.setattr("paper_2411_05288_amd.binding.vp_grad_workspace_bytes", lambda n: 1 << 16)
    plan.clip_gradients(1.0, [other])
    change(other)
    plan.clip_gradients(1.0, [other])
    counts = [list(args[1]) for _, args in library.calls]
    assert counts == [[128, 100], [128, other.numel()]]
    assert library.calls[1][1][0][1] == other.data_ptr()


@pytest.fixture(scope="module")
def real():
    import paper_2411_05288_amd as vp
    return vp.load_library()


def refused(real, name, grads, outs, norm, ws, n_bytes=1 << 14):
    """Whether the library refuses a call with these (address, fp32 elements) lists; the addresses are none, so one that it does
    not refuse ends with a device error where there is no GPU."""
    import ctypes
    n = len(grads)
    a = [(ctypes.c_void_p * n)(*[p for p, _ in grads]), (ctypes.c_int64 * n)(*[c for _, c in grads]), (ctypes.c_int32 * n)(), n]
    if name != "vp_grad_norm":
        a += [None if outs is None else (ctypes.c_void_p * n)(*outs), 1.0]
    return getattr(real, name)(*a, norm, ws, n_bytes, None) == 1      # VP_ERR_INVALID_ARG


NAMES = ("vp_grad_norm", "vp_grad_clip", "vp_grad_scale")
A, G, O, W = 0x100000, 0x200000, 0x300000, 0x400000      # addresses apart from one another


@pytest.mark.skipif(torch.cuda.is_available(), reason="the addresses are none")
@pytest.mark.parametrize("name", NAMES)
def test_the_norm_and_the_workspace_are_apart_from_the_gradients(real, name):
    """They are written while gradients are read (the norm is read by vp_grad_scale while they are written)."""
    for at in (G, G + 4, G + 396):
        assert refused(real, name, [(A, 10), (G, 100)], None, at, W)
    size = real.vp_grad_workspace_bytes(2)
    for at in (G, G + 384, G - size + 16, G - size + 1024):
        assert refused(real, name, [(A, 10), (G, 100)], None, O, at)
    for at in (W, W + size - 4):
        assert refused(real, name, [(A, 10), (G, 100)], None, at, W)
    assert refused(real, name, [(A, 0), (G, 1)], None, G, W)
    if name != "vp_grad_norm":
        assert refused(real, name, [(A, 10), (G, 100)], [A, O], O + 396, W)
        assert refused(real, name, [(A, 10), (G, 100)], [A, O], A, W)
        for at in (O, O + 384, O - size + 16):
            assert refused(real, name, [(A, 10), (G, 100)], [A, O], A + 64, at)


@pytest.mark.skipif(torch.cuda.is_available(), reason="the addresses are none")
@pytest.mark.parametrize("name", NAMES)
def test_a_norm_and_a_workspace_beside_the_gradients_are_taken(real, name):
    size = real.vp_grad_workspace_bytes(2)
    for norm, ws in ((G - 4, W), (G + 400, W), (W - 4, W), (W + size, W), (A, G + 400), (O, G - size), (G, W)):
        assert not refused(real, name, [(O + 64, 10), (G, 0 if norm == G else 100)], None, norm, ws, n_bytes=size)
    # what lies behind the bytes that the call needs is not its workspace
    assert not refused(real, name, [(O, 10), (W + size, 100)], None, A, W)
    if name == "vp_grad_scale":      # two inputs
        assert not refused(real, name, [(A, 10), (G, 100)], [O, O + 4096], G, W)
    assert not refused(real, name, [(A, 10), (G, 100)], [A, G], O, W)


# Buffers of a call of N=8 h=16 bf16, apart from one another; gradients of activations are fp32.
N, H_ = 8, 16
BYTES = dict(x=256, y=256, r=256, H=256, stats=128, gate=64, w=32, b=32, w_post=32, b_post=32, dH=256, dr=512, dx=512, dy=512, dgate=128,
             dw=64, db=64, dw_post=64, db_post=64)
AT = {k: 0x100000 * (i + 1) for i, k in enumerate(BYTES)}
FWD_IN, FWD_OUT = ("x", "y", "gate", "w_post", "b_post", "w", "b"), ("r", "H", "stats")
BWD_IN = ("dH", "dr", "r", "y", "gate", "w_post", "b_post", "w", "stats")
BWD_OUT = ("dx", "dy", "dgate", "dw_post", "db_post", "dw", "db", "ws")
W_BYTES = 1 << 20


def norm_call(real, forward, **at):
    """Status of a call with everything, with the buffers of `at` elsewhere (None: not given)."""
    p = {**AT, "ws": W << 8, **at}
    rows = 2 if p["gate"] else 0
    if forward:
        return real.vp_block_norm_fwd(p["x"], p["y"], p["gate"], rows, p["w_post"], p["b_post"], p["w"], p["b"], N, H_, 1, 24 if p["y"] else 16, 1.0,
                                      1e-5, p["r"], p["H"], p["stats"], None)
    return real.vp_block_norm_bwd(p["dH"], 1, p["dr"], p["r"], p["y"], p["gate"], rows, p["w_post"], p["b_post"], p["w"], p["stats"], N, H_, 1,
                                  24 if p["y"] else 16, 1.0, 0, p["dx"], p["dy"], p["dgate"], p["dw_post"], p["db_post"], p["dw"], p["db"],
                                  p["ws"], W_BYTES, None)


def beside(other, name, size):
    """Places of a buffer that share memory with another one: its first and last 16 bytes, and all of it."""
    return (AT[other], AT[other] + BYTES[other] - 16, AT[other] - size(name) + 16)


@pytest.mark.skipif(torch.cuda.is_available(), reason="the addresses are none")
@pytest.mark.parametrize("forward", [True, False])
def test_outputs_of_the_norms_are_apart(real, forward):
    ins, outs = (FWD_IN, FWD_OUT) if forward else (BWD_IN, BWD_OUT)
    need = real.vp_block_norm_bwd_workspace_bytes(N, H_, 2, 24)

    def size(k):
        return BYTES.get(k, need)
    in_place = {("r", "x"), ("H", "y")} if forward else {("dx", "dr")}
    assert norm_call(real, forward) != 1
    for out in outs:
        for other in ins + tuple(o for o in outs if o != out and o != "ws"):
            for at in beside(other, out, size):
                ok = (out, other) in in_place and at == AT[other]
                assert (norm_call(real, forward, **{out: at}) == 1) != ok, (out, other, hex(at))
    if forward:
        assert norm_call(real, True, r=AT["x"], H=AT["y"]) != 1
        assert norm_call(real, True, r=AT["x"], y=AT["x"]) == 1 and norm_call(real, True, x=AT["y"], H=AT["y"]) == 1
        assert norm_call(real, True, y=AT["x"]) != 1      # two inputs
        alone = dict(y=None, gate=None, r=None, w_post=None, b_post=None)
        assert norm_call(real, True, H=AT["x"], **{**alone, "y": None}) != 1
        assert norm_call(real, True, H=AT["x"] + 16, **alone) == 1
        assert norm_call(real, True, r=None, H=AT["r"]) != 1 and norm_call(real, True, stats=None, H=AT["stats"]) != 1
    else:
        assert norm_call(real, False, dr=None, dx=AT["dr"]) != 1 and norm_call(real, False, dr=AT["dH"]) != 1
        assert norm_call(real, False, dx=AT["dr"], dH=AT["dr"]) == 1
        assert norm_call(real, False, ws=AT["dx"] - need) != 1 and norm_call(real, False, ws=AT["dx"] + BYTES["dx"]) != 1


def test_a_gate_without_rows_is_refused(library, monkeypatch):
    """It has no address, and would be taken for no gate at all."""
    import paper_2411_05288_amd as vp
    import paper_2411_05288_amd.binding as B
    monkeypatch.setattr(B, "_HOST", None)
    x, y, H, stats, gate = torch.zeros(4, 8), torch.zeros(4, 8), torch.zeros(4, 8), torch.zeros(4, 4), torch.zeros(0, 8)
    with pytest.raises(vp.VPError, match="gate must be"):
        vp.vp_block_norm_fwd(x, y, H, gate=gate)
    with pytest.raises(vp.VPError, match="gate must be"):
        vp.vp_block_norm_bwd(x, x, y, stats, dx=H, dy=torch.zeros(4, 8), gate=gate, workspace=torch.zeros(1 << 16, dtype=torch.uint8))
    assert library.calls == []


def test_a_library_that_cannot_be_loaded_says_so_every_time(monkeypatch, tmp_path):
    """After a load that failed, a call tries again: it does not look for the functions of a library that is not there."""
    import paper_2411_05288_amd as vp
    import paper_2411_05288_amd.binding as B
    broken = tmp_path / "libvp.so"
    broken.write_text("no library")
    for name, value in (("_LIB", None), ("_HOST", None), ("_ADDRESS", {}), ("lib_path", lambda: str(broken)), ("_on_current_device", lambda ts: None)):
        monkeypatch.setattr(B, name, value)
    x, y, stats, ws = torch.zeros(4, 8), torch.zeros(4, 8), torch.zeros(4, 4), torch.zeros(1 << 16, dtype=torch.uint8)
    for _ in range(2):
        with pytest.raises(OSError):
            B.load_library()
        with pytest.raises(OSError):
            vp.vp_block_norm_fwd(x, None, y)
        monkeypatch.setattr(B, "_ptr", lambda t, *_: None if t is None else t.data_ptr())
        with pytest.raises(OSError):
            vp.vp_block_norm_bwd(x, x, None, stats, dx=y, workspace=ws)
