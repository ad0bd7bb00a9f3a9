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
