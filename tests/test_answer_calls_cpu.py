"""What the Python calls that answer do before and after the library's function, on the host: a stub stands in for the library."""
import pytest
import torch


class Library:
    def __init__(self, status=0):
        self.calls, self.status = [], status

    def vp_status_string(self, status):
        return b"status %d" % status

    def vp_i8_row_stride(self, h):
        return (h + 127) // 128 * 128

    def __getattr__(self, name):
        def call(*args):
            self.calls.append((name, args))
            return self.status
        return call


@pytest.fixture
def library(monkeypatch):
    import paper_2411_05288_amd.binding as B
    lib = Library()
    monkeypatch.setattr(B, "load_library", lambda: lib)
    monkeypatch.setattr(B, "_HOST", None)
    monkeypatch.setattr(B, "_ptr", lambda t, *_: None if t is None else t.data_ptr())      # host tensors stand for the GPU's
    monkeypatch.setattr(B, "_on_current_device", lambda ts: None)
    monkeypatch.setattr(B, "_stream", lambda s: 0)
    monkeypatch.setattr(B, "_ADDRESS", dict.fromkeys(("vp_quantize_rows", "vp_output_fwd_i8_group", "vp_verify_drafts"), 1))
    return lib


def calls():
    import paper_2411_05288_amd as vp
    i8 = lambda *s: torch.zeros(*s, dtype=torch.int8)      # noqa: E731
    ids, f = torch.zeros(4, dtype=torch.int64), torch.zeros
    ws = torch.zeros(64, dtype=torch.uint8)
    return [
        ("vp_quantize_rows", lambda: vp.vp_quantize_rows(f(4, 100), i8(4, 128), f(4))),
        ("vp_output_fwd_i8_group", lambda: vp.vp_output_fwd_i8_group(i8(4, 128), f(4), [i8(9, 128)], [f(9)], ids, [0], f(1, 4), f(1, 4),
                                                                     f(1, 4), [f(4, 9)], ws)),
        ("vp_output_fwd_i8", lambda: vp.vp_output_fwd_i8(i8(4, 128), f(4), i8(9, 128), f(9), ids, 0, f(4), f(4), f(4), None, ws)),
        ("vp_verify_drafts", lambda: vp.vp_verify_drafts([f(4, 9)], [0], f(4), f(4), ids, torch.tensor([0, 4]), f(4),
                                                         torch.zeros(1, dtype=torch.int32), ids + 1, ws)),
    ]


@pytest.mark.parametrize("which", range(4))
def test_a_status_is_an_exception(library, which):
    import paper_2411_05288_amd as vp
    name, call = calls()[which]
    call()
    assert [n for n, _ in library.calls] == [name]
    library.status = 3
    with pytest.raises(vp.VPError, match="%s failed: status 3" % name):
        call()


@pytest.mark.parametrize("which", [0, 1, 3])
@pytest.mark.parametrize("status", [1, 2, 3, 4])
def test_a_call_that_failed_is_not_made_again(library, monkeypatch, which, status):
    import paper_2411_05288_amd as vp
    import paper_2411_05288_amd.binding as B

    class Host:
        def quantize_rows(self, *a):
            return status
        output_fwd_i8_group = verify_drafts = quantize_rows
    monkeypatch.setattr(B, "_HOST", Host())
    name, call = calls()[which]
    with pytest.raises(vp.VPError, match="%s failed: status %d" % (name, status)):
        call()
    assert library.calls == []


@pytest.mark.parametrize("which", [0, 1, 3])
def test_a_call_that_was_not_made_is_made_with_the_checks_in_python(library, monkeypatch, which):
    import paper_2411_05288_amd.binding as B

    class Host:
        def quantize_rows(self, *a):
            return None
        output_fwd_i8_group = verify_drafts = quantize_rows

        def __getattr__(self, name):
            return lambda *a: None
    monkeypatch.setattr(B, "_HOST", Host())
    name, call = calls()[which]
    call()
    assert [n for n, _ in library.calls] == [name]


def test_types_and_flags_of_the_logits(library):
    import paper_2411_05288_amd as vp
    i8, f = (lambda *s: torch.zeros(*s, dtype=torch.int8)), torch.zeros
    ids, ws = torch.zeros(4, dtype=torch.int64), torch.zeros(64, dtype=torch.uint8)
    for kept, dt, flags in ((None, vp.VP_BF16, 0), (f(4, 9), vp.VP_F32, 1), (f(4, 9, dtype=torch.bfloat16), vp.VP_BF16, 1)):
        vp.vp_output_fwd_i8_group(i8(4, 128), f(4), [i8(9, 128)], [f(9)], ids, [0], f(1, 4), f(1, 4), f(1, 4), None if kept is None else [kept], ws)
        vp.vp_output_fwd_i8(i8(4, 128), f(4), i8(9, 128), f(9), ids, 0, f(4), f(4), f(4), kept, ws)
        group, single = (args for _, args in library.calls[-2:])
        assert (group[10], group[11]) == (single[9], single[10]) == (dt, flags)
