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


def statistics_call():
    import paper_2411_05288_amd as vp
    f = torch.zeros
    vp.vp_logits_stats([f(4, 9)], f(4), f(4), torch.zeros(64, dtype=torch.uint8))


@pytest.mark.parametrize("status", [1, 2, 3, 4])
def test_statistics_status_is_an_exception_and_the_call_is_not_made_again(library, monkeypatch, status):
    import paper_2411_05288_amd as vp
    import paper_2411_05288_amd.binding as B
    statistics_call()
    assert [n for n, _ in library.calls] == ["vp_logits_stats"]
    library.status = status
    with pytest.raises(vp.VPError, match="vp_logits_stats failed: status %d" % status):
        statistics_call()
    library.calls.clear()
    monkeypatch.setitem(B._ADDRESS, "vp_logits_stats", 1)

    class Host:
        def logits_stats(self, *a):
            return status
    monkeypatch.setattr(B, "_HOST", Host())
    with pytest.raises(vp.VPError, match="vp_logits_stats failed: status %d" % status):
        statistics_call()
    assert library.calls == []
    library.status = 0
    Host.logits_stats = lambda self, *a: None      # a call that was not made is made with the checks in Python
    Host.__getattr__ = lambda self, name: lambda *a: None
    statistics_call()
    assert [n for n, _ in library.calls] == ["vp_logits_stats"]


class Kept:
    """What DraftVerifyPlan asks of a plan."""
    N, valid, offsets, workspace = 3, [4, 0, 2], [0, 4, 8], "the plan's"

    def __init__(self, logits=True):
        self.logits = [torch.zeros(3, 4), torch.zeros(3, 0), torch.zeros(3, 2)] if logits else None
        self.global_max, self.global_sumexp = torch.full((3,), 1.0), torch.full((3,), 2.0)


@pytest.mark.parametrize("model", [True, False])
def test_a_verification_takes_statistics_of_the_logits_it_reads(library, monkeypatch, model):
    """The plans' own statistics, of other values, are neither handed on nor written."""
    import copy

    import paper_2411_05288_amd as vp
    monkeypatch.setattr(Library, "vp_verify_workspace_bytes", lambda self, *a: 16, raising=False)
    monkeypatch.setattr(Library, "vp_logits_stats_workspace_bytes", lambda self, *a: 32, raising=False)
    plans = [Kept(), Kept()]
    verify = vp.DraftVerifyPlan(plans[0], torch.tensor([0, 3]), torch.zeros(3, dtype=torch.int64), torch.zeros(3),
                                draft=plans[1] if model else None)
    verify.forward()
    assert [n for n, _ in library.calls] == ["vp_logits_stats"] * (1 + model) + ["vp_verify_drafts"]
    *made, (_, call) = library.calls
    for (_, a), m, s in zip(made, (5, 8), (6, 9)):
        assert a[2] == 2 and a[4] == 3 and a[8] == 32 and a[5] == call[m] and a[6] == call[s]
    assert model or call[7] is call[8] is call[9] is None
    for p in plans:
        assert p.global_max.data_ptr() not in call and p.global_sumexp.data_ptr() not in call
        assert p.global_max.tolist() == [1.0] * 3 and p.global_sumexp.tolist() == [2.0] * 3
    assert verify.target.plan is plans[0] and verify.target.workspace == "the plan's" and verify.target.offsets == [0, 8]
    assert copy.copy(verify.target).plan is plans[0]
    with pytest.raises(AttributeError):
        verify.target.nothing
    with pytest.raises(vp.VPError):
        vp.DraftVerifyPlan(Kept(logits=False), torch.tensor([0, 3]), torch.zeros(3, dtype=torch.int64), torch.zeros(3))
