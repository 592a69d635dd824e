"""CPU test of the filter's and the operators' calls on tensors of another device than the current one: the library is called
with the tensors' device current, whose default stream the null handle is then, and the one that was current is so again
afterwards."""
import contextlib

import pytest

torch = pytest.importorskip("torch")

from tests import test_stream_memory_host as plain  # noqa: E402


class Second(plain.DeviceTensor):
    """A host tensor that passes for one on the second of two devices."""
    device = property(lambda self: torch.device("cuda", 1))


def all_calls(pace):
    tags, off, comp = (plain.T(n, t) for n, t in ((10, torch.int32), (4, torch.int64), (3, torch.int32)))
    step = lambda: pace.FilterStep(3, 10, [torch.int32], "cuda:1", params=object())
    return {
        **plain.calls(pace),
        "filter_step_noalloc": lambda: pace.pace_filter_step_noalloc(tags, off, comp, 1, 3, 2, [tags]),
        "kept_buffers": lambda: step().run(tags, off, comp, 1, 3, 2, [tags]),
        "kept_buffers_score": lambda: step().score_only(tags, off, comp, 1),
    }


@pytest.mark.parametrize("current", [0, 1])
@pytest.mark.parametrize("fails", [False, True])
@pytest.mark.parametrize("name", sorted(all_calls(None)))
def test_a_call_runs_on_its_tensors_device(monkeypatch, name, current, fails):
    import paper_2609_36830_amd as pace
    at, seen, switches = [current], [], []

    class Library:
        def __getattr__(self, entry):
            def call(*args):
                if entry.endswith("workspace_bytes"):
                    return 0
                seen.append(at[0])
                if fails:
                    raise KeyError(entry)
                return 0
            return call

    @contextlib.contextmanager
    def device(d):
        before, at[0] = at[0], d
        switches.append(d)
        try:
            yield
        finally:
            at[0] = before

    empty = torch.empty
    monkeypatch.setattr(plain, "T", lambda shape, dtype=torch.float32: torch.zeros(shape, dtype=dtype).as_subclass(Second))
    monkeypatch.setattr(pace, "lib", Library)
    monkeypatch.setattr(pace.ctypes, "byref", lambda x: x)
    monkeypatch.setattr(pace, "_stream", lambda device, stream=None: 0)
    monkeypatch.setattr(torch.cuda, "is_initialized", lambda: True)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: at[0])
    monkeypatch.setattr(torch.cuda, "device", device)
    monkeypatch.setattr(torch, "empty", lambda shape, dtype=None, device=None: empty(shape, dtype=dtype).as_subclass(Second))
    call = all_calls(pace)[name]
    with pytest.raises(KeyError) if fails else contextlib.nullcontext():
        call()
    assert seen == [1] and at == [current] and switches == ([] if current == 1 else [1])


def test_every_entry_point_with_a_stream_is_called():
    """By this test or the one of the layer norm, the gradients' norm and AdamW."""
    from paper_2609_36830_amd import _lib
    from tests import test_more_devices_host as more
    host = {"pace_default_params", "pace_budget", "pace_time_next_kernel", "pace_strerror"}
    on_streams = {name for name, *_ in _lib.SIGNATURES if not name.endswith("workspace_bytes")} - host
    assert on_streams <= {"pace_" + n for n in list(all_calls(None)) + list(more.CALLS)}
