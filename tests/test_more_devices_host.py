"""CPU test of tensors on another device than the current one: the library is called with the tensors' device current, and the
one that was current is so again afterwards."""
import contextlib

import pytest

torch = pytest.importorskip("torch")

from tests.test_more_stream_memory_host import T, calls  # noqa: E402

STATE = dict(bits=32, exp_avg=[T(5)], exp_avg_sq=[T(5)], scale=None, copies=None)
CALLS = sorted(set(calls(None)) - {"adamw_state"}) + ["adamw"]


@pytest.mark.parametrize("current", [0, 1])
@pytest.mark.parametrize("fails", [False, True])
@pytest.mark.parametrize("name", CALLS)
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

    class Lists:
        """The extension's answers for tensors on the second of two devices."""
        @staticmethod
        def read(tensors, name, types, device, written, sizes, block):
            return len(tensors), 1, b"", b"", b"", sum(t.numel() for t in tensors)

        @staticmethod
        def apart(names, pointers):
            return None

        @staticmethod
        def matrix(t, name, types, device, rows, cols):
            return 0, 0, t.shape[0], t.shape[1], t.shape[1], 1

        @staticmethod
        def vector(t, name, types, device, n):
            return 0, 0, t.numel()

    @contextlib.contextmanager
    def device(d):
        before, at[0] = at[0], d
        switches.append(d)
        try:
            yield
        finally:
            at[0] = before

    empty = torch.empty
    monkeypatch.setattr(pace, "lib", Library)
    monkeypatch.setattr(pace._lib, "lists", lambda: Lists)
    monkeypatch.setattr(pace, "_stream", lambda device, stream=None: 0)
    monkeypatch.setattr(torch.cuda, "is_initialized", lambda: True)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: at[0])
    monkeypatch.setattr(torch.cuda, "device", device)
    monkeypatch.setattr(torch, "empty", lambda shape, dtype=None, device=None: empty(shape, dtype=dtype).as_subclass(type(T(1))))
    call = {**calls(pace), "adamw": lambda: pace.pace_adamw([T(5)], [T(5)], STATE)}[name]
    with pytest.raises(KeyError) if fails else contextlib.nullcontext():
        call()
    assert seen == [1] and at == [current] and switches == ([] if current == 1 else [1])
