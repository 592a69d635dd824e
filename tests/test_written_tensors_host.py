"""CPU tests that torch learns of what AdamW writes through pointers: a tensor that a graph has saved is no longer used, silently,
with its new values."""
import pytest

torch = pytest.importorskip("torch")

from tests.test_stream_memory_host import T  # noqa: E402


class Lists:
    """The extension's answers for host tensors."""
    @staticmethod
    def read(tensors, name, types, device, written, sizes, block):
        return len(list(tensors)), 0, b"", b"", b"", 0

    @staticmethod
    def apart(names, lists):
        return None


@pytest.fixture
def pace(monkeypatch):
    import paper_2609_36830_amd as pace

    class Library:
        status = 0

        def __getattr__(self, name):
            return (lambda code: b"refused") if name == "pace_strerror" else (lambda *args: self.status)

    library = Library()
    monkeypatch.setattr(pace, "lib", lambda: library)
    monkeypatch.setattr(pace._lib, "lists", lambda: Lists)
    monkeypatch.setattr(pace, "_stream", lambda device, stream=None: 0)
    pace.status = lambda code: setattr(Library, "status", code)
    yield pace
    del pace.status


def state(bits, copies=True):
    m, v = (torch.float32,) * 2 if bits == 32 else (torch.int8, torch.uint8)
    return dict(bits=bits, exp_avg=[T(5, m), T(7, m)], exp_avg_sq=[T(5, v), T(7, v)], scale=[T((1, 2)), T((1, 2))] if bits == 8 else None,
                copies=[T(5, torch.bfloat16), T(7, torch.bfloat16)] if copies else None)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("copies", [False, True])
@pytest.mark.parametrize("kind", [list, tuple, iter])
def test_a_step_raises_the_versions_of_what_it_writes(pace, bits, copies, kind):
    params, grads, s = [T(5), T(7)], [T(5), T(7)], state(bits, copies)
    written = params + (s["copies"] or [])
    before = [t._version for t in written], [g._version for g in grads]
    pace.pace_adamw(kind(params), grads, s)
    assert [t._version for t in written] == [v + 1 for v in before[0]] and [g._version for g in grads] == before[1]


def test_a_refused_step_leaves_the_versions(pace):
    params, s = [T(5), T(7)], state(8)
    written = params + s["copies"]
    before = [t._version for t in written]
    pace.status(-1)
    with pytest.raises(pace.PaceError):
        pace.pace_adamw(params, [T(5), T(7)], s)
    pace.status(0)
    with pytest.raises(ValueError):
        pace.pace_adamw(params, [T(5), T(7)], s, weight_decay=[0.1])
    assert [t._version for t in written] == before


def test_a_saved_parameter_is_not_used_with_its_new_values(pace):
    params = [torch.ones(5, requires_grad=True), torch.ones(7, requires_grad=True)]
    loss = sum((p * p).sum() for p in params)
    pace.pace_adamw([p.detach() for p in params], [T(5), T(7)], state(32))
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()
    with torch.inference_mode():
        params = [torch.ones(5), torch.ones(7)]
    pace.pace_adamw(params, [T(5), T(7)], state(32))       # these have no versions
