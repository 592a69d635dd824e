"""CPU test of where the layer norm's, the gradients' norm's and AdamW's calls allocate: with `stream`, every output, state and
workspace that a call makes is that stream's memory."""
import contextlib

import pytest

torch = pytest.importorskip("torch")

from tests.test_stream_memory_host import Library, SideStream, T  # noqa: E402



def calls(pace):
    x, state = T((3, 8)), lambda: dict(bits=8, exp_avg=[T(5, torch.int8)], exp_avg_sq=[T(5, torch.uint8)], scale=[T((1, 2))], copies=None)
    return {
        "layer_norm": lambda **s: pace.pace_layer_norm(x, **s),
        "layer_norm_backward": lambda **s: pace.pace_layer_norm_backward(x, T((3, 2)), T((3, 8)), **s),
        "grad_norm": lambda **s: pace.pace_grad_norm([x], **s),
        "adamw_state": lambda **s: pace.adamw_state([x, T(300)], 8, torch.bfloat16, **s),
        "adamw_unpack": lambda **s: pace.pace_adamw_unpack(state(), **s),
    }


@pytest.mark.parametrize("name", sorted(calls(None)))
def test_a_call_allocates_in_its_streams_memory(monkeypatch, name):
    import paper_2609_36830_amd as pace
    inside, made = [], []
    empty = torch.empty

    @contextlib.contextmanager
    def under(stream):
        inside.append(stream)
        yield
        inside.pop()

    def record(shape, dtype=None, device=None):
        made.append(inside[-1] if inside else None)
        return empty(shape, dtype=dtype).as_subclass(type(T(1)))

    class Lists:
        """The extension's answers for host tensors."""
        @staticmethod
        def read(tensors, name, types, device, written, sizes, block):
            return len(tensors), 0, b"", b"", b"", sum(t.numel() for t in tensors)

        @staticmethod
        def apart(names, pointers):
            return None

        @staticmethod
        def matrix(t, name, types, device, rows, cols):
            return 0, 0, t.shape[0], t.shape[1], t.shape[1], 0

        @staticmethod
        def vector(t, name, types, device, n):
            return 0, 0, t.numel()

    monkeypatch.setattr(pace, "lib", Library)
    monkeypatch.setattr(pace._lib, "lists", lambda: Lists)
    monkeypatch.setattr(pace, "_stream", lambda device, stream=None: 0)
    monkeypatch.setattr(torch.cuda, "stream", under)
    monkeypatch.setattr(torch.cuda, "Stream", SideStream)
    monkeypatch.setattr(torch, "empty", record)
    call, side = calls(pace)[name], SideStream()
    call()
    assert made and not any(made)
    plain = len(made)
    call(stream=side)
    assert len(made) == 2 * plain and all(s is side for s in made[plain:])
