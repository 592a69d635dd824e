"""CPU test of a fresh AdamW state: its moments are zeros, its copies the parameters in the copies' type."""
import pytest

torch = pytest.importorskip("torch")

from tests.test_stream_memory_host import DeviceTensor  # noqa: E402


class Lists:
    """The extension's answers for host tensors."""
    @staticmethod
    def read(tensors, name, types, device, written, sizes, block):
        return len(tensors), 0, b"", b"", b"", sum(t.numel() for t in tensors)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_copies_of_a_fresh_state_are_the_parameters(monkeypatch, bits, dtype):
    import paper_2609_36830_amd as pace
    g = torch.Generator().manual_seed(1)
    params = [torch.randn(s, generator=g, requires_grad=r) for s, r in (((3, 100), False), ((257,), True), ((0,), False))]
    empty = torch.empty
    monkeypatch.setattr(pace._lib, "lists", lambda: Lists)
    monkeypatch.setattr(torch, "empty", lambda shape, dtype=None, device=None: empty(shape, dtype=dtype).fill_(7).as_subclass(DeviceTensor))
    state = pace.adamw_state(params, bits, dtype)
    for copy, p in zip(state["copies"], params):
        assert copy.dtype == dtype and torch.equal(copy, p.detach().to(dtype)) and not copy.requires_grad
    assert not any(t.any() for k in ("exp_avg", "exp_avg_sq") for t in state[k])
    assert bits == 32 or not any(t.any() for t in state["scale"])
