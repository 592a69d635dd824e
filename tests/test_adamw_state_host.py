"""CPU tests of a fresh AdamW state, its moments zeros and its copies the parameters in the copies' type, and of what moments
in 8 bits hold over many steps."""
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


@pytest.mark.parametrize("beta2, code, share", [(0.9, 19, 0.006), (0.95, 39, 0.023), (0.98, 99, 0.151), (0.99, 199, 0.61), (0.9921, 252, 0.98),
                                                (0.9922, 255, 1.0), (0.999, 255, 1.0)])
def test_second_moments_that_stay(beta2, code, share):
    """The largest code that a shrinking v keeps while its block's largest stays, and what its root is of the largest root."""
    stays = [c for c in range(1, 256) if round(255 * (beta2 * (c / 255) ** 4) ** 0.25) == c]
    assert stays == list(range(1, code + 1)) and abs((code / 255) ** 2 - share) < 0.006


@pytest.mark.parametrize("beta2, low, high", [(0.9, 0.93, 1.07), (0.95, 0.93, 1.07), (0.98, 0.9, 1.1), (0.99, 0.9, 1.16), (0.999, 8.0, 10.0)])
def test_second_moments_after_gradients_fell(beta2, low, high):
    """Half of a block's random gradients fall to a tenth: their roots beside those held in 64 bits, 5000 steps later."""
    import numpy as np
    r = np.random.default_rng(0)
    scale, codes, ref, half = 0.0, np.zeros(256), np.zeros(256), np.arange(256) < 128
    for t in range(7000):
        g = r.standard_normal(256)
        g = np.where(half, g / 10, g) if t >= 2000 else g
        v = beta2 * ((codes / 255) ** 4 * scale) + (1 - beta2) * g * g
        codes = np.rint(255 * np.sqrt(np.sqrt(v / v.max())))
        codes, scale = np.where((v > 0) & (codes < 1), 1, codes), float(np.float32(v.max()))
        ref = beta2 * ref + (1 - beta2) * g * g
    root = (codes / 255) ** 2 * scale ** 0.5 / np.sqrt(ref)
    assert low < np.percentile(root[half], 5) and np.percentile(root[half], 95) < high
