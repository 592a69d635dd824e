"""CPU tests of lists of tensors that share memory: refused whichever tensors they are, in whole or in part, before any call."""
import array
import os
import random

import pytest

torch = pytest.importorskip("torch")

WIDTH = (4, 2, 2, 1, 1, 8)


@pytest.fixture(scope="module")
def apart():
    from paper_2609_36830_amd import _lib
    if not os.path.exists(_lib.lists_path):
        from paper_2609_36830_amd import build
        build.build()
    return _lib.lists().apart


def read(*tensors):
    """A list as the extension reads it: tensors are (address, code of the type, elements)."""
    of = lambda kind, at: array.array(kind, [t[at] for t in tensors]).tobytes()
    return len(tensors), 0, of("Q", 0), of("i", 1), of("q", 2), sum(t[2] for t in tensors)


@pytest.mark.parametrize("lists", [
    (read((1000, 0, 10), (2000, 0, 10)), read((2000, 0, 10), (1000, 0, 10))),                  # in another order
    (read((1000, 0, 10)), read((1036, 0, 10))),                                                # shifted, the last element
    (read((1000, 1, 10)), read((1018, 4, 1))),
    (read((1000, 0, 10), (5000, 0, 1)), read((0, 0, 0), (900, 3, 101))),
    (read((1000, 0, 1000)), read((1100, 1, 3))),                                               # within
    (read((1100, 1, 3)), read((1000, 0, 1000))),
    (read((1000, 5, 4)), read((1024, 0, 2))),
    (read((9000, 0, 5), (1000, 0, 5), (5000, 0, 5)), read((7000, 0, 5), (1019, 4, 1), (3000, 0, 5))),
])
def test_tensors_of_two_lists_overlap(apart, lists):
    a, b = lists
    other = read((50000, 0, 100), (60000, 0, 100))
    for names, given in ((("a", "b"), (a, b)), (("x", "a", "y", "b"), (other, a, None, b)), (("a", "b", "x"), (a, b, other))):
        with pytest.raises(ValueError, match="a and b must not overlap each other"):
            apart(names, given)


def test_tensors_that_only_touch(apart):
    assert apart(("a", "b", "c"), (read((1000, 0, 10), (1040, 0, 10)), read((1080, 1, 5), (996, 0, 1)), read((1090, 3, 7)))) is None
    assert apart(("a", "b"), (read((1000, 0, 0)), read((1000, 0, 10)))) is None                 # an empty one has no place
    assert apart(("a", "b"), (read((1000, 0, 10), (1000, 0, 10)), read((2000, 0, 10)))) is None  # gradients may be one tensor
    assert apart((), ()) is None and apart(("a", "b"), (None, None)) is None and apart(("a",), (read(),)) is None
    for bad in ((1, 2), read((1, 0, 1))[:5], (1, 0, b"", b"", 3, 0), (1, 0, b"12345678", b"", b"", 0), read((1000, 6, 1)), read((1000, 0, -1)), 3):
        with pytest.raises(ValueError):
            apart(("a", "b"), (read((10, 0, 1)), bad))


def test_against_every_byte(apart):
    rng = random.Random(1)
    seen = [0, 0]
    for _ in range(3000):
        lists = [[(rng.randint(0, 2500), rng.randint(0, 5), rng.choice([0, 1, 2, rng.randint(0, 30)])) for _ in range(rng.randint(0, 6))]
                 for _ in range(rng.randint(1, 6))]
        taken, want = {}, False
        for k, ts in enumerate(lists):
            for p, code, n in ts:
                for byte in range(p, p + n * WIDTH[code]):
                    want |= taken.setdefault(byte, k) != k
        names = tuple("abcdef"[: len(lists)])
        seen[want] += 1
        if want:
            with pytest.raises(ValueError, match="must not overlap each other"):
                apart(names, tuple(read(*ts) for ts in lists))
        else:
            assert apart(names, tuple(read(*ts) for ts in lists)) is None
    assert min(seen) > 500


def test_the_binding_gives_every_list(monkeypatch):
    """The step and the unpacking hand over what was read of each of their lists."""
    import paper_2609_36830_amd as pace
    from tests.test_stream_memory_host import Library, T
    given = []

    class Lists:
        @staticmethod
        def read(tensors, name, types, device, written, sizes, block):
            return len(tensors), 0, b"", b"", b"", name

        @staticmethod
        def apart(names, lists):
            given.append([(n, list and list[5]) for n, list in zip(names, lists)])

    monkeypatch.setattr(pace, "lib", Library)
    monkeypatch.setattr(pace._lib, "lists", lambda: Lists)
    monkeypatch.setattr(pace, "_stream", lambda device, stream=None: 0)
    state = dict(bits=8, exp_avg=[T(5, torch.int8)], exp_avg_sq=[T(5, torch.uint8)], scale=[T((1, 2))], copies=[T(5, torch.bfloat16)])
    pace.pace_adamw([T(5)], [T(5)], state)
    pace.pace_adamw([T(5)], [T(5)], dict(state, bits=32, copies=None))
    pace.pace_adamw_unpack(state, out=([T(5)], [T(5)]))
    names = ("params", "grads", "exp_avg", "exp_avg_sq", "scale", "copies")
    assert given[0] == [(n, n) for n in names]
    assert given[1] == [(n, n) for n in names[:4]] + [("scale", None), ("copies", None)]
    assert given[2] == [(n, n) for n in names[2:5]] + [("out[0]", "out"), ("out[1]", "out")]
