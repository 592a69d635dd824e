"""CPU tests that the GPU tests' shapes reach every form of the operators' kernels, by the library's own rules."""


def test_logprob_by_workgroups():
    """Eight waves a row, whole and in parts, each in several rounds of 4 vectors of 16 bytes a thread."""
    from tests.operator_rules import rules
    from tests.test_gpu_logprob_workgroups import PARTS, WHOLE
    R = rules()
    for shapes, whole in ((WHOLE, True), (PARTS, False)):
        for n, vocab, k in shapes:
            parts, waves = R.parts(n, vocab, k), R.waves(n, vocab, k)
            assert (waves, parts == 1) == (8, whole), (n, vocab, k, waves, parts)
        for size in (2, 4):
            most = max(v // (16 // size) / R.parts(n, v, k) / (4 * 512) for n, v, k in shapes)
            assert most > 2, most
    assert {k > 0 for _, _, k in WHOLE} == {k > 0 for _, _, k in PARTS} == {True, False}


def test_largest_tiles_of_the_updates_products():
    """With test_gpu_orthogonalize.py's shapes, each of the three products goes in each of the four tiles."""
    from tests.operator_rules import CUS, rules
    from tests.test_gpu_orthogonalize import TILES
    from tests.test_gpu_orthogonalize_tiles import LARGEST
    R = rules()
    gram, square, apply = set(), set(), set()
    for b, r, c in TILES + LARGEST:
        m, n = min(r, c), max(r, c)
        gram.add(R.lower(m, b, -(-n // 64), CUS))
        square.add(R.lower(m, b, -(-m // 64), CUS))
        apply.add(R.full(m, n, b, -(-m // 64), CUS))
    assert gram == square == apply == {64, 128, 192, 256}
