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
