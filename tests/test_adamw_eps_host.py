"""CPU test of the least eps that pace_adamw takes with moments in 8 bits (the refusals return before any launch, and nothing
is launched for empty tensors)."""
import ctypes
import math
import os

import pytest


@pytest.fixture(scope="module")
def L():
    from paper_2609_36830_amd import _lib
    if not os.path.exists(_lib.library_path):
        from paper_2609_36830_amd import build
        build.build()
    return _lib.lib()


def call(L, bits, beta2, eps, schedule=None):
    from paper_2609_36830_amd._lib import AdamwParams
    sizes, types, none = (ctypes.c_int64 * 1)(0), (ctypes.c_int32 * 1)(0), (ctypes.c_void_p * 1)(None)
    hyper = AdamwParams(1e-3, 0.9, beta2, eps, 1)
    return L.pace_adamw(1, sizes, none, types, none, types, bits, none, none, none, None, None, None, ctypes.byref(hyper), None, schedule, None)


@pytest.mark.parametrize("schedule", [None, 0x1000])
@pytest.mark.parametrize("beta2", [0.0, 0.5, 0.9, 0.95, 0.99, 0.999, 0.999999, 1 - 2.0 ** -53])
def test_eps_that_a_lost_second_moment_would_outweigh(L, beta2, schedule):
    least = 2.0 ** -55 / math.sqrt(1 - beta2)
    assert least < 1e-8                              # the binding's default does with every beta2
    for eps in (1e-30, least / 2, least * (1 - 1e-12)):
        assert call(L, 8, beta2, eps, schedule) == -1, (beta2, eps)
    for eps in (least * (1 + 1e-12), 2 * least, 1e-8, 1.0):
        assert call(L, 8, beta2, eps, schedule) == 0, (beta2, eps)
    assert call(L, 32, beta2, 1e-30, schedule) == 0


def test_what_a_lost_second_moment_changes():
    """The definition in 64 bits beside one whose second moment counts as zero below 2^-126: at the least eps the steps are
    within a 256th of each other, whatever the gradients' size and however long it lasts; far below it they are not."""
    def steps(gs, beta2, eps, lost):
        m = v = 0.0
        got = []
        for t, g in enumerate(gs, 1):
            m, v = 0.9 * m + (1 - 0.9) * g, beta2 * v + (1 - beta2) * g * g
            got.append(m / (1 - 0.9 ** t) / (math.sqrt(v / -math.expm1(t * math.log(beta2))) + eps))
            if lost and v < 2.0 ** -126:
                v = 0.0
        return got

    for beta2 in (0.9, 0.95, 0.99, 0.999, 0.9999):
        least = 2.0 ** -55 / math.sqrt(1 - beta2)
        for k in range(-90, -10):
            g = 2.0 ** k
            for gs in ([g, 0.0, 0.0], [g] * 300, [g, g / 8] * 100, [g * 2.0 ** -j for j in range(40)], [g * 2.0 ** (j / 4) for j in range(100)]):
                for a, b in zip(steps(gs, beta2, least, True), steps(gs, beta2, least, False)):
                    assert abs(a - b) <= 2.0 ** -8 * abs(b) * (1 + 1e-9) + 1e-300, (beta2, k)
    assert steps([1e-18, 0.0], 0.999, 1e-30, True)[1] > 1e11 * steps([1e-18, 0.0], 0.999, 1e-30, False)[1]
