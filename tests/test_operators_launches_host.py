"""CPU test of the rules that keep the operators' launches within a grid's range (csrc/rules.hpp, compiled for the
host): fewer than 2^32 threads in a dimension, whatever number of rows, channels or updates the calls accept."""
import ctypes
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SOURCE = """
#include "%s"
using namespace pace;
extern "C" {
int64_t backward_parts(int64_t rows, int64_t vocab) { return logprob_backward_parts(rows, vocab); }
int64_t batch_most(int64_t m, int64_t n) { return ortho_batch_most(m, n); }
// Launches of n workgroups, or -1 where they are not the n in order or one has too many threads.
int64_t launches(int64_t n, int64_t threads, int64_t fail_at) {
    int64_t k = 0, at = 0;
    const int e = in_launches(n, threads, [&](int64_t first, int64_t count) {
        if (first != at || count < 1 || count * threads >= ((int64_t)1 << 32)) at = -n - 1;
        at += count;
        return k++ == fail_at ? 7 : 0;
    });
    return e ? -e - 100 * k : (at == n ? k : -1);
}
}
""" % os.path.join(ROOT, "paper_2609_36830_amd", "csrc", "rules.hpp")


@pytest.fixture(scope="module")
def R(tmp_path_factory):
    d = tmp_path_factory.mktemp("rules")
    (d / "r.cpp").write_text(SOURCE)
    subprocess.check_call(["g++", "-O1", "-std=c++17", "-shared", "-fPIC", str(d / "r.cpp"), "-o", str(d / "r.so")])
    lib = ctypes.CDLL(str(d / "r.so"))
    for name in ("backward_parts", "batch_most", "launches"):
        getattr(lib, name).restype, getattr(lib, name).argtypes = ctypes.c_int64, [ctypes.c_int64] * (3 if name == "launches" else 2)
    return lib


def test_launches_hold_the_grid(R):
    for threads in (64, 256, 512):
        most = (2 ** 32 - 1) // threads
        for n in (1, 2, most - 1, most, most + 1, 2 * most, 2 * most + 1, 2 ** 31):
            assert R.launches(n, threads, -1) == -(-n // most)
    assert R.launches(2 ** 31, 512, 1) == -7 - 200        # the second fails: no third


def test_backward_parts(R):
    for rows in (1, 4096, 2 ** 20, 2 ** 24 - 1, 2 ** 24, 2 ** 31 - 2):
        for vocab in (1, 16384, 16385, 150000, 2 ** 31 - 2):
            p = R.backward_parts(rows, vocab)
            assert 1 <= p <= -(-vocab // 16384)
            assert p == 1 or rows * p * 256 < 2 ** 32      # only whole rows go in several launches
    assert R.backward_parts(4096, 150000) == 10


def test_batches_of_updates(R):
    for m, n in ((1, 1), (1, 2 ** 21), (64, 2 ** 21), (4096, 16384), (2 ** 21, 2 ** 21)):
        b = R.batch_most(m, n)
        tiles = -(-m // 64) * -(-n // 64)
        assert b >= 1 and (b == 1 or b * tiles * 512 < 2 ** 32)
    assert R.batch_most(1, 2 ** 21) == 255 and R.batch_most(256, 1024) > 65535
