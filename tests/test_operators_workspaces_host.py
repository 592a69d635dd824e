"""CPU tests of the operators' workspace sizes: what a query gives for a size does for every smaller problem, and a call
asks for no more than that (csrc/rules.hpp, compiled for the host)."""
import ctypes
import os
import random
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SOURCE = """
#include "%s"
using namespace pace;
extern "C" {
int64_t span(int64_t nt) { return policy_loss_span(nt); }
int64_t spans_most(int64_t nt) { return policy_loss_spans_most(nt); }
int64_t parts(int64_t steps, int64_t tiles) { return product_parts(steps, tiles); }
int64_t jobs_most(int64_t steps, int64_t tiles) { return product_jobs_most(steps, tiles); }
int64_t i8(int64_t m, int64_t n, int64_t k, int64_t cus) { const int p = i8_parts(m, n, k, k %% 128 == 0, cus); return p == 1 ? 0 : p * ((m + 63) / 64) * ((n + 63) / 64); }
int64_t i8_most(int64_t m, int64_t n, int64_t k, int64_t cus) { return i8_jobs_most(m, n, k, cus); }
}
""" % os.path.join(ROOT, "paper_2609_36830_amd", "csrc", "rules.hpp")


@pytest.fixture(scope="module")
def R(tmp_path_factory):
    d = tmp_path_factory.mktemp("rules")
    (d / "r.cpp").write_text(SOURCE)
    subprocess.check_call(["g++", "-O1", "-std=c++17", "-shared", "-fPIC", str(d / "r.cpp"), "-o", str(d / "r.so")])
    lib = ctypes.CDLL(str(d / "r.so"))
    for name, n in (("span", 1), ("spans_most", 1), ("parts", 2), ("jobs_most", 2), ("i8", 4), ("i8_most", 4)):
        getattr(lib, name).restype, getattr(lib, name).argtypes = ctypes.c_int64, [ctypes.c_int64] * n
    return lib


@pytest.fixture(scope="module")
def pace():
    from paper_2609_36830_amd import _lib
    if not os.path.exists(_lib.library_path):
        from paper_2609_36830_amd import build
        build.build()
    import paper_2609_36830_amd as pace
    return pace


def log_int(rng, most):
    return int(2 ** rng.uniform(0, most.bit_length() - 1))


def test_spans_of_every_smaller_batch(R):
    rng = random.Random(1)
    sizes = sorted({0, 1, 255, 256, 257} | {8192 * q + d for q in (255, 256, 257, 512, 513, 1024) for d in (-1, 0, 1, 8191)} |
                   {log_int(rng, 2 ** 40) for _ in range(3000)})
    most = 0
    for nt in sizes:
        most = max(most, -(-nt // R.span(nt)))
        assert most <= R.spans_most(nt)


def test_parts_of_every_smaller_product(R):
    rng = random.Random(2)
    for _ in range(20000):
        steps, tiles = log_int(rng, 2 ** 15), log_int(rng, 2 ** 12)
        s, t = rng.randint(1, steps), rng.randint(1, tiles)
        p = R.parts(s, t)
        assert (0 if p == 1 else p * t) <= R.jobs_most(steps, tiles) <= 512
        assert R.jobs_most(s, t) <= R.jobs_most(steps, tiles)


def test_jobs_of_every_smaller_8_bit_product(R):
    rng = random.Random(3)
    for _ in range(20000):
        cus = rng.choice([32, 64, 256, 304])
        m, n, k = log_int(rng, 2 ** 13), log_int(rng, 2 ** 18), log_int(rng, 2 ** 17)
        a, b, c = rng.randint(1, m), rng.randint(1, n), max(1, rng.randint(1, k) // 128 * 128)
        assert R.i8(a, b, c, cus) <= R.i8_most(m, n, k, cus)
        assert R.i8_most(a, b, c, cus) <= R.i8_most(m, n, k, cus)
    assert R.i8_most(4, 4096, 8192, 256) == R.i8_most(8, 4096, 8192, 256) == R.i8_most(4096, 16384, 6143, 256) == 0


def test_queries_do_not_fall(pace):
    """A workspace of the largest problem is one of every smaller problem."""
    rng = random.Random(4)
    for query, most in ((pace.pace_policy_loss_workspace_bytes, (2 ** 20, 2 ** 34)), (pace.pace_matmul_i8_workspace_bytes, (2 ** 14, 2 ** 18, 2 ** 16)),
                        (pace.pace_orthogonalize_workspace_bytes, (100, 2 ** 13, 2 ** 13))):
        for _ in range(3000):
            large = [log_int(rng, v) for v in most]
            small = [rng.randint(1, v) for v in large]
            assert 256 <= query(*small) <= query(*large)
    assert pace.pace_policy_loss_workspace_bytes(1, 2100000) <= pace.pace_policy_loss_workspace_bytes(1, 2200000)
    assert pace.pace_matmul_i8_workspace_bytes(128, 4096, 8192) <= pace.pace_matmul_i8_workspace_bytes(4096, 4096, 8192)
    assert pace.pace_orthogonalize_workspace_bytes(1, 256, 8192) <= pace.pace_orthogonalize_workspace_bytes(1, 257, 8192)
