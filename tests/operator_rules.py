"""The library's rule for the tiles of matrix products (csrc/rules.hpp), compiled
for the host: tests choose sizes that reach every tile by the rule itself."""
import ctypes
import os
import subprocess
import tempfile

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "paper_2609_36830_amd", "csrc", "rules.hpp")
SOURCE = """
#include "%s"
using namespace pace;
extern "C" {
int full(int64_t m, int64_t n, int64_t batch, int64_t steps, int64_t cus) {
    return product_tile(steps, cus, [=](int64_t s) { return ((m + s - 1) / s) * ((n + s - 1) / s) * batch; });
}
int lower(int64_t m, int64_t batch, int64_t steps, int64_t cus) {
    return product_tile(steps, cus, [=](int64_t s) { const int64_t t = (m + s - 1) / s; return t * (t + 1) / 2 * batch; });
}
int64_t parts(int64_t rows, int64_t vocab, int k) { return logprob_plan(rows, vocab, k).parts; }
int waves(int64_t rows, int64_t vocab, int k) { return logprob_plan(rows, vocab, k).waves; }
int product(int64_t steps, int64_t tiles) { return product_parts(steps, tiles); }
int cols(int64_t mp, int64_t n, int64_t batch, int64_t cus) { return ortho_step_cols(mp, n, batch, cus); }
int whole(int64_t mp, int64_t np) { return ortho_whole(mp, np); }
int64_t span(int64_t n_tokens) { return policy_loss_span(n_tokens); }
}
""" % HEADER
CUS = 256

_lib = None


def rules():
    global _lib
    if _lib is None:
        with tempfile.TemporaryDirectory() as d:
            src, so = os.path.join(d, "r.cpp"), os.path.join(d, "r.so")
            with open(src, "w") as fh:
                fh.write(SOURCE)
            subprocess.check_call(["g++", "-O1", "-std=c++17", "-shared", "-fPIC", src, "-o", so])
            _lib = ctypes.CDLL(so)
        i64 = ctypes.c_int64
        for name, res, args in (("full", ctypes.c_int, (i64,) * 5), ("lower", ctypes.c_int, (i64,) * 4), ("parts", i64, (i64, i64, ctypes.c_int)), ("waves", ctypes.c_int, (i64, i64, ctypes.c_int)),
                                ("product", ctypes.c_int, (i64, i64)), ("cols", ctypes.c_int, (i64,) * 4), ("whole", ctypes.c_int, (i64, i64)), ("span", i64, (i64,))):
            f = getattr(_lib, name)
            f.restype, f.argtypes = res, args
    return _lib
