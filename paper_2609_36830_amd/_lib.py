"""Loader of the in-tree ``libpace.so`` and its C signatures (include/pace.h)."""
from __future__ import annotations

import ctypes
import os

_HERE = os.path.dirname(os.path.abspath(__file__))
library_path = os.path.join(_HERE, "libpace.so")
lists_path = os.path.join(_HERE, "_lists.so")
_lib = None
_lists = None


class PaceParams(ctypes.Structure):
    """Mirror of ``pace_params``."""
    _fields_ = [("w_wait", ctypes.c_double), ("gamma", ctypes.c_int32),
                ("window_min", ctypes.c_int32), ("beta", ctypes.c_double),
                ("r_max", ctypes.c_double)]


class AdamwParams(ctypes.Structure):
    """Mirror of ``pace_adamw_params``."""
    _fields_ = [("lr", ctypes.c_double), ("beta1", ctypes.c_double), ("beta2", ctypes.c_double), ("eps", ctypes.c_double),
                ("step", ctypes.c_int64)]


# (name, restype, argtypes) of every exported entry point.
P, i64, i32, d, sz = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32, ctypes.c_double, ctypes.c_size_t
SIGNATURES = [
    ("pace_default_params", None, [P]),
    ("pace_workspace_bytes", ctypes.c_int, [ctypes.c_int, i64, i64, P]),
    ("pace_score", ctypes.c_int, [P, P, i64, i64, P, i32, P, P, i64, P, P, P, P, P, sz, P]),
    ("pace_budget", ctypes.c_int, [i64, i64, P, P, P]),
    ("pace_select", ctypes.c_int, [P, i64, i64, P, P, P, sz, P]),
    ("pace_compact", ctypes.c_int, [P, i64, i64, P, ctypes.c_int, P, P, P, P, P, P, P, sz, P]),
    ("pace_validate", ctypes.c_int, [P, P, i64, i64, P, i32, P, i64, P, P]),
    ("pace_filter_step", ctypes.c_int, [P, P, i64, i64, P, i32, P, P, i64, i64, i64, P, P, P, P, P, P,
                                        P, P, ctypes.c_int, P, P, P, P, P, P, P, sz, P]),
    ("pace_filter_step_noalloc", ctypes.c_int, [P, P, i64, i64, P, i32, P, P, i64, i64, i64, P, P, P, P, P,
                                                P, P, P, ctypes.c_int, P, P, P, P, P, P, P]),
    ("pace_group_score", ctypes.c_int, [P, i64, P, i64, P, P]),
    ("pace_group_expand", ctypes.c_int, [P, i64, i64, P, P, P]),
    ("pace_validate_groups", ctypes.c_int, [P, i64, i64, P, P]),
    ("pace_group_filter_step", ctypes.c_int, [P, P, i64, i64, P, i32, P, P, i64, P, i64, i64, i64, P, P, P,
                                              P, P, P, P, P, P, P, ctypes.c_int, P, P, P, P, P, P, P, sz, P]),
    ("pace_stream_admit", ctypes.c_int, [P, i64, d, P, i64, P, i64, P, P, P, P, P, P, P]),
    ("pace_stream_step", ctypes.c_int, [P, P, i64, i64, P, i32, P, P, i64, i64, i64, P, P, i64, P, i64, P,
                                        P, P, P, P, P, P, P, P, ctypes.c_int, P, P, P, P, P, P, P, sz, P]),
    ("pace_prefix_score", ctypes.c_int, [P, P, P, P, i64, i64, i64, i64, P, P]),
    ("pace_stale_k", ctypes.c_int, [P, P, P, i32, i64, i64, P, P, P]),
    ("pace_diagnostics", ctypes.c_int, [P, P, P, P, i32, P, i64, P, ctypes.c_int, P, P, P]),
    ("pace_token_logprob_workspace_bytes", ctypes.c_int, [i64, i64, ctypes.c_int, P]),
    ("pace_token_logprob", ctypes.c_int, [P, ctypes.c_int, i64, i64, i64, P, d, ctypes.c_int, P, P, P, P, P, P, sz, P]),
    ("pace_token_logprob_backward", ctypes.c_int, [P, ctypes.c_int, i64, i64, i64, P, d, P, P, P, P, P, i64, P]),
    ("pace_policy_loss_workspace_bytes", ctypes.c_int, [i64, i64, P]),
    ("pace_policy_loss", ctypes.c_int, [P, P, P, P, i64, i64, P, P, d, d, d, d, P, P, P, P, P, sz, P]),
    ("pace_quantize_rows", ctypes.c_int, [P, ctypes.c_int, i64, i64, i64, P, P, P]),
    ("pace_matmul_i8_workspace_bytes", ctypes.c_int, [i64, i64, i64, P]),
    ("pace_matmul_i8", ctypes.c_int, [P, i64, P, P, i64, P, i64, i64, i64, P, ctypes.c_int, i64, P, sz, P]),
    ("pace_orthogonalize_workspace_bytes", ctypes.c_int, [i64, i64, i64, P]),
    ("pace_orthogonalize", ctypes.c_int, [P, ctypes.c_int, i64, i64, i64, i64, i64, ctypes.c_int, P, d, P, P, sz, P]),
    ("pace_layer_norm", ctypes.c_int, [P, ctypes.c_int, i64, i64, i64, P, P, ctypes.c_int, d, P, i64, P, P]),
    ("pace_layer_norm_backward_workspace_bytes", ctypes.c_int, [i64, i64, P]),
    ("pace_layer_norm_backward", ctypes.c_int, [P, ctypes.c_int, i64, i64, i64, P, ctypes.c_int, P, P, i64, P, i64, P, P, P, sz, P]),
    ("pace_grad_norm_workspace_bytes", ctypes.c_int, [i64, i64, P]),
    ("pace_grad_norm", ctypes.c_int, [i64, P, P, P, d, P, P, P, sz, P]),
    ("pace_adamw", ctypes.c_int, [i64, P, P, P, P, P, ctypes.c_int, P, P, P, P, P, P, P, P, P, P]),
    ("pace_adamw_unpack", ctypes.c_int, [i64, P, P, P, P, P, P, P]),
    ("pace_time_next_kernel", ctypes.c_int, [ctypes.c_int, P, P]),
    ("pace_strerror", ctypes.c_char_p, [ctypes.c_int]),
]


def load(path: str = library_path):
    """Open the library; raises if it has not been built (no fallback exists)."""
    if not os.path.exists(path):
        raise ImportError("libpace.so is not built at %s; run __graft_entry__.build() "
                          "or python -m paper_2609_36830_amd.build" % path)
    h = ctypes.CDLL(path)
    for name, res, args in SIGNATURES:
        fn = getattr(h, name)
        fn.restype = res
        fn.argtypes = args
    return h


def _extension():
    global _lists
    if _lists is None:
        import importlib.util
        import torch  # noqa: F401  (its libraries)
        if not os.path.exists(lists_path):
            raise ImportError("_lists.so is not built at %s; run __graft_entry__.build() "
                              "or python -m paper_2609_36830_amd.build" % lists_path)
        spec = importlib.util.spec_from_file_location(__package__ + "._lists", lists_path)
        _lists = importlib.util.module_from_spec(spec)
        spec.loader.exec_module(_lists)
    return _lists


def lists():
    """The extension that reads lists of tensors; raises if it has not been built (no fallback exists)."""
    return _extension()


def wrote(*tensors):
    """Tells torch, as its own operations in place do, that lists of tensors (or None) have been written through their pointers."""
    _extension().wrote(*tensors)


def lib():
    global _lib
    if _lib is None:
        _lib = load()
    return _lib
