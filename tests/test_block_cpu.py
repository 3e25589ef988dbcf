"""Argument errors of the calls around the projections that need no GPU."""
import ctypes

from paper_2609_32814_b200 import binding, build


def _lib():
    build.build()
    return binding.lib()


def test_checkpoint_handles_refuse_bad_arguments_first():
    L, h = _lib(), ctypes.c_void_p()
    ref = ctypes.byref(h)
    assert L.alg_ckpt_create(None, 64, 0, 1, 0) == 1
    for cols, fmt, act in ((0, 0, 1), (-8, 0, 1), (262145, 0, 1), (64, 2, 1), (64, -1, 1), (64, 0, 4), (64, 0, -1)):
        assert L.alg_ckpt_create(ref, cols, fmt, act, 0) == 1
        assert not h.value
    n = ctypes.c_size_t()
    assert L.alg_ckpt_row_bytes(None, ctypes.byref(n)) == 1 and L.alg_ckpt_destroy(None) == 1
    assert L.alg_ckpt_store(None, None, 0, 0, 0, None, None) == 1 and L.alg_ckpt_load(None, None, 0, None, 0, 0, None) == 1
    assert L.alg_ckpt_act_forward(None, None, 0, 0, None, 0, 0, None, None) == 1
    assert L.alg_ckpt_act_backward(None, None, None, 0, 0, None, 0, None, 0, 0, None) == 1


def test_norm_handles_refuse_bad_arguments_first():
    L, h = _lib(), ctypes.c_void_p()
    ref = ctypes.byref(h)
    nan, inf = float("nan"), float("inf")
    assert L.alg_norm_create(None, 64, 0, 2, 1e-6, 1, 1) == 1
    for D, kind, flags, eps, st, dt in ((0, 0, 2, 1e-6, 1, 1), (64, 2, 2, 1e-6, 1, 1), (64, 0, 0, 1e-6, 1, 1), (64, 0, 4, 1e-6, 1, 1),
                                        (64, 0, 2 | 4, 1e-6, 1, 1), (64, 0, 1 | 8 | 16, 1e-6, 1, 1), (64, 0, 1 | 32, 1e-6, 1, 1),
                                        (64, 0, 64 | 2, 1e-6, 1, 1), (64, 0, -1, 1e-6, 1, 1), (64, 0, 2, -1e-6, 1, 1), (64, 0, 2, nan, 1, 1),
                                        (64, 0, 2, inf, 1, 1), (64, 0, 2, 1e-6, 2, 1), (64, 0, 2, 1e-6, 1, -1)):
        assert L.alg_norm_create(ref, D, kind, flags, eps, st, dt) == 1
        assert not h.value
    assert L.alg_norm_create(ref, 8193, 0, 2, 1e-6, 1, 1) == 2
    n = ctypes.c_size_t()
    assert L.alg_norm_workspace_bytes(None, ctypes.byref(n)) == 1 and L.alg_norm_destroy(None) == 1
    assert L.alg_norm_forward(None, None, 0, None, 0, None, 0, None, None, None, 1.0, None, None, 0, None, 0, None, 0, None) == 1
    assert L.alg_norm_backward(None, None, 0, None, 0, None, 0, None, 0, None, 0, None, None, None, 1.0, None, 0, None, 0, None, 0, None, 0, None,
                               None, None, None, None, None, 0, None) == 1
    s = ctypes.c_int()
    assert L.alg_norm_last_status(None, None, ctypes.byref(s)) == 1


def test_expert_handles_refuse_bad_arguments_first():
    L, h = _lib(), ctypes.c_void_p()
    ref = ctypes.byref(h)
    assert L.alg_moe_create(None, 64, 64, 8, 2, 0, 1, 1.0, 1) == 1
    for code, args in ((1, (0, 64, 8, 2, 0, 1, 1.0, 1)), (1, (64, 0, 8, 2, 0, 1, 1.0, 1)), (1, (64, 64, 0, 1, 0, 1, 1.0, 1)), (1, (64, 64, 8, 9, 0, 1, 1.0, 1)),
                       (1, (64, 64, 8, 0, 0, 1, 1.0, 1)), (1, (64, 64, 8, 2, 2, 1, 1.0, 1)), (1, (64, 64, 8, 2, 0, 1, float("nan"), 1)),
                       (1, (64, 64, 8, 2, 0, 1, 1.0, 2)), (2, (60, 64, 8, 2, 0, 1, 1.0, 1)), (2, (64, 4, 8, 2, 0, 1, 1.0, 1)),
                       (2, (64, 64, 513, 2, 0, 1, 1.0, 1)), (2, (64, 64, 64, 33, 0, 1, 1.0, 1))):
        assert L.alg_moe_create(ref, *args) == code, args
        assert not h.value
    n, s = ctypes.c_size_t(), ctypes.c_int()
    assert L.alg_moe_workspace_bytes(None, 1, ctypes.byref(n)) == 1 and L.alg_moe_destroy(None) == 1
    assert L.alg_moe_forward(None, None, 0, 1, None, None, None, None, None, 0, 1, None, None, None, 0, None) == 1
    assert L.alg_moe_last_status(None, None, ctypes.byref(s)) == 1


def test_norm_handles_have_options():
    L = _lib()
    assert L.alg_norm_set_option(None, 5, 1000) == 1


def test_expert_handles_have_options():
    L = _lib()
    assert L.alg_moe_set_option(None, 5, 1000) == 1
