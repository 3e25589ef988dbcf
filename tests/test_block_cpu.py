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
