"""Thin ctypes binding over libalgproj.so -- argument marshalling only.

Function names mirror ``include/algproj.h``.  PyTorch appears here solely as the owner of device
memory and streams: tensors are turned into raw pointers and every step of the path runs inside
the CUDA library.  There is no CPU or eager fallback; a missing library is an error.
"""
from __future__ import annotations

import ctypes
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libalgproj.so")

ALG_OK = 0
STATUS = {0: "ALG_OK", 1: "ALG_ERR_INVALID_ARG", 2: "ALG_ERR_UNSUPPORTED_SHAPE", 3: "ALG_ERR_WORKSPACE_TOO_SMALL",
          4: "ALG_ERR_CUDA", 5: "ALG_ERR_BAD_TYPE", 6: "ALG_ERR_DEVICE_TIMEOUT"}
ALG_F32, ALG_BF16 = 0, 1
ALG_TABLE_QQ, ALG_TABLE_DENSE, ALG_TABLE_CUSTOM, ALG_TABLE_Q2POW = 0, 1, 2, 3
ALG_ACT_NONE, ALG_ACT_GELU_ERF, ALG_ACT_GELU_TANH, ALG_ACT_SILU = 0, 1, 2, 3
ALG_SCHED_EXPLICIT, ALG_SCHED_CYCLIC, ALG_SCHED_INTERVAL = 0, 1, 2
ALG_Q8_E4M3, ALG_Q8_INT8 = 0, 1
ALG_NORM_RMS, ALG_NORM_LAYER = 0, 1
ALG_NORM_JOIN, ALG_NORM_PRE, ALG_NORM_POST, ALG_NORM_GATE_ROW, ALG_NORM_GATE_ELEMENT, ALG_NORM_GATE_SIGMOID = 1, 2, 4, 8, 16, 32
ALG_MOE_SOFTMAX, ALG_MOE_SIGMOID = 0, 1
ALG_PATH_SIMT, ALG_PATH_TCGEN05, ALG_PATH_DECODE = 0, 1, 2
OPTIONS = {"gemm_kernel": 1, "tile_n": 2, "small_m_kernel": 3, "host_plan": 4, "wait_limit_cycles": 5,
           "test_stall_bytes": 6, "stage_k": 7, "interval_period": 8, "row_gather": 9, "weight_packed": 10}

_DTYPES = {"f32": ALG_F32, "bf16": ALG_BF16, torch.float32: ALG_F32, torch.bfloat16: ALG_BF16}
_TABLES = {"qq": ALG_TABLE_QQ, "dense": ALG_TABLE_DENSE, "custom": ALG_TABLE_CUSTOM, "q2pow": ALG_TABLE_Q2POW}
_ACTS = {None: ALG_ACT_NONE, "none": ALG_ACT_NONE, "gelu": ALG_ACT_GELU_ERF, "gelu_erf": ALG_ACT_GELU_ERF,
         "gelu_tanh": ALG_ACT_GELU_TANH}
_CKPT_ACTS = {**_ACTS, "silu": ALG_ACT_SILU}
_Q8 = {"e4m3": ALG_Q8_E4M3, "int8": ALG_Q8_INT8}
_SCHEDS = {"explicit": ALG_SCHED_EXPLICIT, "cyclic": ALG_SCHED_CYCLIC, "interval": ALG_SCHED_INTERVAL}

EXPORTS = [
    "alg_proj_create", "alg_proj_destroy", "alg_proj_set_option", "alg_ffn_set_option", "alg_proj_workspace_bytes", "alg_proj_forward", "alg_proj_gemm_count",
    "alg_proj_forward_static", "alg_proj_host_workspace_bytes", "alg_proj_forward_host", "alg_proj_packed_weight_bytes", "alg_proj_pack_weight", "alg_proj_macs", "alg_proj_kernel_path", "alg_proj_last_status", "alg_ffn_create", "alg_ffn_destroy",
    "alg_ffn_workspace_bytes", "alg_ffn_forward", "alg_ffn_host_workspace_bytes", "alg_ffn_forward_host",
    "alg_ffn_gated_create", "alg_ffn_gated_forward", "alg_proj_grad_create", "alg_proj_grad_destroy",
    "alg_proj_grad_workspace_bytes", "alg_proj_grad_input", "alg_proj_grad_weight", "alg_proj_grad_last_status", "alg_ffn_macs", "alg_ffn_last_status", "alg_ffn_set_timing", "alg_ffn_get_timing", "alg_status_string", "alg_launch_count",
    "alg_moe_create", "alg_moe_destroy", "alg_moe_set_option", "alg_moe_workspace_bytes", "alg_moe_forward", "alg_moe_last_status",
    "alg_norm_create", "alg_norm_destroy", "alg_norm_set_option", "alg_norm_workspace_bytes", "alg_norm_forward", "alg_norm_backward", "alg_norm_last_status",
    "alg_ckpt_create", "alg_ckpt_destroy", "alg_ckpt_row_bytes", "alg_ckpt_store", "alg_ckpt_load", "alg_ckpt_act_forward",
    "alg_ckpt_act_backward",
]

_lib = None


class AlgError(RuntimeError):
    def __init__(self, code: int, where: str):
        super().__init__(f"{where}: {STATUS.get(code, code)}")
        self.code = code


def lib() -> ctypes.CDLL:
    """Load libalgproj.so (built by ``python -m paper_2609_32814_b200.build``)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise FileNotFoundError(
                f"{LIB_PATH} is missing: build it with `python -m paper_2609_32814_b200.build`; "
                "there is no fallback implementation")
        L = ctypes.CDLL(LIB_PATH)
        vp, i64, i32 = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int
        L.alg_proj_create.argtypes = [ctypes.POINTER(vp), i32, vp, vp, i32, i32, vp, i32]
        L.alg_proj_destroy.argtypes = [vp]
        L.alg_proj_set_option.argtypes = [vp, i32, i64]
        L.alg_ffn_set_option.argtypes = [vp, i32, i64]
        L.alg_proj_workspace_bytes.argtypes = [vp, i64, ctypes.POINTER(ctypes.c_size_t)]
        L.alg_proj_forward.argtypes = [vp, vp, i64, vp, i64, vp, i64, vp, i32, vp, i64, i32, vp, ctypes.c_size_t, vp]
        L.alg_proj_forward_static.argtypes = [vp, vp, i64, vp, i64, vp, i64, vp, i32, vp, i64, i32, vp]
        L.alg_proj_host_workspace_bytes.argtypes = [vp, i64, i32, ctypes.POINTER(ctypes.c_size_t)]
        L.alg_proj_packed_weight_bytes.argtypes = [vp, ctypes.POINTER(ctypes.c_size_t)]
        L.alg_proj_pack_weight.argtypes = [vp, vp, i64, vp, ctypes.c_size_t, vp]
        L.alg_proj_forward_host.argtypes = [vp, vp, vp, i64, vp, i64, vp, i32, vp, i32, vp, ctypes.c_size_t, vp]
        L.alg_proj_gemm_count.argtypes = [vp, ctypes.POINTER(i64)]
        L.alg_proj_macs.argtypes = [vp, ctypes.POINTER(i64), ctypes.POINTER(i64)]
        L.alg_proj_kernel_path.argtypes = [vp, i64, ctypes.POINTER(i32)]
        L.alg_proj_last_status.argtypes = [vp, vp, ctypes.POINTER(i32)]
        L.alg_ffn_create.argtypes = [ctypes.POINTER(vp), i32, vp, vp, i32, i32, vp, i32]
        L.alg_ffn_destroy.argtypes = [vp]
        L.alg_proj_grad_create.argtypes = [ctypes.POINTER(vp), i32, vp, vp, i32, vp, i32]
        L.alg_proj_grad_destroy.argtypes = [vp]
        L.alg_proj_grad_workspace_bytes.argtypes = [vp, i64, ctypes.POINTER(ctypes.c_size_t)]
        L.alg_proj_grad_input.argtypes = [vp, vp, i64, vp, i64, vp, i64, vp, i64, i32, vp, ctypes.c_size_t, vp]
        L.alg_proj_grad_weight.argtypes = [vp, vp, i64, vp, i64, vp, i64, vp, i64, i32, vp, ctypes.c_size_t, vp]
        L.alg_proj_grad_last_status.argtypes = [vp, vp, ctypes.POINTER(i32)]
        L.alg_ffn_gated_create.argtypes = [ctypes.POINTER(vp), i32, vp, vp, i32, i32, vp, i32]
        L.alg_ffn_gated_forward.argtypes = [vp, vp, vp, i64, vp, vp, vp, i32, vp, ctypes.c_size_t, vp]
        L.alg_ffn_workspace_bytes.argtypes = [vp, i64, ctypes.POINTER(ctypes.c_size_t)]
        L.alg_ffn_forward.argtypes = [vp, vp, vp, i64, vp, vp, vp, vp, i32, vp, i32, vp, ctypes.c_size_t, vp]
        L.alg_ffn_host_workspace_bytes.argtypes = [vp, i64, i32, ctypes.POINTER(ctypes.c_size_t)]
        L.alg_ffn_forward_host.argtypes = [vp, vp, vp, i64, vp, vp, vp, vp, i32, vp, i32, vp, ctypes.c_size_t, vp]
        L.alg_ffn_macs.argtypes = [vp, ctypes.POINTER(i64), ctypes.POINTER(i64)]
        L.alg_ffn_last_status.argtypes = [vp, vp, ctypes.POINTER(i32)]
        L.alg_ffn_set_timing.argtypes = [vp, i32]
        L.alg_ffn_get_timing.argtypes = [vp, ctypes.POINTER(ctypes.c_float)]
        L.alg_moe_create.argtypes = [ctypes.POINTER(vp), i32, i32, i32, i32, i32, i32, ctypes.c_float, i32]
        L.alg_moe_destroy.argtypes = [vp]
        L.alg_moe_set_option.argtypes = [vp, i32, i64]
        L.alg_moe_workspace_bytes.argtypes = [vp, i64, ctypes.POINTER(ctypes.c_size_t)]
        L.alg_moe_forward.argtypes = [vp, vp, i64, i64, vp, vp, vp, vp, vp, i64, i32, vp, vp, vp, ctypes.c_size_t, vp]
        L.alg_moe_last_status.argtypes = [vp, vp, ctypes.POINTER(i32)]
        L.alg_norm_create.argtypes = [ctypes.POINTER(vp), i32, i32, i32, ctypes.c_float, i32, i32]
        L.alg_norm_destroy.argtypes = [vp]
        L.alg_norm_set_option.argtypes = [vp, i32, i64]
        L.alg_norm_workspace_bytes.argtypes = [vp, ctypes.POINTER(ctypes.c_size_t)]
        L.alg_norm_forward.argtypes = [vp, vp, i64, vp, i64, vp, i64, vp, vp, vp, ctypes.c_float, vp, vp, i64, vp, i64, vp, i64, vp]
        L.alg_norm_backward.argtypes = [vp, vp, i64, vp, i64, vp, i64, vp, i64, vp, i64, vp, vp, vp, ctypes.c_float, vp, i64, vp, i64, vp, i64,
                                        vp, i64, vp, vp, vp, vp, vp, vp, ctypes.c_size_t, vp]
        L.alg_norm_last_status.argtypes = [vp, vp, ctypes.POINTER(i32)]
        L.alg_ckpt_create.argtypes = [ctypes.POINTER(vp), i32, i32, i32, i32]
        L.alg_ckpt_destroy.argtypes = [vp]
        L.alg_ckpt_row_bytes.argtypes = [vp, ctypes.POINTER(ctypes.c_size_t)]
        L.alg_ckpt_store.argtypes = [vp, vp, i64, i32, i64, vp, vp]
        L.alg_ckpt_load.argtypes = [vp, vp, i64, vp, i64, i32, vp]
        L.alg_ckpt_act_forward.argtypes = [vp, vp, i64, i64, vp, i64, i32, vp, vp]
        L.alg_ckpt_act_backward.argtypes = [vp, vp, vp, i64, i64, vp, i64, vp, i64, i32, vp]
        L.alg_status_string.argtypes = [i32]
        L.alg_status_string.restype = ctypes.c_char_p
        L.alg_launch_count.argtypes = []
        L.alg_launch_count.restype = i64
        _lib = L
    return _lib


def _check(code: int, where: str):
    if code != ALG_OK:
        raise AlgError(code, where)


# (plain integers: the functions' argtypes turn them into pointers, and a call of a few microseconds notices every object made)
def _ptr(t):
    return None if t is None else t.data_ptr()


def _stream(stream=None):
    if stream is not None:
        return stream.cuda_stream
    # what torch.cuda.current_stream().cuda_stream is, without the Stream object (3.3 -> 0.3 us)
    return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())


def _rows(t, what, M, cols, dtype, device):
    """The leading dimension of an M x cols operand with contiguous rows, of this dtype, on the handle's device."""
    # (one test where all is well: these calls take a few microseconds, and have up to eight operands)
    if t.shape == (M, cols) and t.dtype is dtype and t.get_device() == device:
        ld, step = t.stride()
        if M <= 1:
            return cols if step == 1 or cols == 1 else _bad_rows(what)
        return ld if ld >= cols and (step == 1 or cols == 1) else _bad_rows(what)
    if t.dim() != 2 or t.shape[0] != M or t.shape[1] != cols:
        raise ValueError(f"{what} must be {M} x {cols}, got {tuple(t.shape)}")
    if t.dtype is not dtype:
        raise ValueError(f"{what} must be {dtype}, got {t.dtype}")
    raise ValueError(f"{what} must be on the handle's device, cuda:{device}")


def _bad_rows(what):
    raise ValueError(f"{what} must have contiguous rows that do not overlap")


def _widths(w):
    arr = (ctypes.c_int32 * len(w))(*[int(v) for v in w])
    return arr


def launch_count() -> int:
    return int(lib().alg_launch_count())


class _Handle:
    _destroy = None
    _set_option = None

    def __init__(self):
        self._h = ctypes.c_void_p()
        self._ws = None
        self._need = (-1, 0)   # (rows, workspace bytes) of the last call that brought no workspace

    def close(self):
        if self._h:
            getattr(lib(), self._destroy)(self._h)
            self._h = ctypes.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def set_option(self, name: str, value: int):
        """alg_*_set_option: per-handle switches (see OPTIONS and the header)."""
        _check(getattr(lib(), self._set_option)(self._h, OPTIONS[name], int(value)), self._set_option)
        self._need = (-1, 0)   # (an option may select another kernel)

    def _own_workspace(self, M: int, device) -> torch.Tensor:
        """The handle's own workspace, grown to what a call with M rows needs."""
        need = self._need
        if need[0] != M:
            need = self._need = (M, self.workspace_bytes(M))
        return self._workspace(need[1], device)

    def _workspace(self, nbytes: int, device) -> torch.Tensor:
        if self._ws is None or self._ws.numel() < nbytes or self._ws.device != device:
            self._ws = torch.empty(max(nbytes, 256), dtype=torch.uint8, device=device)
        return self._ws

    def _scratch(self, workspace, nbytes: int) -> torch.Tensor:
        """The caller's workspace, packed memory on the handle's device, or the handle's own."""
        if workspace is None:
            return self._workspace(nbytes, self._dev)
        if workspace.get_device() != self._device or not workspace.is_contiguous():
            raise ValueError("the workspace must be packed memory on the handle's device")
        return workspace


def _keep_arg(table, custom_keep, q):
    if _TABLES[table] != ALG_TABLE_CUSTOM:
        return None, None
    flat = [int(bool(v)) for v in custom_keep.reshape(-1).tolist()]
    if len(flat) != q * q * q:
        raise ValueError("custom_keep must hold q*q*q entries")
    buf = (ctypes.c_uint8 * len(flat))(*flat)
    return buf, ctypes.cast(buf, ctypes.c_void_p)


class Proj(_Handle):
    """alg_proj_* : Y = act(X *_q W + bias)."""
    _destroy = "alg_proj_destroy"
    _set_option = "alg_proj_set_option"

    def __init__(self, in_widths, out_widths, dtype="bf16", table="qq", custom_keep=None, schedule="explicit"):
        super().__init__()
        self.q = len(in_widths)
        self.in_widths, self.out_widths = list(in_widths), list(out_widths)
        self.K, self.N = sum(self.in_widths), sum(self.out_widths)
        self.dtype = _DTYPES[dtype]
        self.schedule = _SCHEDS[schedule]
        buf, keep = _keep_arg(table, custom_keep, self.q)
        s, r = _widths(in_widths), _widths(out_widths)
        _check(lib().alg_proj_create(ctypes.byref(self._h), self.q, ctypes.cast(s, ctypes.c_void_p),
                                     ctypes.cast(r, ctypes.c_void_p), self.dtype, _TABLES[table], keep,
                                     self.schedule), "alg_proj_create")

    def workspace_bytes(self, max_M: int) -> int:
        out = ctypes.c_size_t()
        _check(lib().alg_proj_workspace_bytes(self._h, max_M, ctypes.byref(out)), "alg_proj_workspace_bytes")
        return out.value

    def forward(self, X, types, W, bias=None, act=None, out=None, out_dtype=None, workspace=None, stream=None):
        M = X.shape[0]
        if out is None:
            out = torch.empty((M, self.N), dtype=out_dtype or X.dtype, device=X.device)
        ws = workspace if workspace is not None else self._own_workspace(M, X.device)
        _check(lib().alg_proj_forward(self._h, _ptr(X), X.stride(0) if M else self.K, _ptr(types), M, _ptr(W),
                                      W.stride(0), _ptr(bias), _ACTS[act], _ptr(out),
                                      out.stride(0) if M else self.N, _DTYPES[out.dtype], _ptr(ws), ws.numel(),
                                      _stream(stream)), "alg_proj_forward")
        return out

    def forward_static(self, X, types, W, out, bias=None, act=None, stream=None):
        """alg_proj_forward_static: same result as forward(), but the scratch is the fixed array
        inside the library, so nothing is allocated -- `out` must be supplied by the caller, and
        problems needing more than the built-in scratch raise ALG_ERR_WORKSPACE_TOO_SMALL."""
        M = X.shape[0]
        _check(lib().alg_proj_forward_static(self._h, _ptr(X), X.stride(0) if M else self.K, _ptr(types), M,
                                             _ptr(W), W.stride(0), _ptr(bias), _ACTS[act], _ptr(out),
                                             out.stride(0) if M else self.N, _DTYPES[out.dtype], _stream(stream)),
               "alg_proj_forward_static")
        return out

    def packed_weight_bytes(self) -> int:
        out = ctypes.c_size_t()
        _check(lib().alg_proj_packed_weight_bytes(self._h, ctypes.byref(out)), "alg_proj_packed_weight_bytes")
        return out.value

    def pack_weight(self, W, stream=None):
        """alg_proj_pack_weight: the padded bank as a flat bf16 tensor (pass it to forward with option weight_packed = 1)."""
        out = torch.empty(self.packed_weight_bytes() // 2, dtype=torch.bfloat16, device=W.device)
        _check(lib().alg_proj_pack_weight(self._h, _ptr(W), W.stride(0), _ptr(out), out.numel() * 2, _stream(stream)),
               "alg_proj_pack_weight")
        return out

    def host_workspace_bytes(self, max_M: int, out_dtype) -> int:
        out = ctypes.c_size_t()
        _check(lib().alg_proj_host_workspace_bytes(self._h, max_M, _DTYPES[out_dtype], ctypes.byref(out)),
               "alg_proj_host_workspace_bytes")
        return out.value

    def forward_host(self, X_host, types_host, W, Y_host, bias=None, act=None, workspace=None, stream=None):
        """alg_proj_forward_host: X_host / types_host / Y_host are packed CPU tensors (pinned for asynchronous copies)."""
        M = X_host.shape[0]
        need = self.host_workspace_bytes(M, Y_host.dtype)
        ws = workspace if workspace is not None else self._workspace(need, W.device)
        _check(lib().alg_proj_forward_host(self._h, _ptr(X_host), _ptr(types_host), M, _ptr(W), W.stride(0), _ptr(bias),
                                           _ACTS[act], _ptr(Y_host), _DTYPES[Y_host.dtype], _ptr(ws), ws.numel(),
                                           _stream(stream)), "alg_proj_forward_host")
        return Y_host

    def gemm_count(self) -> int:
        n = ctypes.c_int64()
        _check(lib().alg_proj_gemm_count(self._h, ctypes.byref(n)), "alg_proj_gemm_count")
        return n.value

    def macs(self, rows_per_type) -> int:
        rows = (ctypes.c_int64 * self.q)(*[int(v) for v in rows_per_type])
        out = ctypes.c_int64()
        _check(lib().alg_proj_macs(self._h, rows, ctypes.byref(out)), "alg_proj_macs")
        return out.value

    def kernel_path(self, M: int) -> int:
        p = ctypes.c_int()
        _check(lib().alg_proj_kernel_path(self._h, M, ctypes.byref(p)), "alg_proj_kernel_path")
        return p.value

    def last_status(self, stream=None) -> int:
        s = ctypes.c_int()
        _check(lib().alg_proj_last_status(self._h, _stream(stream), ctypes.byref(s)), "alg_proj_last_status")
        return s.value


class FFN(_Handle):
    """alg_ffn_* : Y = act(X *_q W_up + b_up) *_q W_down + b_down."""
    _destroy = "alg_ffn_destroy"
    _set_option = "alg_ffn_set_option"
    _create = "alg_ffn_create"

    def __init__(self, d_widths, f_widths, dtype="bf16", table="qq", custom_keep=None, schedule="explicit"):
        super().__init__()
        self.q = len(d_widths)
        self.D, self.F = sum(d_widths), sum(f_widths)
        self.dtype = _DTYPES[dtype]
        self.schedule = _SCHEDS[schedule]
        buf, keep = _keep_arg(table, custom_keep, self.q)
        d, f = _widths(d_widths), _widths(f_widths)
        _check(getattr(lib(), self._create)(ctypes.byref(self._h), self.q, ctypes.cast(d, ctypes.c_void_p),
                                            ctypes.cast(f, ctypes.c_void_p), self.dtype, _TABLES[table], keep,
                                            self.schedule), self._create)

    def workspace_bytes(self, max_M: int) -> int:
        out = ctypes.c_size_t()
        _check(lib().alg_ffn_workspace_bytes(self._h, max_M, ctypes.byref(out)), "alg_ffn_workspace_bytes")
        return out.value

    def host_workspace_bytes(self, max_M: int, out_dtype) -> int:
        out = ctypes.c_size_t()
        _check(lib().alg_ffn_host_workspace_bytes(self._h, max_M, _DTYPES[out_dtype], ctypes.byref(out)),
               "alg_ffn_host_workspace_bytes")
        return out.value

    def forward(self, X, types, W_up, W_down, b_up=None, b_down=None, act="gelu", out=None, out_dtype=None,
                workspace=None, stream=None):
        M = X.shape[0]
        if not (X.is_contiguous() and W_up.is_contiguous() and W_down.is_contiguous()):
            raise ValueError("alg_ffn_forward takes packed row-major tensors")
        if out is None:
            out = torch.empty((M, self.D), dtype=out_dtype or X.dtype, device=X.device)
        ws = workspace if workspace is not None else self._own_workspace(M, X.device)
        _check(lib().alg_ffn_forward(self._h, _ptr(X), _ptr(types), M, _ptr(W_up), _ptr(b_up), _ptr(W_down),
                                     _ptr(b_down), _ACTS[act], _ptr(out), _DTYPES[out.dtype], _ptr(ws), ws.numel(),
                                     _stream(stream)), "alg_ffn_forward")
        return out

    def forward_host(self, X_host, types_host, W_up, W_down, Y_host, b_up=None, b_down=None, act="gelu",
                     workspace=None, stream=None):
        """X_host / types_host / Y_host are CPU tensors (pinned for asynchronous copies)."""
        M = X_host.shape[0]
        need = self.host_workspace_bytes(M, Y_host.dtype)
        ws = workspace if workspace is not None else self._workspace(need, W_up.device)
        _check(lib().alg_ffn_forward_host(self._h, _ptr(X_host), _ptr(types_host), M, _ptr(W_up), _ptr(b_up),
                                          _ptr(W_down), _ptr(b_down), _ACTS[act], _ptr(Y_host), _DTYPES[Y_host.dtype],
                                          _ptr(ws), ws.numel(), _stream(stream)), "alg_ffn_forward_host")
        return Y_host

    def set_timing(self, enable: bool):
        _check(lib().alg_ffn_set_timing(self._h, int(enable)), "alg_ffn_set_timing")

    def get_timing(self):
        """Milliseconds of the last forward call: (bucketing, gather, up projection, down projection)."""
        ms = (ctypes.c_float * 4)()
        _check(lib().alg_ffn_get_timing(self._h, ms), "alg_ffn_get_timing")
        return tuple(float(v) for v in ms)

    def macs(self, rows_per_type) -> int:
        rows = (ctypes.c_int64 * self.q)(*[int(v) for v in rows_per_type])
        out = ctypes.c_int64()
        _check(lib().alg_ffn_macs(self._h, rows, ctypes.byref(out)), "alg_ffn_macs")
        return out.value

    def last_status(self, stream=None) -> int:
        s = ctypes.c_int()
        _check(lib().alg_ffn_last_status(self._h, _stream(stream), ctypes.byref(s)), "alg_ffn_last_status")
        return s.value


class GatedFFN(FFN):
    """alg_ffn_gated_* : Y = (silu(X *_q W_gate) .* (X *_q W_up)) *_q W_down, W_gate_up = [W_gate | W_up] (D x 2F)."""
    _create = "alg_ffn_gated_create"

    def forward(self, X, types, W_gate_up, W_down, out=None, out_dtype=None, workspace=None, stream=None):
        M = X.shape[0]
        if not (X.is_contiguous() and W_gate_up.is_contiguous() and W_down.is_contiguous()):
            raise ValueError("alg_ffn_gated_forward takes packed row-major tensors")
        if W_gate_up.shape != (self.D, 2 * self.F):
            raise ValueError("W_gate_up must be D x 2F: [W_gate | W_up]")
        if out is None:
            out = torch.empty((M, self.D), dtype=out_dtype or X.dtype, device=X.device)
        ws = workspace if workspace is not None else self._own_workspace(M, X.device)
        _check(lib().alg_ffn_gated_forward(self._h, _ptr(X), _ptr(types), M, _ptr(W_gate_up), _ptr(W_down), _ptr(out),
                                           _DTYPES[out.dtype], _ptr(ws), ws.numel(), _stream(stream)),
               "alg_ffn_gated_forward")
        return out

    def forward_host(self, *a, **k):
        raise NotImplementedError("the gated FFN has no host entry point")


class ProjGrad(_Handle):
    """alg_proj_grad_* : the two gradient maps of Y = X *_q W (dX from G and W, dW from X and G)."""
    _destroy = "alg_proj_grad_destroy"

    def __init__(self, in_widths, out_widths, table="qq", custom_keep=None, schedule="explicit"):
        super().__init__()
        self.q = len(in_widths)
        self.K, self.N = sum(in_widths), sum(out_widths)
        self.schedule = _SCHEDS[schedule]
        buf, keep = _keep_arg(table, custom_keep, self.q)
        s, r = _widths(in_widths), _widths(out_widths)
        _check(lib().alg_proj_grad_create(ctypes.byref(self._h), self.q, ctypes.cast(s, ctypes.c_void_p),
                                          ctypes.cast(r, ctypes.c_void_p), _TABLES[table], keep, self.schedule),
               "alg_proj_grad_create")

    def workspace_bytes(self, max_M: int) -> int:
        out = ctypes.c_size_t()
        _check(lib().alg_proj_grad_workspace_bytes(self._h, max_M, ctypes.byref(out)), "alg_proj_grad_workspace_bytes")
        return out.value

    def grad_input(self, G, types, W, out=None, out_dtype=None, workspace=None, stream=None):
        M = G.shape[0]
        if out is None:
            out = torch.empty((M, self.K), dtype=out_dtype or G.dtype, device=G.device)
        ws = workspace if workspace is not None else self._own_workspace(M, G.device)
        _check(lib().alg_proj_grad_input(self._h, _ptr(G), G.stride(0) if M else self.N, _ptr(types), M, _ptr(W), W.stride(0),
                                         _ptr(out), out.stride(0) if M else self.K, _DTYPES[out.dtype], _ptr(ws), ws.numel(),
                                         _stream(stream)), "alg_proj_grad_input")
        return out

    def grad_weight(self, X, G, types, out=None, out_dtype=torch.float32, workspace=None, stream=None):
        M = X.shape[0]
        if out is None:
            out = torch.empty((self.K, self.N), dtype=out_dtype, device=X.device)
        ws = workspace if workspace is not None else self._own_workspace(M, X.device)
        _check(lib().alg_proj_grad_weight(self._h, _ptr(X), X.stride(0) if M else self.K, _ptr(G), G.stride(0) if M else self.N,
                                          _ptr(types), M, _ptr(out), out.stride(0), _DTYPES[out.dtype], _ptr(ws), ws.numel(),
                                          _stream(stream)), "alg_proj_grad_weight")
        return out

    def last_status(self, stream=None) -> int:
        s = ctypes.c_int()
        _check(lib().alg_proj_grad_last_status(self._h, _stream(stream), ctypes.byref(s)), "alg_proj_grad_last_status")
        return s.value


class MoE(_Handle):
    """alg_moe_* : Y = sum_j weight_j * (silu(X W_gate[e_j]) .* (X W_up[e_j])) W_down[e_j], the experts e_j of a row chosen by
    its router scores.  W_router: D x E (``router_dtype``); W_gate_up: E x D x 2F, [W_gate | W_up]; W_down: E x F x D."""
    _destroy = "alg_moe_destroy"
    _set_option = "alg_moe_set_option"

    def __init__(self, D, F, experts, top_k, score="softmax", renormalise=True, route_scale=1.0, router_dtype="bf16"):
        super().__init__()
        self.D, self.F, self.E, self.top_k = int(D), int(F), int(experts), int(top_k)
        self.router_type = torch.float32 if _DTYPES[router_dtype] == ALG_F32 else torch.bfloat16
        _check(lib().alg_moe_create(ctypes.byref(self._h), self.D, self.F, self.E, self.top_k,
                                    {"softmax": ALG_MOE_SOFTMAX, "sigmoid": ALG_MOE_SIGMOID}[score], int(bool(renormalise)), float(route_scale),
                                    _DTYPES[router_dtype]), "alg_moe_create")
        self._device = torch.cuda.current_device()
        self._dev = torch.device("cuda", self._device)
        self._bytes = self.workspace_bytes(64)   # one size for every call: memory a captured call holds is never exchanged for more

    def workspace_bytes(self, max_M: int) -> int:
        out = ctypes.c_size_t()
        _check(lib().alg_moe_workspace_bytes(self._h, max_M, ctypes.byref(out)), "alg_moe_workspace_bytes")
        return out.value

    def _packed(self, t, what, shape, dtype):
        if t.shape != shape or t.dtype is not dtype or t.get_device() != self._device or not t.is_contiguous():
            raise ValueError(f"{what} must be a packed {shape} {dtype} tensor on the handle's device")
        return t.data_ptr()

    def forward(self, X, W_router, W_gate_up, W_down, select_bias=None, out=None, out_dtype=None, routing=False, experts=None, weights=None,
                workspace=None, stream=None):
        """Y, or (Y, experts, weights) with ``routing``: the rows' experts (int32) and their weights (fp32), M x top_k.  Calls of a handle,
        captured ones too, must follow one another on the GPU."""
        M = X.shape[0]
        ldx = _rows(X, "X", M, self.D, torch.bfloat16, self._device)
        if M > 64:
            raise AlgError(2, "alg_moe_forward")
        if out is None:
            out = torch.empty_like(X) if out_dtype is None or out_dtype is X.dtype else torch.empty_like(X, dtype=out_dtype)
            ldo = self.D
        else:
            ldo = _rows(out, "out", M, self.D, out.dtype, self._device)
        if routing:
            experts = torch.empty((M, self.top_k), dtype=torch.int32, device=self._dev) if experts is None else experts
            weights = torch.empty((M, self.top_k), dtype=torch.float32, device=self._dev) if weights is None else weights
        pairs = (M, self.top_k)
        ws = self._scratch(workspace, self._bytes)
        _check(lib().alg_moe_forward(self._h, X.data_ptr(), ldx, M, self._packed(W_router, "W_router", (self.D, self.E), self.router_type),
                                     None if select_bias is None else self._packed(select_bias, "select_bias", (self.E,), torch.float32),
                                     self._packed(W_gate_up, "W_gate_up", (self.E, self.D, 2 * self.F), torch.bfloat16),
                                     self._packed(W_down, "W_down", (self.E, self.F, self.D), torch.bfloat16), out.data_ptr(), ldo,
                                     _DTYPES[out.dtype], None if experts is None else self._packed(experts, "experts", pairs, torch.int32),
                                     None if weights is None else self._packed(weights, "weights", pairs, torch.float32), _ptr(ws), ws.numel(),
                                     _stream(stream)), "alg_moe_forward")
        return (out, experts, weights) if routing else out

    def last_status(self, stream=None) -> int:
        s = ctypes.c_int()
        _check(lib().alg_moe_last_status(self._h, _stream(stream), ctypes.byref(s)), "alg_moe_last_status")
        return s.value


class BlockNorm(_Handle):
    """alg_norm_* : Y = R + alpha * scale * gate * (norm(F) * post_weight + post_bias),  N = norm(Y) * pre_weight + pre_bias.

    ``join``: F is added to the residual stream R (else Y is R); ``post``: F is normed; ``pre``: N is wanted; ``gate``: None, "row"
    (one value for each row) or "element".  R, Y and their gradients have ``stream_dtype``, F, gate, N and theirs ``dtype``."""
    _destroy = "alg_norm_destroy"
    _set_option = "alg_norm_set_option"

    def __init__(self, D, kind="rms", join=False, pre=True, post=False, gate=None, gate_act=None, eps=1e-6, dtype="bf16", stream_dtype="bf16"):
        super().__init__()
        self.D, self.join, self.pre, self.post, self.gate = int(D), bool(join), bool(pre), bool(post), gate
        self._shape = (self.D,)
        self.stream_type, self.type = (torch.float32 if _DTYPES[t] == ALG_F32 else torch.bfloat16 for t in (stream_dtype, dtype))
        flags = ((ALG_NORM_JOIN if join else 0) | (ALG_NORM_PRE if pre else 0) | (ALG_NORM_POST if post else 0) |
                 {None: 0, "row": ALG_NORM_GATE_ROW, "element": ALG_NORM_GATE_ELEMENT}[gate] |
                 {None: 0, "sigmoid": ALG_NORM_GATE_SIGMOID}[gate_act])
        _check(lib().alg_norm_create(ctypes.byref(self._h), self.D, {"rms": ALG_NORM_RMS, "layer": ALG_NORM_LAYER}[kind], flags, float(eps),
                                     _DTYPES[stream_dtype], _DTYPES[dtype]), "alg_norm_create")
        self._device = torch.cuda.current_device()
        self._dev = torch.device("cuda", self._device)
        out = ctypes.c_size_t()
        _check(lib().alg_norm_workspace_bytes(self._h, ctypes.byref(out)), "alg_norm_workspace_bytes")
        self._bytes = out.value

    def workspace_bytes(self) -> int:
        """Bytes a backward call with column sums needs."""
        return self._bytes

    def _matrix(self, t, what, M, dtype):
        """(address, leading dimension) of an operand."""
        return (None, 0) if t is None else (t.data_ptr(), _rows(t, what, M, self.D, dtype, self._device))

    def _gate(self, t, what, M):
        if t is None:
            return None, 0
        if self.gate != "row":
            return t.data_ptr(), _rows(t, what, M, self.D, self.type, self._device)
        if t.shape != (M,) or t.dtype is not self.type or t.get_device() != self._device or (M > 1 and t.stride(0) != 1):
            raise ValueError(f"{what} must hold {M} packed {self.type} values on the handle's device")
        return t.data_ptr(), 0

    def _vector(self, t, what):
        if t is None:
            return None
        if t.shape != self._shape or t.dtype is not torch.float32 or t.get_device() != self._device or (t.stride(0) != 1 and self.D > 1):
            raise ValueError(f"{what} must hold {self.D} packed float32 values on the handle's device")
        return t.data_ptr()

    def _new(self, M, dtype):
        return torch.empty((M, self.D), dtype=dtype, device=self._dev)

    def forward(self, R, F=None, gate=None, post_weight=None, post_bias=None, scale=None, alpha=1.0, pre_weight=None, pre_bias=None, out=None,
                normed=None, stream=None):
        """(Y, N); Y is R without ``join``, N is None without ``pre``."""
        M, D, dev, st, dt, vec = R.shape[0], self.D, self._device, self.stream_type, self.type, self._vector
        if self.join and out is None:
            out, ldo = torch.empty_like(R), D
        else:
            ldo = 0 if out is None else _rows(out, "out", M, D, st, dev)
        if self.pre and normed is None:
            normed, ldn = torch.empty_like(R) if st is dt else torch.empty_like(R, dtype=dt), D
        else:
            ldn = 0 if normed is None else _rows(normed, "normed", M, D, dt, dev)
        g, ldg = self._gate(gate, "gate", M)
        code = lib().alg_norm_forward(
            self._h, R.data_ptr(), _rows(R, "R", M, D, st, dev), None if F is None else F.data_ptr(), 0 if F is None else _rows(F, "F", M, D, dt, dev),
            g, ldg, vec(post_weight, "post_weight"), vec(post_bias, "post_bias"), vec(scale, "scale"), alpha, vec(pre_weight, "pre_weight"),
            vec(pre_bias, "pre_bias"), M, None if out is None else out.data_ptr(), ldo, None if normed is None else normed.data_ptr(), ldn,
            _stream(stream))
        if code:
            _check(code, "alg_norm_forward")
        return (out if self.join else R), normed

    def backward(self, Y, dY=None, dN=None, F=None, gate=None, post_weight=None, post_bias=None, scale=None, alpha=1.0, pre_weight=None,
                 pre_bias=None, want=None, out=None, workspace=None, stream=None):
        """The gradients, by name: "R", "F", "gate" and those of the vectors given.  ``want``: the names to compute (R always is) instead of
        all of these; ``out``: tensors to write some of them to.  Without ``workspace`` (``workspace_bytes`` bytes) the calls of a handle share
        one: calls on several streams, or graphs that are replayed at the same time, need one each."""
        M, D, dev, st, dt, vec = Y.shape[0], self.D, self._device, self.stream_type, self.type, self._vector
        ldy = _rows(Y, "Y", M, D, st, dev)
        got = dict(out) if out else {}
        names = ("post_weight", "post_bias", "scale", "pre_weight", "pre_bias")
        given = (post_weight, post_bias, scale, pre_weight, pre_bias)
        read = [vec(v, k) for v, k in zip(given, names)]
        rows, gates = self._matrix, self._gate
        f_at, g_at = rows(F, "F", M, dt), gates(gate, "gate", M)
        # (what is allocated here needs no checks, and lies as the operand it is the gradient of: with contiguous rows)
        if "R" in got:
            r_to = rows(got["R"], "the gradient of R", M, st)
        else:
            got["R"] = t = torch.empty_like(Y)
            r_to = t.data_ptr(), D
        if want is None:
            want = [k for k, at in zip(names, read) if at is not None]
            if self.join and F is not None:
                want += ("F",) if gate is None else ("F", "gate")
        own = {}
        for k in want:
            if k in got:
                continue
            if k in names:
                t = torch.empty((D,), dtype=torch.float32, device=self._dev) if pre_weight is None else torch.empty_like(pre_weight)
            elif k == "F":
                t = self._new(M, dt) if F is None else torch.empty_like(F)
            elif k == "gate":
                t = torch.empty((M,) if self.gate == "row" else (M, D), dtype=dt, device=self._dev) if gate is None else torch.empty_like(gate)
            else:
                raise ValueError(f"no gradient is called {k}")
            got[k], own[k] = t, t.data_ptr()
        f_to = (own["F"], D) if "F" in own else rows(got.get("F"), "the gradient of F", M, dt)
        g_to = (own["gate"], D) if "gate" in own else gates(got.get("gate"), "the gradient of gate", M)
        to = [own[k] if k in own else vec(got.get(k), "the gradient of " + k) for k in names]
        ws = None
        if to != [None] * 5:
            ws = self._scratch(workspace, self._bytes)
        code = lib().alg_norm_backward(
            self._h, Y.data_ptr(), ldy, *rows(dY, "dY", M, st), *rows(dN, "dN", M, dt), *f_at, *g_at, *read[:3], alpha, read[3], M, *r_to, *f_to,
            *g_to, *to, _ptr(ws), 0 if ws is None else ws.numel(), _stream(stream))
        if code:
            _check(code, "alg_norm_backward")
        return got

    def last_status(self, stream=None) -> int:
        s = ctypes.c_int()
        _check(lib().alg_norm_last_status(self._h, _stream(stream), ctypes.byref(s)), "alg_norm_last_status")
        return s.value


class ActCheckpoint(_Handle):
    """alg_ckpt_* : an activation's input, or any other matrix, kept in 8 bits for the backward pass.

    ``cols`` is the width of A = act(Z), or of X for store and load; a gated handle takes Z = [G | U], 2 cols wide.  A
    checkpoint is a uint8 tensor of M records (``new``), whose rows can be sliced."""
    _destroy = "alg_ckpt_destroy"

    def __init__(self, cols, act=None, gated=False, fmt="e4m3"):
        super().__init__()
        self.cols, self.wide = int(cols), int(cols) * (2 if gated else 1)
        _check(lib().alg_ckpt_create(ctypes.byref(self._h), self.cols, _Q8[fmt], _CKPT_ACTS[act], int(bool(gated))), "alg_ckpt_create")
        self._device = torch.cuda.current_device()
        self._dev = torch.device("cuda", self._device)
        out = ctypes.c_size_t()
        _check(lib().alg_ckpt_row_bytes(self._h, ctypes.byref(out)), "alg_ckpt_row_bytes")
        self.row_bytes = out.value

    def set_option(self, name, value):
        raise NotImplementedError("checkpoint handles have no options")

    def new(self, M):
        """Memory for M records."""
        return torch.empty((M, self.row_bytes), dtype=torch.uint8, device=self._dev)

    def _records(self, ckpt, M):
        if _rows(ckpt, "the checkpoint", M, self.row_bytes, torch.uint8, self._device) != self.row_bytes:
            raise ValueError("the checkpoint's records must be packed")
        return ckpt.data_ptr()

    def _out(self, out, what, M, cols, dtype, like=None):
        if out is None:
            return (torch.empty((M, cols), dtype=dtype, device=self._dev) if like is None else torch.empty_like(like)), cols
        return out, _rows(out, what, M, cols, dtype, self._device)

    def store(self, X, out=None, stream=None):
        """The checkpoint of X."""
        M = X.shape[0]
        ldx = _rows(X, "X", M, self.cols, X.dtype, self._device)
        out = self.new(M) if out is None else out
        _check(lib().alg_ckpt_store(self._h, X.data_ptr(), ldx, _DTYPES[X.dtype], M, self._records(out, M), _stream(stream)), "alg_ckpt_store")
        return out

    def load(self, ckpt, out=None, out_dtype=torch.bfloat16, stream=None):
        """The values a checkpoint stands for."""
        M = ckpt.shape[0]
        out, ldo = self._out(out, "out", M, self.cols, out_dtype if out is None else out.dtype)
        _check(lib().alg_ckpt_load(self._h, self._records(ckpt, M), M, out.data_ptr(), ldo, _DTYPES[out.dtype], _stream(stream)), "alg_ckpt_load")
        return out

    def forward(self, Z, out=None, ckpt=None, keep=True, stream=None):
        """(A, checkpoint of Z); keep=False: (A, None), nothing is kept."""
        M = Z.shape[0]
        ldz = _rows(Z, "Z", M, self.wide, Z.dtype, self._device)
        out, ldo = self._out(out, "out", M, self.cols, Z.dtype, Z if self.wide == self.cols else None)
        if keep and ckpt is None:
            ckpt = self.new(M)
        _check(lib().alg_ckpt_act_forward(self._h, Z.data_ptr(), ldz, M, out.data_ptr(), ldo, _DTYPES[Z.dtype],
                                          self._records(ckpt, M) if keep else None, _stream(stream)), "alg_ckpt_act_forward")
        return out, ckpt if keep else None

    def backward(self, ckpt, dA, out=None, again=True, stream=None):
        """(dZ, A) from the checkpoint of Z and the gradient of A.  ``again``: a tensor for A, True for a new one, False for none."""
        M = dA.shape[0]
        ldd = _rows(dA, "dA", M, self.cols, dA.dtype, self._device)
        out, ldo = self._out(out, "out", M, self.wide, dA.dtype, dA if self.wide == self.cols else None)
        A, lda = (None, 0) if again is False or again is None else self._out(None if again is True else again, "again", M, self.cols, dA.dtype, dA)
        _check(lib().alg_ckpt_act_backward(self._h, self._records(ckpt, M), dA.data_ptr(), ldd, M, out.data_ptr(), ldo, _ptr(A), lda,
                                           _DTYPES[dA.dtype], _stream(stream)), "alg_ckpt_act_backward")
        return out, A
