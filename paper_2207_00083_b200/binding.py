"""Thin ctypes binding over libdk.so: argument marshalling only.

Every function has the name of the C entry point it calls (see include/dk.h).
Tensors are torch CUDA tensors (fp32, contiguous) used purely as device
memory; coefficient matrices are NumPy float32 arrays on the host.  Nothing
here computes: if libdk.so is missing, loading the library fails loudly,
there is no CPU fallback.
"""
from __future__ import annotations

import ctypes
import os
from types import SimpleNamespace
from typing import Optional

import numpy as np
import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libdk.so")

DK_FC, DK_CONV2D = 0, 1
DK_NHWC, DK_NCHW = 0, 1
DK_PREC_DEFAULT, DK_TF32X3, DK_FP32_SIMT, DK_FP64_SIMT, DK_TF32X2_WUNSPLIT = 0, 1, 2, 3, 4
(DK_OPT_TC_CHUNK, DK_OPT_WG_CHUNK, DK_OPT_TC_BK, DK_OPT_TC_PAIR, DK_OPT_WG_PACK, DK_OPT_WG_PAIR, DK_OPT_TC_STEM,
 DK_OPT_FIELD_PATH, DK_OPT_SPIN_LIMIT, DK_OPT_TEST_WITHHOLD, DK_OPT_XBAR_HI, DK_OPT_TC_MPACK,
 DK_OPT_SLABS, DK_OPT_SLABS_FORCE, DK_OPT_TC_CHUNK_ADAPT, DK_OPT_WG_PACE, DK_OPT_TC_LO_INKERNEL, DK_OPT_TC_SPLIT_RING, DK_OPT_NOISE_ROWS, DK_OPT_TC_PACE) = range(20)
DK_ERR_TIMEOUT = 6
STATUS_NAMES = ["DK_OK", "DK_ERR_INVALID_ARG", "DK_ERR_SHAPE", "DK_ERR_SINGULAR", "DK_ERR_WORKSPACE",
                "DK_ERR_CUDA", "DK_ERR_TIMEOUT", "DK_ERR_UNSUPPORTED"]


class DkError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        name = STATUS_NAMES[status] if 0 <= status < len(STATUS_NAMES) else str(status)
        super().__init__(f"{where} failed with {name}")


class dk_problem(ctypes.Structure):
    _fields_ = [("kind", ctypes.c_int32), ("layout", ctypes.c_int32),
                ("cin", ctypes.c_int32), ("cout", ctypes.c_int32),
                ("h", ctypes.c_int32), ("w", ctypes.c_int32),
                ("kh", ctypes.c_int32), ("kw", ctypes.c_int32),
                ("stride", ctypes.c_int32), ("pad", ctypes.c_int32),
                ("K", ctypes.c_int32), ("G", ctypes.c_int32),
                ("precision", ctypes.c_int32), ("tol", ctypes.c_float)]


class dk_verdict(ctypes.Structure):
    _fields_ = [("ok", ctypes.c_int32), ("n_flagged", ctypes.c_uint32),
                ("first_index", ctypes.c_int64), ("max_ratio", ctypes.c_float),
                ("status", ctypes.c_int32)]


class dk_fault(ctypes.Structure):
    _fields_ = [("group", ctypes.c_int32), ("enc", ctypes.c_int32),
                ("out_index", ctypes.c_int64), ("delta", ctypes.c_float)]


class dk_field_fault(ctypes.Structure):
    _fields_ = [("group", ctypes.c_int32), ("enc", ctypes.c_int32),
                ("out_index", ctypes.c_int64), ("delta", ctypes.c_uint32)]


DK_F32, DK_BF16 = 0, 1
DK_ACT_NONE, DK_ACT_RELU, DK_ACT_SILU = 0, 1, 2


class dk_norm(ctypes.Structure):
    _fields_ = [("n", ctypes.c_int64), ("h", ctypes.c_int32), ("w", ctypes.c_int32), ("c", ctypes.c_int32),
                ("groups", ctypes.c_int32), ("act", ctypes.c_int32), ("dtype", ctypes.c_int32), ("eps", ctypes.c_float)]


class dk_xent(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int64), ("d", ctypes.c_int32), ("vocab", ctypes.c_int32), ("dtype", ctypes.c_int32)]


class dk_ortho(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("m", ctypes.c_int32), ("n", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("steps", ctypes.c_int32), ("a", ctypes.c_float), ("b", ctypes.c_float), ("c", ctypes.c_float),
                ("eps", ctypes.c_float)]


DK_BLOCK_RMS, DK_BLOCK_LAYER = 0, 1


class dk_ckpt8(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int64), ("d", ctypes.c_int32), ("dtype", ctypes.c_int32)]


class dk_wgrad8(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int64), ("d", ctypes.c_int32), ("out", ctypes.c_int32), ("dtype", ctypes.c_int32)]


class dk_block(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int64), ("d", ctypes.c_int32), ("rows_per_gate", ctypes.c_int64),
                ("kind", ctypes.c_int32), ("dtype", ctypes.c_int32), ("eps", ctypes.c_float), ("keep", ctypes.c_float),
                ("scale", ctypes.c_float)]


VERDICT_BYTES = ctypes.sizeof(dk_verdict)
_lib = None


def _signatures():
    vp, i32 = ctypes.c_void_p, ctypes.c_int32
    pp = ctypes.POINTER(dk_problem)
    return {
        "dk_create": [ctypes.POINTER(vp), ctypes.c_int],
        "dk_destroy": [vp],
        "dk_status_string": [ctypes.c_int],
        "dk_workspace_bytes": [pp, ctypes.POINTER(ctypes.c_size_t)],
        "dk_set_workspace": [vp, vp, ctypes.c_size_t],
        "dk_set_option": [vp, i32, i32],
        "dk_get_option": [vp, i32, ctypes.POINTER(i32)],
        "dk_encode": [vp, pp, vp, vp, vp, vp, vp],
        "dk_linear_fwd": [vp, pp, vp, vp, vp, vp],
        "dk_decode_verify": [vp, pp, vp, vp, vp, vp, vp, vp],
        "dk_masked_linear": [vp, pp, vp, vp, vp, vp, vp, vp, vp, vp, ctypes.POINTER(dk_fault), vp],
        "dk_linear_bwd_wgrad": [vp, pp, vp, vp, i32, vp, vp, ctypes.c_float, vp, vp],
        "dk_linear_bwd_wgrad_accumulate": [vp, pp, vp, vp, i32, vp, vp, ctypes.c_float, vp, vp],
        "dk_linear_bwd_dgrad": [vp, pp, vp, vp, vp, vp],
        "dk_relu_pool_fwd": [vp, vp, ctypes.c_int64, i32, i32, i32, i32, vp, vp],
        "dk_relu_pool_bwd": [vp, vp, vp, ctypes.c_int64, i32, i32, i32, i32, vp, vp],
        "dk_linear_bwd_wgrad_verify": [vp, pp, vp, vp, vp, vp, ctypes.c_float, ctypes.c_float, vp, vp,
                                       ctypes.POINTER(dk_fault), vp],
        "dk_decode_verify_static": [ctypes.c_int, pp, vp, vp, vp, vp, vp, vp],
        "dk_device_status": [vp, ctypes.POINTER(ctypes.c_int32)],
        "dk_field_workspace_bytes": [pp, ctypes.POINTER(ctypes.c_size_t)],
        "dk_field_quantize": [vp, vp, ctypes.c_int64, i32, ctypes.c_uint32, vp, vp],
        "dk_field_dequantize": [vp, vp, ctypes.c_int64, i32, ctypes.c_uint32, vp, vp],
        "dk_field_encode": [vp, pp, ctypes.c_uint32, vp, vp, vp, vp, vp],
        "dk_field_linear_fwd": [vp, pp, ctypes.c_uint32, vp, vp, vp, vp],
        "dk_field_decode_verify": [vp, pp, ctypes.c_uint32, i32, vp, vp, vp, vp, vp, vp, vp],
        "dk_field_masked_linear": [vp, pp, ctypes.c_uint32, i32, vp, vp, vp, vp, vp, vp, vp, vp, vp,
                                   ctypes.POINTER(dk_field_fault), vp],
        "dk_field_linear_bwd_wgrad": [vp, pp, ctypes.c_uint32, vp, vp, i32, vp, vp, vp, vp],
        "dk_norm_workspace_bytes": [ctypes.POINTER(dk_norm), ctypes.POINTER(ctypes.c_size_t)],
        "dk_group_norm_fwd": [vp, ctypes.POINTER(dk_norm), vp, vp, vp, vp, vp, vp],
        "dk_group_norm_bwd": [vp, ctypes.POINTER(dk_norm), vp, vp, vp, vp, vp, vp, vp, vp, vp],
        "dk_xent_workspace_bytes": [ctypes.POINTER(dk_xent), ctypes.POINTER(ctypes.c_size_t)],
        "dk_xent_fwd_workspace_bytes": [ctypes.POINTER(dk_xent), ctypes.POINTER(ctypes.c_size_t)],
        "dk_linear_xent_fwd": [vp, ctypes.POINTER(dk_xent), vp, vp, vp, vp, vp, vp],
        "dk_linear_xent_bwd": [vp, ctypes.POINTER(dk_xent), vp, vp, vp, vp, vp, ctypes.c_float, vp, vp, vp],
        "dk_ortho_workspace_bytes": [ctypes.POINTER(dk_ortho), ctypes.POINTER(ctypes.c_size_t)],
        "dk_orthogonalize": [vp, ctypes.POINTER(dk_ortho), vp, ctypes.c_float, ctypes.c_float, vp, vp],
        "dk_ckpt8_bytes": [ctypes.POINTER(dk_ckpt8), ctypes.POINTER(ctypes.c_size_t)],
        "dk_ckpt8_store": [vp, ctypes.POINTER(dk_ckpt8), vp, vp, vp],
        "dk_ckpt8_load": [vp, ctypes.POINTER(dk_ckpt8), vp, vp, vp],
        "dk_group_norm_fwd_ckpt8": [vp, ctypes.POINTER(dk_norm), vp, vp, vp, vp, vp, vp, vp],
        "dk_group_norm_bwd_ckpt8": [vp, ctypes.POINTER(dk_norm), vp, vp, vp, vp, vp, vp, vp, vp, vp],
        "dk_wgrad8_workspace_bytes": [ctypes.POINTER(dk_wgrad8), ctypes.POINTER(ctypes.c_size_t)],
        "dk_linear_bwd_wgrad_ckpt8": [vp, ctypes.POINTER(dk_wgrad8), vp, vp, ctypes.c_float, ctypes.c_float, vp, vp, vp],
        "dk_block_workspace_bytes": [ctypes.POINTER(dk_block), ctypes.POINTER(ctypes.c_size_t)],
        "dk_block_norm_fwd": [vp, ctypes.POINTER(dk_block)] + [vp] * 12,
        "dk_block_norm_bwd": [vp, ctypes.POINTER(dk_block)] + [vp] * 15,
        "dk_block_norm_bwd_ckpt8": [vp, ctypes.POINTER(dk_block)] + [vp] * 15,
        "dk_profile_enable": [vp, ctypes.c_int],
        "dk_profile_read": [vp, ctypes.c_int, ctypes.POINTER(ctypes.c_double),
                            ctypes.POINTER(ctypes.c_int64), ctypes.POINTER(ctypes.c_int64)],
        "dk_profile_reset": [vp],
    }


EXPORTS = list(_signatures().keys())


def lib() -> ctypes.CDLL:
    """Loads libdk.so (once).  Raises if the library has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError(f"{LIB_PATH} not found: build it with `python -m paper_2207_00083_b200.build`")
        L = ctypes.CDLL(LIB_PATH)
        for name, argtypes in _signatures().items():
            fn = getattr(L, name)
            fn.argtypes = argtypes
            fn.restype = ctypes.c_char_p if name == "dk_status_string" else ctypes.c_int
        _lib = L
    return _lib


def problem_from_spec(spec, layout: int = DK_NHWC, precision: Optional[int] = None,
                      tol: float = 0.0, G: Optional[int] = None) -> dk_problem:
    """dk_problem for a ``synth.LayerSpec``-like object.  ``precision=None``
    follows the spec's own hint (fp64 for the high-noise workload)."""
    kind = DK_FC if spec.kind == "fc" else DK_CONV2D
    if precision is None:
        precision = DK_FP64_SIMT if getattr(spec, "precision", "default") == "fp64" else DK_PREC_DEFAULT
    return dk_problem(kind, layout, spec.cin, spec.cout, spec.h, spec.w, spec.kh, spec.kw,
                      spec.stride, spec.pad, spec.K, spec.G if G is None else G, precision, tol)


def _dev(ctx, t: Optional[torch.Tensor]):
    if t is None:
        return None
    if not (t.get_device() == ctx.device and t.dtype == torch.float32 and t.is_contiguous()):
        raise ValueError(f"expected a contiguous fp32 tensor on CUDA device {ctx.device}")
    return ctypes.c_void_p(t.data_ptr())


def _host(a: np.ndarray):
    if not (isinstance(a, np.ndarray) and a.dtype == np.float32 and a.flags["C_CONTIGUOUS"]):
        raise ValueError("expected a C-contiguous float32 NumPy array")
    return ctypes.c_void_p(a.ctypes.data)


# (some of the calls take microseconds on the GPU for small layers: their marshalling is kept to plain integers)
_raw_stream = torch._C._cuda_getCurrentRawStream


def _stream(ctx) -> ctypes.c_void_p:
    return ctypes.c_void_p(_raw_stream(ctx.device))


def _check(status: int, where: str):
    if status != 0:
        raise DkError(status, where)


class Context:
    """Owns a dk_ctx and (optionally) a torch-allocated workspace."""

    def __init__(self, device: int = 0):
        self._h = ctypes.c_void_p()
        self._ws = None
        torch.cuda.init()
        _check(lib().dk_create(ctypes.byref(self._h), device), "dk_create")
        self.device = device

    def close(self):
        if self._h:
            lib().dk_destroy(self._h)
            self._h = ctypes.c_void_p()
            self._ws = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    @property
    def handle(self):
        return self._h

    def workspace_bytes(self, p: dk_problem) -> int:
        n = ctypes.c_size_t()
        _check(lib().dk_workspace_bytes(ctypes.byref(p), ctypes.byref(n)), "dk_workspace_bytes")
        return n.value

    def field_workspace_bytes(self, p: dk_problem) -> int:
        n = ctypes.c_size_t()
        _check(lib().dk_field_workspace_bytes(ctypes.byref(p), ctypes.byref(n)), "dk_field_workspace_bytes")
        return n.value

    def step_workspace_bytes(self, q, forward: bool = False) -> int:
        """Workspace of a dk_norm, dk_xent, dk_ortho, dk_wgrad8 or dk_block call (``forward=True``: of
        dk_linear_xent_fwd alone)."""
        name = f"{type(q).__name__}{'_fwd' if forward and isinstance(q, dk_xent) else ''}_workspace_bytes"
        n = ctypes.c_size_t()
        _check(getattr(lib(), name)(ctypes.byref(q), ctypes.byref(n)), name)
        return n.value

    def ensure_workspace(self, p, field: bool = False, forward: bool = False):
        """Grows the torch-owned workspace to what `p` (a dk_problem, dk_norm, dk_xent, dk_ortho, dk_wgrad8 or dk_block)
        needs and registers it (``field=True``: what the finite-field calls need; ``forward=True`` with a dk_xent: what
        dk_linear_xent_fwd alone needs).  Growing it releases the buffer before: no call in flight on another stream
        and no captured graph may still use that."""
        if not isinstance(p, dk_problem):
            need = self.step_workspace_bytes(p, forward)
        else:
            need = self.field_workspace_bytes(p) if field else self.workspace_bytes(p)
        if self._ws is None or self._ws.numel() < need + 256:
            self._ws = None
            self._ws = torch.empty(need + 256, dtype=torch.uint8, device=f"cuda:{self.device}")
        base = self._ws.data_ptr()
        off = (-base) % 256
        _check(lib().dk_set_workspace(self._h, ctypes.c_void_p(base + off), self._ws.numel() - off),
               "dk_set_workspace")


def dk_set_option(ctx: Context, option: int, value: int):
    _check(lib().dk_set_option(ctx.handle, option, value), "dk_set_option")


def dk_get_option(ctx: Context, option: int) -> int:
    v = ctypes.c_int32()
    _check(lib().dk_get_option(ctx.handle, option, ctypes.byref(v)), "dk_get_option")
    return v.value


KERNEL_KINDS = ["encode", "linear_fwd", "decode_verify", "mix_delta", "wgrad", "other"]


def dk_profile_enable(ctx: Context, on: bool):
    _check(lib().dk_profile_enable(ctx.handle, int(on)), "dk_profile_enable")


def dk_profile_reset(ctx: Context):
    _check(lib().dk_profile_reset(ctx.handle), "dk_profile_reset")


def dk_profile_read(ctx: Context) -> dict:
    """{kind: (ms_total, timed_launches, all_launches)} since the last reset."""
    out = {}
    for k, name in enumerate(KERNEL_KINDS):
        ms, nt, na = ctypes.c_double(), ctypes.c_int64(), ctypes.c_int64()
        _check(lib().dk_profile_read(ctx.handle, k, ctypes.byref(ms), ctypes.byref(nt), ctypes.byref(na)),
               "dk_profile_read")
        out[name] = (ms.value, nt.value, na.value)
    return out


def new_verdict(device: int = 0) -> torch.Tensor:
    """Device storage for one dk_verdict."""
    return torch.zeros(VERDICT_BYTES, dtype=torch.uint8, device=f"cuda:{device}")


def read_verdict(v: torch.Tensor) -> dict:
    """Synchronising device->host read of a dk_verdict."""
    raw = v.cpu().numpy().tobytes()
    s = dk_verdict.from_buffer_copy(raw)
    return {"ok": int(s.ok), "n_flagged": int(s.n_flagged), "first_index": int(s.first_index),
            "max_ratio": float(s.max_ratio), "status": int(s.status)}


def dk_encode(ctx: Context, p: dk_problem, x, r, C: np.ndarray, xbar):
    _check(lib().dk_encode(ctx.handle, ctypes.byref(p), _dev(ctx, x), _dev(ctx, r), _host(C), _dev(ctx, xbar),
                           _stream(ctx)), "dk_encode")


def dk_linear_fwd(ctx: Context, p: dk_problem, W, xbar, ybar):
    _check(lib().dk_linear_fwd(ctx.handle, ctypes.byref(p), _dev(ctx, W), _dev(ctx, xbar), _dev(ctx, ybar),
                               _stream(ctx)), "dk_linear_fwd")


def dk_decode_verify(ctx: Context, p: dk_problem, ybar, C: np.ndarray, bias, y, verdict):
    _check(lib().dk_decode_verify(ctx.handle, ctypes.byref(p), _dev(ctx, ybar), _host(C), _dev(ctx, bias),
                                  _dev(ctx, y), ctypes.c_void_p(verdict.data_ptr()), _stream(ctx)),
           "dk_decode_verify")


def dk_decode_verify_static(device: int, p: dk_problem, ybar, C: np.ndarray, bias, y, verdict):
    """Same result as dk_decode_verify, for callers that may not allocate: no
    context, scratch in a fixed array inside the library (see include/dk.h)."""
    on = SimpleNamespace(device=device)
    _check(lib().dk_decode_verify_static(device, ctypes.byref(p), _dev(on, ybar), _host(C), _dev(on, bias),
                                         _dev(on, y), ctypes.c_void_p(verdict.data_ptr()), _stream(on)),
           "dk_decode_verify_static")


def dk_device_status(ctx: Context) -> int:
    """Synchronises and returns (then clears) the status raised on the device by
    calls that have no verdict (0 = none)."""
    v = ctypes.c_int32()
    _check(lib().dk_device_status(ctx.handle, ctypes.byref(v)), "dk_device_status")
    return v.value


def dk_masked_linear(ctx: Context, p: dk_problem, W, x, r, C: np.ndarray, bias, y, xbar_save, verdict,
                     fault: Optional[dk_fault] = None):
    fp = ctypes.byref(fault) if fault is not None else None
    _check(lib().dk_masked_linear(ctx.handle, ctypes.byref(p), _dev(ctx, W), _dev(ctx, x), _dev(ctx, r), _host(C),
                                  _dev(ctx, bias), _dev(ctx, y), _dev(ctx, xbar_save),
                                  ctypes.c_void_p(verdict.data_ptr()), fp, _stream(ctx)), "dk_masked_linear")


def dk_linear_bwd_wgrad_verify(ctx: Context, p: dk_problem, delta, xbar, C: np.ndarray, gamma: np.ndarray,
                               scale: float, tol_w: float, dW, verdict, fault=None):
    fp = ctypes.byref(fault) if fault is not None else None
    _check(lib().dk_linear_bwd_wgrad_verify(ctx.handle, ctypes.byref(p), _dev(ctx, delta), _dev(ctx, xbar), _host(C),
                                            _host(gamma), ctypes.c_float(scale), ctypes.c_float(tol_w), _dev(ctx, dW),
                                            ctypes.c_void_p(verdict.data_ptr()), fp, _stream(ctx)),
           "dk_linear_bwd_wgrad_verify")


def dk_linear_bwd_wgrad(ctx: Context, p: dk_problem, delta, xbar, xbar_rows: int, C: np.ndarray,
                        gamma: np.ndarray, scale: float, dW):
    _check(lib().dk_linear_bwd_wgrad(ctx.handle, ctypes.byref(p), _dev(ctx, delta), _dev(ctx, xbar), xbar_rows,
                                     _host(C), _host(gamma), ctypes.c_float(scale), _dev(ctx, dW), _stream(ctx)),
           "dk_linear_bwd_wgrad")


def dk_linear_bwd_wgrad_accumulate(ctx: Context, p: dk_problem, delta, xbar, xbar_rows: int, C: np.ndarray,
                                   gamma: np.ndarray, scale: float, dW):
    _check(lib().dk_linear_bwd_wgrad_accumulate(ctx.handle, ctypes.byref(p), _dev(ctx, delta), _dev(ctx, xbar),
                                                xbar_rows, _host(C), _host(gamma), ctypes.c_float(scale),
                                                _dev(ctx, dW), _stream(ctx)), "dk_linear_bwd_wgrad_accumulate")


def dk_linear_bwd_dgrad(ctx: Context, p: dk_problem, W, delta, dx):
    _check(lib().dk_linear_bwd_dgrad(ctx.handle, ctypes.byref(p), _dev(ctx, W), _dev(ctx, delta), _dev(ctx, dx),
                                     _stream(ctx)), "dk_linear_bwd_dgrad")


def dk_relu_pool_fwd(ctx: Context, x, n: int, h: int, w: int, c: int, pool: bool, y):
    _check(lib().dk_relu_pool_fwd(ctx.handle, _dev(ctx, x), n, h, w, c, int(pool), _dev(ctx, y), _stream(ctx)),
           "dk_relu_pool_fwd")


def dk_relu_pool_bwd(ctx: Context, dy, x, n: int, h: int, w: int, c: int, pool: bool, dx):
    _check(lib().dk_relu_pool_bwd(ctx.handle, _dev(ctx, dy), _dev(ctx, x), n, h, w, c, int(pool), _dev(ctx, dx),
                                  _stream(ctx)), "dk_relu_pool_bwd")


# ---------------------------------------------------------------------------
# finite-field calls: residues are int32 CUDA tensors holding values in [0, p)
# (the library reads them as uint32), coefficient arrays NumPy uint32 on the host
# ---------------------------------------------------------------------------
def _res(ctx, t: Optional[torch.Tensor]):
    if t is None:
        return None
    if not (t.get_device() == ctx.device and t.dtype == torch.int32 and t.is_contiguous()):
        raise ValueError(f"expected a contiguous int32 tensor of residues on CUDA device {ctx.device}")
    return ctypes.c_void_p(t.data_ptr())


def _host_u32(a: np.ndarray):
    if not (isinstance(a, np.ndarray) and a.dtype == np.uint32 and a.flags["C_CONTIGUOUS"]):
        raise ValueError("expected a C-contiguous uint32 NumPy array")
    return ctypes.c_void_p(a.ctypes.data)


def dk_field_quantize(ctx: Context, v, scale_bits: int, prime: int, vq):
    _check(lib().dk_field_quantize(ctx.handle, _dev(ctx, v), v.numel(), scale_bits, prime, _res(ctx, vq),
                                   _stream(ctx)), "dk_field_quantize")


def dk_field_dequantize(ctx: Context, vq, scale_bits: int, prime: int, v):
    _check(lib().dk_field_dequantize(ctx.handle, _res(ctx, vq), vq.numel(), scale_bits, prime, _dev(ctx, v),
                                     _stream(ctx)), "dk_field_dequantize")


def dk_field_encode(ctx: Context, p: dk_problem, prime: int, xq, rq, C: np.ndarray, xbar):
    _check(lib().dk_field_encode(ctx.handle, ctypes.byref(p), prime, _res(ctx, xq), _res(ctx, rq), _host_u32(C),
                                 _res(ctx, xbar), _stream(ctx)), "dk_field_encode")


def dk_field_linear_fwd(ctx: Context, p: dk_problem, prime: int, Wq, xbar, ybar):
    _check(lib().dk_field_linear_fwd(ctx.handle, ctypes.byref(p), prime, _res(ctx, Wq), _res(ctx, xbar),
                                     _res(ctx, ybar), _stream(ctx)), "dk_field_linear_fwd")


def dk_field_decode_verify(ctx: Context, p: dk_problem, prime: int, l: int, ybar, C: np.ndarray, bias_q, yq, y,
                           verdict):
    _check(lib().dk_field_decode_verify(ctx.handle, ctypes.byref(p), prime, l, _res(ctx, ybar), _host_u32(C),
                                        _res(ctx, bias_q), _res(ctx, yq), _dev(ctx, y),
                                        ctypes.c_void_p(verdict.data_ptr()), _stream(ctx)), "dk_field_decode_verify")


def dk_field_masked_linear(ctx: Context, p: dk_problem, prime: int, l: int, W, x, rq, C: np.ndarray, bias, y, yq,
                           xbar_save, verdict, fault: Optional[dk_field_fault] = None):
    fp = ctypes.byref(fault) if fault is not None else None
    _check(lib().dk_field_masked_linear(ctx.handle, ctypes.byref(p), prime, l, _dev(ctx, W), _dev(ctx, x),
                                        _res(ctx, rq), _host_u32(C), _dev(ctx, bias), _dev(ctx, y), _res(ctx, yq),
                                        _res(ctx, xbar_save), ctypes.c_void_p(verdict.data_ptr()), fp,
                                        _stream(ctx)), "dk_field_masked_linear")


def dk_field_linear_bwd_wgrad(ctx: Context, p: dk_problem, prime: int, deltaq, xbar, xbar_rows: int, C: np.ndarray,
                              gamma: np.ndarray, dWq):
    _check(lib().dk_field_linear_bwd_wgrad(ctx.handle, ctypes.byref(p), prime, _res(ctx, deltaq), _res(ctx, xbar),
                                           xbar_rows, _host_u32(C), _host_u32(gamma), _res(ctx, dWq), _stream(ctx)),
           "dk_field_linear_bwd_wgrad")


# ---------------------------------------------------------------------------
# the rest of a training step: group normalisation with activation, linear layer with softmax cross entropy,
# orthogonalised update.  x, y, h, W and their gradients are fp32 or bf16 as the descriptor's dtype says,
# parameters, statistics and losses fp32, targets int64.
# ---------------------------------------------------------------------------
_STEP_TYPES = {DK_F32: torch.float32, DK_BF16: torch.bfloat16}


def _typed(ctx, t: torch.Tensor, dtype: int, numel: int, what: str) -> int:
    if (t.dtype is not _STEP_TYPES.get(dtype) or t.numel() != numel or not t.is_contiguous()
            or t.get_device() != ctx.device):
        raise ValueError(f"{what}: expected a contiguous {_STEP_TYPES.get(dtype)} tensor of {numel} elements on CUDA "
                         f"device {ctx.device}")
    return t.data_ptr()


def _f32(ctx, t: torch.Tensor, numel: int, what: str):
    return _typed(ctx, t, DK_F32, numel, what)


def _norm_sizes(q: dk_norm):
    n, c = q.n, q.c
    return n * q.h * q.w * c, c, n * q.groups * 2


def dk_group_norm_fwd(ctx: Context, q: dk_norm, x, gamma, beta, y, stats):
    e, c, s = _norm_sizes(q)
    _check(lib().dk_group_norm_fwd(ctx.handle, ctypes.byref(q), _typed(ctx, x, q.dtype, e, "x"),
                                   _f32(ctx, gamma, c, "gamma"), _f32(ctx, beta, c, "beta"),
                                   _typed(ctx, y, q.dtype, e, "y"), _f32(ctx, stats, s, "stats"),
                                   _raw_stream(ctx.device)), "dk_group_norm_fwd")


def dk_group_norm_bwd(ctx: Context, q: dk_norm, dy, x, gamma, beta, stats, dx, dgamma, dbeta):
    e, c, s = _norm_sizes(q)
    _check(lib().dk_group_norm_bwd(ctx.handle, ctypes.byref(q), _typed(ctx, dy, q.dtype, e, "dy"),
                                   _typed(ctx, x, q.dtype, e, "x"), _f32(ctx, gamma, c, "gamma"),
                                   _f32(ctx, beta, c, "beta"), _f32(ctx, stats, s, "stats"),
                                   _typed(ctx, dx, q.dtype, e, "dx"), _f32(ctx, dgamma, c, "dgamma"),
                                   _f32(ctx, dbeta, c, "dbeta"), _raw_stream(ctx.device)), "dk_group_norm_bwd")


def _targets(ctx, t: torch.Tensor, rows: int):
    if not (t.get_device() == ctx.device and t.dtype == torch.int64 and t.is_contiguous() and t.numel() == rows):
        raise ValueError(f"target: expected a contiguous int64 tensor of {rows} elements on CUDA device {ctx.device}")
    return t.data_ptr()


def dk_linear_xent_fwd(ctx: Context, q: dk_xent, h, W, target, loss, lse):
    _check(lib().dk_linear_xent_fwd(ctx.handle, ctypes.byref(q), _typed(ctx, h, q.dtype, q.rows * q.d, "h"),
                                    _typed(ctx, W, q.dtype, q.vocab * q.d, "W"), _targets(ctx, target, q.rows),
                                    _f32(ctx, loss, q.rows, "loss"), _f32(ctx, lse, q.rows, "lse"),
                                    _raw_stream(ctx.device)), "dk_linear_xent_fwd")


def dk_linear_xent_bwd(ctx: Context, q: dk_xent, h, W, target, lse, dloss: Optional[torch.Tensor], scale: float, dh,
                       dW):
    _check(lib().dk_linear_xent_bwd(ctx.handle, ctypes.byref(q), _typed(ctx, h, q.dtype, q.rows * q.d, "h"),
                                    _typed(ctx, W, q.dtype, q.vocab * q.d, "W"), _targets(ctx, target, q.rows),
                                    _f32(ctx, lse, q.rows, "lse"),
                                    None if dloss is None else _f32(ctx, dloss, q.rows, "dloss"), scale,
                                    _typed(ctx, dh, q.dtype, q.rows * q.d, "dh"),
                                    _typed(ctx, dW, q.dtype, q.vocab * q.d, "dW"), _raw_stream(ctx.device)),
           "dk_linear_xent_bwd")


def dk_orthogonalize(ctx: Context, q: dk_ortho, x, scale: float, keep: float, out):
    e = q.batch * q.m * q.n
    _check(lib().dk_orthogonalize(ctx.handle, ctypes.byref(q), _typed(ctx, x, q.dtype, e, "x"), scale,
                                  keep, _typed(ctx, out, q.dtype, e, "out"), _raw_stream(ctx.device)),
           "dk_orthogonalize")


# ---------------------------------------------------------------------------
# what is kept between the two directions in 8 bits, and the norms between two residual blocks: checkpoints are uint8
# tensors of dk_ckpt8_bytes
# ---------------------------------------------------------------------------
# (A token between two blocks takes the GPU 4 us; what a call checks of its tensors is kept to four attributes each, and the
# function is looked up once.)
def _ptr(t: torch.Tensor, dtype, numel: int, device: int, what: str) -> int:
    if t.dtype is not dtype or t.numel() != numel or t.get_device() != device or not t.is_contiguous():
        raise ValueError(f"{what}: expected a contiguous {dtype} tensor of {numel} elements on CUDA device {device}")
    return t.data_ptr()


def _kept_numel(rows: int, d: int) -> int:
    blocks = (d + 31) // 32
    return rows * blocks * 33


_functions = {}


def _call(name: str, *args):
    f = _functions.get(name)
    if f is None:
        f = _functions[name] = getattr(lib(), name)
    status = f(*args)
    if status:
        raise DkError(status, name)


def dk_ckpt8_bytes(q: dk_ckpt8) -> int:
    n = ctypes.c_size_t()
    _call("dk_ckpt8_bytes", q, n)
    return n.value


def dk_ckpt8_store(ctx: Context, q: dk_ckpt8, x, ckpt):
    dev, rows, d = ctx.device, q.rows, q.d
    _call("dk_ckpt8_store", ctx.handle, q, _ptr(x, _STEP_TYPES.get(q.dtype), rows * d, dev, "x"),
          _ptr(ckpt, torch.uint8, _kept_numel(rows, d), dev, "ckpt"), _raw_stream(dev))


def dk_ckpt8_load(ctx: Context, q: dk_ckpt8, ckpt, x):
    dev, rows, d = ctx.device, q.rows, q.d
    _call("dk_ckpt8_load", ctx.handle, q, _ptr(ckpt, torch.uint8, _kept_numel(rows, d), dev, "ckpt"),
          _ptr(x, _STEP_TYPES.get(q.dtype), rows * d, dev, "x"), _raw_stream(dev))


def dk_group_norm_fwd_ckpt8(ctx: Context, q: dk_norm, x, gamma, beta, y, stats, ckpt):
    dev, t, f = ctx.device, _STEP_TYPES.get(q.dtype), torch.float32
    e, c, s = _norm_sizes(q)
    _call("dk_group_norm_fwd_ckpt8", ctx.handle, q, _ptr(x, t, e, dev, "x"), _ptr(gamma, f, c, dev, "gamma"),
          _ptr(beta, f, c, dev, "beta"), _ptr(y, t, e, dev, "y"), _ptr(stats, f, s, dev, "stats"),
          _ptr(ckpt, torch.uint8, _kept_numel(q.n * q.h * q.w, c), dev, "ckpt"), _raw_stream(dev))


def dk_group_norm_bwd_ckpt8(ctx: Context, q: dk_norm, dy, ckpt, gamma, beta, stats, dx, dgamma, dbeta):
    dev, t, f = ctx.device, _STEP_TYPES.get(q.dtype), torch.float32
    e, c, s = _norm_sizes(q)
    _call("dk_group_norm_bwd_ckpt8", ctx.handle, q, _ptr(dy, t, e, dev, "dy"),
          _ptr(ckpt, torch.uint8, _kept_numel(q.n * q.h * q.w, c), dev, "ckpt"), _ptr(gamma, f, c, dev, "gamma"),
          _ptr(beta, f, c, dev, "beta"), _ptr(stats, f, s, dev, "stats"), _ptr(dx, t, e, dev, "dx"),
          _ptr(dgamma, f, c, dev, "dgamma"), _ptr(dbeta, f, c, dev, "dbeta"), _raw_stream(dev))


def dk_linear_bwd_wgrad_ckpt8(ctx: Context, q: dk_wgrad8, dy, ckpt, scale: float, keep: float, dW,
                              db: Optional[torch.Tensor]):
    dev, f, rows, d, out = ctx.device, torch.float32, q.rows, q.d, q.out
    _call("dk_linear_bwd_wgrad_ckpt8", ctx.handle, q, _ptr(dy, _STEP_TYPES.get(q.dtype), rows * out, dev, "dy"),
          _ptr(ckpt, torch.uint8, _kept_numel(rows, d), dev, "ckpt"), scale, keep, _ptr(dW, f, out * d, dev, "dW"),
          None if db is None else _ptr(db, f, out, dev, "db"), _raw_stream(dev))


def _gates(q: dk_block) -> int:
    return -(-q.rows // q.rows_per_gate) * q.d if q.rows_per_gate > 0 else -1


def dk_block_norm_fwd(ctx: Context, q: dk_block, h, u, gate, post, pre, shift, h_out, n, stats, ckpt_h=None, ckpt_u=None):
    """Every tensor but h may be None where the C call takes NULL."""
    dev, rows, d, t, f = ctx.device, q.rows, q.d, _STEP_TYPES.get(q.dtype), torch.float32
    e = rows * d
    _call("dk_block_norm_fwd", ctx.handle, q, _ptr(h, t, e, dev, "h"), None if u is None else _ptr(u, t, e, dev, "u"),
          None if gate is None else _ptr(gate, f, _gates(q), dev, "gate"),
          None if post is None else _ptr(post, f, d, dev, "post"), None if pre is None else _ptr(pre, f, d, dev, "pre"),
          None if shift is None else _ptr(shift, f, d, dev, "shift"),
          None if h_out is None else _ptr(h_out, t, e, dev, "h_out"), None if n is None else _ptr(n, t, e, dev, "n"),
          None if stats is None else _ptr(stats, f, 4 * rows, dev, "stats"),
          None if ckpt_h is None else _ptr(ckpt_h, torch.uint8, _kept_numel(rows, d), dev, "ckpt_h"),
          None if ckpt_u is None else _ptr(ckpt_u, torch.uint8, _kept_numel(rows, d), dev, "ckpt_u"), _raw_stream(dev))


def _block_bwd(name, held, held_numel, ctx, q, dh_out, dn, h, u, gate, post, pre, stats, dh, du, dgate, dpost, dpre, dshift):
    dev, rows, d, t, f = ctx.device, q.rows, q.d, _STEP_TYPES.get(q.dtype), torch.float32
    e = rows * d
    _call(name, ctx.handle, q, None if dh_out is None else _ptr(dh_out, t, e, dev, "dh_out"),
          None if dn is None else _ptr(dn, t, e, dev, "dn"), _ptr(h, held, held_numel, dev, "h"),
          None if u is None else _ptr(u, held, held_numel, dev, "u"),
          None if gate is None else _ptr(gate, f, _gates(q), dev, "gate"),
          None if post is None else _ptr(post, f, d, dev, "post"), None if pre is None else _ptr(pre, f, d, dev, "pre"),
          _ptr(stats, f, 4 * rows, dev, "stats"), _ptr(dh, t, e, dev, "dh"),
          None if du is None else _ptr(du, t, e, dev, "du"), None if dgate is None else _ptr(dgate, f, _gates(q), dev, "dgate"),
          None if dpost is None else _ptr(dpost, f, d, dev, "dpost"), None if dpre is None else _ptr(dpre, f, d, dev, "dpre"),
          None if dshift is None else _ptr(dshift, f, d, dev, "dshift"), _raw_stream(dev))


def dk_block_norm_bwd(ctx: Context, q: dk_block, dh_out, dn, h, u, gate, post, pre, stats, dh, du, dgate, dpost, dpre,
                      dshift):
    _block_bwd("dk_block_norm_bwd", _STEP_TYPES.get(q.dtype), q.rows * q.d, ctx, q, dh_out, dn, h, u, gate, post, pre, stats,
               dh, du, dgate, dpost, dpre, dshift)


def dk_block_norm_bwd_ckpt8(ctx: Context, q: dk_block, dh_out, dn, ckpt_h, ckpt_u, gate, post, pre, stats, dh, du, dgate,
                            dpost, dpre, dshift):
    _block_bwd("dk_block_norm_bwd_ckpt8", torch.uint8, _kept_numel(q.rows, q.d), ctx, q, dh_out, dn, ckpt_h, ckpt_u, gate,
               post, pre, stats, dh, du, dgate, dpost, dpre, dshift)
