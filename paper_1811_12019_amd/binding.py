"""ctypes binding of the K-FAC C ABI (include/kfac.h).  Argument marshalling only.

Every function here has the name and argument order of the C entry point it calls; tensors are
torch device tensors used purely as owned device memory (``data_ptr()``), and the stream is torch's
current HIP stream unless one is given.  Nothing is computed in Python, and there is no fallback:
if the compiled library is missing, loading raises.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional, Sequence

import torch

from . import synth

PKG_DIR = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(PKG_DIR, "libkfac_hip.so")

KFAC_OK = 0
KFAC_ERR_INVALID_ARG, KFAC_ERR_UNSUPPORTED, KFAC_ERR_WORKSPACE, KFAC_ERR_HIP, KFAC_ERR_TOO_LARGE = -1, -2, -3, -4, -5
KFAC_F32, KFAC_BF16, KFAC_F16 = 0, 1, 2
KFAC_NCHW, KFAC_NHWC = 0, 1
KFAC_ORDER_C_KH_KW, KFAC_ORDER_KH_KW_C = 0, 1
KFAC_OP_FACTOR_A, KFAC_OP_FACTOR_G = 0, 1

EXPORTED_SYMBOLS = (
    "kfac_status_string", "kfac_factor_workspace_bytes", "kfac_factor_A", "kfac_factor_G", "kfac_factor_batched",
    "kfac_ema", "kfac_ema_batched", "kfac_pack_upper_batched", "kfac_ema_packed_batched",
    "kfac_factor_diff_workspace_bytes", "kfac_factor_diff_batched", "kfac_factor_diff_batched_noalloc",
    "kfac_factor_diff_noalloc_max_elements",
    "kfac_weight_update_workspace_bytes", "kfac_weight_update_batched",
    "kfac_grad_norm_workspace_bytes", "kfac_grad_norm_batched", "kfac_grad_clip_batched",
    "kfac_expert_sort_workspace_bytes", "kfac_expert_sort", "kfac_expert_dispatch", "kfac_expert_combine",
    "kfac_expert_combine_backward", "kfac_expert_factor_workspace_bytes", "kfac_expert_factor",
    "kfac_bn_sample_grads_workspace_bytes", "kfac_bn_sample_grads", "kfac_bn_diag_precondition",
    "kfac_bn_sample_grads_batched_workspace_bytes", "kfac_bn_sample_grads_batched",
    "kfac_inverse_workspace_bytes", "kfac_inverse_planes_bytes", "kfac_damped_inverse", "kfac_damped_inverse_batched",
    "kfac_pi_damping_batched", "kfac_warmup_damping_alpha", "kfac_warmup_damping_next", "kfac_bn_damping",
    "kfac_refresh_interval",
    "kfac_precondition_workspace_bytes", "kfac_precondition", "kfac_precondition_batched",
    "kfac_kernel_timing_enable", "kfac_kernel_timing_report", "kfac_probe_mfma", "kfac_probe_copy", "kfac_probe_read",
)


class kfac_layer_desc(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in
                ("N", "C_in", "H", "W", "C_out", "kh", "kw", "stride", "pad", "has_bias", "layout", "dtype", "order")]


class kfac_factor_item(ctypes.Structure):
    _fields_ = [("desc", kfac_layer_desc), ("x", ctypes.c_void_p), ("out", ctypes.c_void_p), ("ws", ctypes.c_void_p),
                ("ws_bytes", ctypes.c_size_t), ("scale", ctypes.c_float), ("op", ctypes.c_int32),
                ("running", ctypes.c_void_p), ("decay", ctypes.c_float), ("packed", ctypes.c_int32)]


class kfac_ema_item(ctypes.Structure):
    _fields_ = [("running", ctypes.c_void_p), ("fresh", ctypes.c_void_p), ("dim", ctypes.c_int32)]


class kfac_pack_item(ctypes.Structure):
    _fields_ = [("full", ctypes.c_void_p), ("packed", ctypes.c_void_p), ("dim", ctypes.c_int32)]


class kfac_ema_packed_item(ctypes.Structure):
    _fields_ = [("running", ctypes.c_void_p), ("packed_fresh", ctypes.c_void_p), ("dim", ctypes.c_int32)]


class kfac_diff_item(ctypes.Structure):
    _fields_ = [("x", ctypes.c_void_p), ("x_prev", ctypes.c_void_p), ("dim", ctypes.c_int32)]


class kfac_bn_item(ctypes.Structure):
    _fields_ = [("xhat", ctypes.c_void_p), ("gout", ctypes.c_void_p), ("g", ctypes.c_void_p), ("N", ctypes.c_int32),
                ("C", ctypes.c_int32), ("HW", ctypes.c_int32), ("dtype", ctypes.c_int32)]


class kfac_update_item(ctypes.Structure):
    _fields_ = [("w", ctypes.c_void_p), ("w_prev", ctypes.c_void_p), ("precond", ctypes.c_void_p),
                ("n", ctypes.c_int32), ("d_out", ctypes.c_int32)]


class kfac_grad_item(ctypes.Structure):
    _fields_ = [("g", ctypes.c_void_p), ("out", ctypes.c_void_p), ("n", ctypes.c_int64), ("dtype", ctypes.c_int32)]


class kfac_expert_desc(ctypes.Structure):
    _fields_ = ([(n, ctypes.c_int32) for n in ("tokens", "choices", "experts", "dim", "dtype")] +
                [(n, ctypes.c_int64) for n in ("ld_token", "ld_row", "ld_grad")])


class kfac_expert_factor_desc(ctypes.Structure):
    _fields_ = ([(n, ctypes.c_int32) for n in ("rows", "experts", "dim", "dtype", "has_bias", "packed")] +
                [("ld", ctypes.c_int64)])


class kfac_inverse_item(ctypes.Structure):
    _fields_ = [("S", ctypes.c_void_p), ("Minv", ctypes.c_void_p), ("ws", ctypes.c_void_p), ("info", ctypes.c_void_p),
                ("dim", ctypes.c_int32), ("damping", ctypes.c_float), ("damping_dev", ctypes.c_void_p),
                ("planes", ctypes.c_void_p)]


class kfac_pi_item(ctypes.Structure):
    _fields_ = [("A", ctypes.c_void_p), ("G", ctypes.c_void_p), ("dA", ctypes.c_int32), ("dG", ctypes.c_int32)]


class kfac_precond_item(ctypes.Structure):
    _fields_ = [("Ginv", ctypes.c_void_p), ("Ainv", ctypes.c_void_p), ("gradW", ctypes.c_void_p),
                ("out", ctypes.c_void_p), ("ws", ctypes.c_void_p), ("dG", ctypes.c_int32), ("dA", ctypes.c_int32),
                ("Ginv_planes", ctypes.c_void_p), ("Ainv_planes", ctypes.c_void_p)]


class KfacError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {status_string(status)} ({status})")


_lib = None


def load_library() -> ctypes.CDLL:
    """Load libkfac_hip.so (built by paper_1811_12019_amd.build / __graft_entry__.build)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise FileNotFoundError(
            f"{LIB_PATH} is missing: build it first (python -m paper_1811_12019_amd.build). "
            "There is no CPU fallback.")
    lib = ctypes.CDLL(LIB_PATH)
    vp, sz, i32, f32 = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int32, ctypes.c_float
    descp = ctypes.POINTER(kfac_layer_desc)
    itemp = ctypes.POINTER(kfac_inverse_item)
    lib.kfac_status_string.restype = ctypes.c_char_p
    lib.kfac_status_string.argtypes = [ctypes.c_int]
    lib.kfac_factor_workspace_bytes.restype = sz
    lib.kfac_factor_workspace_bytes.argtypes = [ctypes.c_int, descp]
    for name in ("kfac_factor_A", "kfac_factor_G"):
        fn = getattr(lib, name)
        fn.restype = ctypes.c_int
        fn.argtypes = [descp, vp, f32, vp, vp, sz, vp]
    lib.kfac_factor_batched.restype = ctypes.c_int
    lib.kfac_factor_batched.argtypes = [ctypes.POINTER(kfac_factor_item), vp, i32, vp]
    lib.kfac_ema.restype = ctypes.c_int
    lib.kfac_ema.argtypes = [vp, vp, i32, f32, vp]
    lib.kfac_ema_batched.restype = ctypes.c_int
    lib.kfac_ema_batched.argtypes = [ctypes.POINTER(kfac_ema_item), i32, f32, vp]
    lib.kfac_pack_upper_batched.restype = ctypes.c_int
    lib.kfac_pack_upper_batched.argtypes = [ctypes.POINTER(kfac_pack_item), i32, vp]
    lib.kfac_ema_packed_batched.restype = ctypes.c_int
    lib.kfac_ema_packed_batched.argtypes = [ctypes.POINTER(kfac_ema_packed_item), i32, f32, vp]
    lib.kfac_factor_diff_workspace_bytes.restype = sz
    lib.kfac_factor_diff_workspace_bytes.argtypes = [ctypes.POINTER(kfac_diff_item), i32]
    lib.kfac_factor_diff_batched.restype = ctypes.c_int
    lib.kfac_factor_diff_batched.argtypes = [ctypes.POINTER(kfac_diff_item), i32, vp, vp, sz, vp]
    lib.kfac_factor_diff_batched_noalloc.restype = ctypes.c_int
    lib.kfac_factor_diff_batched_noalloc.argtypes = [ctypes.POINTER(kfac_diff_item), i32, vp, vp]
    lib.kfac_factor_diff_noalloc_max_elements.restype = sz
    lib.kfac_factor_diff_noalloc_max_elements.argtypes = []
    lib.kfac_weight_update_workspace_bytes.restype = sz
    lib.kfac_weight_update_workspace_bytes.argtypes = [ctypes.POINTER(kfac_update_item), i32]
    lib.kfac_weight_update_batched.restype = ctypes.c_int
    lib.kfac_weight_update_batched.argtypes = [ctypes.POINTER(kfac_update_item), i32, f32, f32, f32, vp, sz, vp]
    lib.kfac_grad_norm_workspace_bytes.restype = sz
    lib.kfac_grad_norm_workspace_bytes.argtypes = [ctypes.POINTER(kfac_grad_item), i32]
    lib.kfac_grad_norm_batched.restype = ctypes.c_int
    lib.kfac_grad_norm_batched.argtypes = [ctypes.POINTER(kfac_grad_item), i32, vp, vp, sz, vp]
    lib.kfac_grad_clip_batched.restype = ctypes.c_int
    lib.kfac_grad_clip_batched.argtypes = [ctypes.POINTER(kfac_grad_item), i32, f32, vp, vp, vp, sz, vp]
    expertp, efactorp = ctypes.POINTER(kfac_expert_desc), ctypes.POINTER(kfac_expert_factor_desc)
    lib.kfac_expert_sort_workspace_bytes.restype = sz
    lib.kfac_expert_sort_workspace_bytes.argtypes = [expertp]
    lib.kfac_expert_sort.restype = ctypes.c_int
    lib.kfac_expert_sort.argtypes = [expertp, vp, vp, vp, vp, vp, sz, vp]
    lib.kfac_expert_dispatch.restype = ctypes.c_int
    lib.kfac_expert_dispatch.argtypes = [expertp, vp, vp, vp, vp]
    lib.kfac_expert_combine.restype = ctypes.c_int
    lib.kfac_expert_combine.argtypes = [expertp, vp, vp, vp, vp, vp]
    lib.kfac_expert_combine_backward.restype = ctypes.c_int
    lib.kfac_expert_combine_backward.argtypes = [expertp, vp, vp, vp, vp, vp, vp, vp]
    lib.kfac_expert_factor_workspace_bytes.restype = sz
    lib.kfac_expert_factor_workspace_bytes.argtypes = [efactorp]
    lib.kfac_expert_factor.restype = ctypes.c_int
    lib.kfac_expert_factor.argtypes = [efactorp, vp, vp, f32, vp, vp, f32, vp, sz, vp]
    lib.kfac_bn_sample_grads_workspace_bytes.restype = sz
    lib.kfac_bn_sample_grads_workspace_bytes.argtypes = [i32, i32, i32]
    lib.kfac_bn_sample_grads.restype = ctypes.c_int
    lib.kfac_bn_sample_grads.argtypes = [vp, vp, i32, i32, i32, i32, vp, vp, sz, vp]
    lib.kfac_bn_sample_grads_batched_workspace_bytes.restype = sz
    lib.kfac_bn_sample_grads_batched_workspace_bytes.argtypes = [ctypes.POINTER(kfac_bn_item), i32]
    lib.kfac_bn_sample_grads_batched.restype = ctypes.c_int
    lib.kfac_bn_sample_grads_batched.argtypes = [ctypes.POINTER(kfac_bn_item), i32, vp, sz, vp]
    lib.kfac_bn_diag_precondition.restype = ctypes.c_int
    lib.kfac_bn_diag_precondition.argtypes = [vp, i32, i32, vp, f32, vp, vp, vp]
    lib.kfac_inverse_workspace_bytes.restype = sz
    lib.kfac_inverse_workspace_bytes.argtypes = [i32]
    lib.kfac_inverse_planes_bytes.restype = sz
    lib.kfac_inverse_planes_bytes.argtypes = [i32]
    lib.kfac_damped_inverse.restype = ctypes.c_int
    lib.kfac_damped_inverse.argtypes = [vp, i32, f32, vp, vp, vp, sz, vp]
    lib.kfac_damped_inverse_batched.restype = ctypes.c_int
    lib.kfac_damped_inverse_batched.argtypes = [itemp, i32, vp]
    lib.kfac_pi_damping_batched.restype = ctypes.c_int
    lib.kfac_pi_damping_batched.argtypes = [ctypes.POINTER(kfac_pi_item), i32, f32, vp, vp]
    f64 = ctypes.c_double
    lib.kfac_warmup_damping_alpha.restype = f64
    lib.kfac_warmup_damping_alpha.argtypes = [f64, f64, f64]
    lib.kfac_warmup_damping_next.restype = f64
    lib.kfac_warmup_damping_next.argtypes = [f64, f64, f64]
    lib.kfac_bn_damping.restype = f64
    lib.kfac_bn_damping.argtypes = [f64, f64]
    lib.kfac_refresh_interval.restype = i32
    lib.kfac_refresh_interval.argtypes = [i32, i32]
    lib.kfac_precondition_workspace_bytes.restype = sz
    lib.kfac_precondition_workspace_bytes.argtypes = [i32, i32]
    lib.kfac_precondition.restype = ctypes.c_int
    lib.kfac_precondition.argtypes = [vp, vp, vp, i32, i32, vp, vp, sz, vp]
    lib.kfac_precondition_batched.restype = ctypes.c_int
    lib.kfac_precondition_batched.argtypes = [ctypes.POINTER(kfac_precond_item), vp, i32, vp]
    lib.kfac_kernel_timing_enable.restype = ctypes.c_int
    lib.kfac_kernel_timing_enable.argtypes = [ctypes.c_int]
    lib.kfac_kernel_timing_report.restype = ctypes.c_int
    lib.kfac_kernel_timing_report.argtypes = [ctypes.c_char_p, sz]
    lib.kfac_probe_mfma.restype = ctypes.c_int
    lib.kfac_probe_mfma.argtypes = [i32, i32, i32, vp, vp]
    lib.kfac_probe_copy.restype = ctypes.c_int
    lib.kfac_probe_copy.argtypes = [vp, vp, sz, i32, vp]
    lib.kfac_probe_read.restype = ctypes.c_int
    lib.kfac_probe_read.argtypes = [vp, vp, sz, i32, vp]
    _lib = lib
    return lib


def status_string(status: int) -> str:
    return load_library().kfac_status_string(int(status)).decode()


def _check(status: int, where: str) -> None:
    if status != KFAC_OK:
        raise KfacError(status, where)


def _stream(stream) -> int:
    if stream is not None:
        return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)
    # The current stream's handle without a Stream object around it (0.2 us instead of 2.8 us on every call), where this torch
    # has the two functions for that: they are not part of its public interface.
    raw, device = getattr(torch._C, "_cuda_getCurrentRawStream", None), getattr(torch._C, "_cuda_getDevice", None)
    if raw is None or device is None or not torch.cuda.is_initialized():
        return torch.cuda.current_stream().cuda_stream
    return raw(device())


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


_TORCH_DTYPE = {KFAC_F32: torch.float32, KFAC_BF16: torch.bfloat16, KFAC_F16: torch.float16}


def make_desc(shape: "synth.LayerShape", layout: int, dtype: int, order: int) -> kfac_layer_desc:
    return kfac_layer_desc(shape.N, shape.C_in, shape.H, shape.W, shape.C_out, shape.kh, shape.kw, shape.stride,
                           shape.pad, int(shape.has_bias), layout, dtype, order)


def to_device_tensor(x_nchw, layout: int, dtype: int, device="cuda") -> torch.Tensor:
    """Place a logical (n, c, y, x) array in device memory in the given layout and dtype (contiguous)."""
    t = torch.as_tensor(x_nchw)
    if layout == KFAC_NHWC:
        t = t.permute(0, 2, 3, 1)
    return t.contiguous().to(device=device, dtype=_TORCH_DTYPE[dtype]).contiguous()


def alloc_workspace(nbytes: int, device="cuda") -> Optional[torch.Tensor]:
    """Device scratch of at least nbytes (torch's allocator hands out 512-byte aligned blocks)."""
    if nbytes <= 0:
        return None
    return torch.empty(int(nbytes), dtype=torch.uint8, device=device)


# ------------------------------------------------------------------------------------------------
# entry points, same names as the C ABI
# ------------------------------------------------------------------------------------------------
def kfac_factor_workspace_bytes(op: int, desc: kfac_layer_desc) -> int:
    return int(load_library().kfac_factor_workspace_bytes(op, ctypes.byref(desc)))


def _factor(name: str, op: int, desc, x, scale, out, ws, stream):
    lib = load_library()
    ws_bytes = 0 if ws is None else ws.numel() * ws.element_size()
    rc = getattr(lib, name)(ctypes.byref(desc), _ptr(x), float(scale), _ptr(out), _ptr(ws), ws_bytes, _stream(stream))
    _check(rc, name)
    return out


def kfac_factor_A(desc: kfac_layer_desc, act: torch.Tensor, scale: float, A: torch.Tensor,
                  ws: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    return _factor("kfac_factor_A", KFAC_OP_FACTOR_A, desc, act, scale, A, ws, stream)


def kfac_factor_G(desc: kfac_layer_desc, gout: torch.Tensor, scale: float, G: torch.Tensor,
                  ws: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    return _factor("kfac_factor_G", KFAC_OP_FACTOR_G, desc, gout, scale, G, ws, stream)


class FactorBatch:
    """Host + device copies of a kfac_factor_item table (built once, reused every step).

    builds: sequence of (op, desc, x tensor, out tensor, scale).
    running: None, or one tensor per build: the build's result is folded into it (running average with `decay`) and the
    out tensor of that build is not written.  packed: the out tensors receive packed upper triangles.
    ws: None (scratch is allocated here), or one scratch tensor (or None where none is needed) per build, at least
    kfac_factor_workspace_bytes(op, desc) bytes each, which tables that never run at the same time may share."""

    def __init__(self, builds, device="cuda", running=None, decay: float = 0.0, packed: bool = False, ws=None):
        n = len(builds)
        self.count = n
        self.ws = (list(ws) if ws is not None else
                   [alloc_workspace(kfac_factor_workspace_bytes(op, desc), device) for op, desc, _, _, _ in builds])
        self.keep = (list(builds), running)
        arr = (kfac_factor_item * n)()
        for i, (op, desc, x, out, scale) in enumerate(builds):
            ws = self.ws[i]
            run = None if running is None else running[i]
            arr[i] = kfac_factor_item(desc, x.data_ptr(), None if run is not None else out.data_ptr(), _ptr(ws),
                                      0 if ws is None else ws.numel(), float(scale), int(op),
                                      _ptr(run), float(decay) if run is not None else 0.0, int(bool(packed)))
        self.host = arr
        self.dev = torch.frombuffer(bytearray(bytes(arr)), dtype=torch.uint8).to(device)


def kfac_factor_batched(batch: FactorBatch, stream=None) -> None:
    rc = load_library().kfac_factor_batched(batch.host, batch.dev.data_ptr(), batch.count, _stream(stream))
    _check(rc, "kfac_factor_batched")


def kfac_ema(running: torch.Tensor, fresh: torch.Tensor, dim: int, decay: float, stream=None) -> torch.Tensor:
    _check(load_library().kfac_ema(_ptr(running), _ptr(fresh), int(dim), float(decay), _stream(stream)), "kfac_ema")
    return running


class EmaBatch:
    """A kfac_ema_item table (host memory; built once, reused every step)."""

    def __init__(self, running: Sequence[torch.Tensor], fresh: Sequence[torch.Tensor]):
        n = len(running)
        self.count = n
        self.keep = (list(running), list(fresh))
        arr = (kfac_ema_item * max(n, 1))()
        for i in range(n):
            arr[i] = kfac_ema_item(running[i].data_ptr(), fresh[i].data_ptr(), int(running[i].shape[0]))
        self.host = arr


def kfac_ema_batched(batch: EmaBatch, decay: float, stream=None) -> None:
    rc = load_library().kfac_ema_batched(batch.host, batch.count, float(decay), _stream(stream))
    _check(rc, "kfac_ema_batched")


def packed_elems(dim: int) -> int:
    return dim * (dim + 1) // 2


class PackBatch:
    """kfac_pack_item / kfac_ema_packed_item tables (host memory) over the same (full, packed) tensor pairs."""

    def __init__(self, full: Sequence[torch.Tensor], packed: Sequence[torch.Tensor]):
        n = len(full)
        self.count = n
        self.keep = (list(full), list(packed))
        self.pack_items = (kfac_pack_item * max(n, 1))()
        self.ema_items = (kfac_ema_packed_item * max(n, 1))()
        for i in range(n):
            d = int(full[i].shape[0])
            assert packed[i].numel() == packed_elems(d)
            self.pack_items[i] = kfac_pack_item(full[i].data_ptr(), packed[i].data_ptr(), d)
            self.ema_items[i] = kfac_ema_packed_item(full[i].data_ptr(), packed[i].data_ptr(), d)


def kfac_pack_upper_batched(batch: PackBatch, stream=None) -> None:
    """packed[i] <- upper triangle of full[i]."""
    _check(load_library().kfac_pack_upper_batched(batch.pack_items, batch.count, _stream(stream)), "kfac_pack_upper_batched")


def kfac_ema_packed_batched(batch: PackBatch, decay: float, stream=None) -> None:
    """full[i] (a running average) <- decay * full[i] + (1 - decay) * unpack(packed[i])."""
    _check(load_library().kfac_ema_packed_batched(batch.ema_items, batch.count, float(decay), _stream(stream)),
           "kfac_ema_packed_batched")


class DiffBatch:
    """A kfac_diff_item table (host memory), its scratch and its device output (one float per matrix)."""

    def __init__(self, x: Sequence[torch.Tensor], x_prev: Sequence[torch.Tensor], device="cuda"):
        n = len(x)
        self.count = n
        self.keep = (list(x), list(x_prev))
        self.host = (kfac_diff_item * max(n, 1))()
        for i in range(n):
            self.host[i] = kfac_diff_item(x[i].data_ptr(), x_prev[i].data_ptr(), int(x[i].shape[0]))
        nbytes = int(load_library().kfac_factor_diff_workspace_bytes(self.host, n)) if n else 0
        self.ws = alloc_workspace(nbytes, device) if nbytes else None
        self.out = torch.zeros(max(n, 1), dtype=torch.float32, device=device)


def kfac_factor_diff_batched(batch: DiffBatch, stream=None) -> torch.Tensor:
    """out[i] = ||x[i] - x_prev[i]||_F / ||x_prev[i]||_F; returns the device tensor of results."""
    ws_bytes = 0 if batch.ws is None else batch.ws.numel() * batch.ws.element_size()
    rc = load_library().kfac_factor_diff_batched(batch.host, batch.count, _ptr(batch.out), _ptr(batch.ws), ws_bytes,
                                                 _stream(stream))
    _check(rc, "kfac_factor_diff_batched")
    return batch.out[:batch.count]


def kfac_factor_diff_batched_noalloc(items_host, count: int, out: torch.Tensor, stream=None) -> torch.Tensor:
    """The same computation with the library's fixed scratch: nothing is allocated (items_host: a kfac_diff_item array)."""
    rc = load_library().kfac_factor_diff_batched_noalloc(items_host, int(count), _ptr(out), _stream(stream))
    _check(rc, "kfac_factor_diff_batched_noalloc")
    return out


def kfac_factor_diff_noalloc_max_elements() -> int:
    return int(load_library().kfac_factor_diff_noalloc_max_elements())


class UpdateBatch:
    """A kfac_update_item table (host memory) and its scratch; d_out of a layer = rows of its weight matrix."""

    def __init__(self, w: Sequence[torch.Tensor], w_prev: Sequence[torch.Tensor], precond: Sequence[torch.Tensor],
                 device="cuda"):
        n = len(w)
        self.count = n
        self.keep = (list(w), list(w_prev), list(precond))
        self.host = (kfac_update_item * max(n, 1))()
        for i in range(n):
            self.host[i] = kfac_update_item(w[i].data_ptr(), w_prev[i].data_ptr(), precond[i].data_ptr(),
                                            int(w[i].numel()), int(w[i].shape[0]))
        nbytes = int(load_library().kfac_weight_update_workspace_bytes(self.host, n)) if n else 0
        self.ws = alloc_workspace(nbytes, device) if nbytes else None


def kfac_weight_update_batched(batch: UpdateBatch, eta: float, momentum: float, eps: float = 1e-9, stream=None) -> None:
    ws_bytes = 0 if batch.ws is None else batch.ws.numel() * batch.ws.element_size()
    rc = load_library().kfac_weight_update_batched(batch.host, batch.count, float(eta), float(momentum), float(eps),
                                                   _ptr(batch.ws), ws_bytes, _stream(stream))
    _check(rc, "kfac_weight_update_batched")


# The operators below take their sizes from the tensors, so they look at them: another type, shape, stride or device than the call
# wants raises KfacError with KFAC_ERR_INVALID_ARG before anything is launched.
_KFAC_DTYPE = {t: k for k, t in _TORCH_DTYPE.items()}


def _want(ok: bool, where: str, what: str) -> None:
    if not ok:
        raise KfacError(KFAC_ERR_INVALID_ARG, f"{where} ({what})")


def _gpu(device, where: str) -> torch.device:
    """The GPU `device` names, which has to be the current one: the stream a call goes to is the current device's."""
    device = torch.device(device)
    _want(device.type == "cuda", where, "tensors of a GPU are wanted")
    current = torch.cuda.current_device()
    _want(device.index in (None, current), where, f"the tensors' device {device.index} is not the current one, {current}")
    return torch.device("cuda", current)


def _stream_on(index: int, where: str, stream) -> int:
    """The stream of a call on tensors of GPU `index`, which has to be the current one."""
    private = torch._C              # (see _stream; there is a tensor, so that the GPU is initialised)
    try:
        current = private._cuda_getDevice()
        found = private._cuda_getCurrentRawStream(current) if stream is None else None
    except AttributeError:
        current, found = torch.cuda.current_device(), None
    if current != index:
        _want(False, where, f"the tensors' device {index} is not the current one, {current}")
    return _stream(stream) if found is None else found


def _flat(t: torch.Tensor, dtype: torch.dtype, shape, device, where: str, name: str) -> torch.Tensor:
    _want(t.dtype == dtype and tuple(t.shape) == tuple(shape) and t.is_contiguous() and t.device == device, where,
          f"{name}: contiguous {dtype} of shape {tuple(shape)} on {device}")
    return t


def _dense(t: torch.Tensor) -> bool:
    """Whether t's elements lie side by side, in whatever order of dimensions."""
    step = 1
    for stride, size in sorted((st, n) for st, n in zip(t.stride(), t.shape) if n != 1):
        if stride != step:
            return False
        step *= size
    return True


class GradBatch:
    """A kfac_grad_item table (host memory; built once, reused every step), its scratch and the device float `norm`.  It stands for the memory
    of these very tensors, which it keeps alive: gradients that are allocated anew need a new table.
    g: gradient tensors of any of the three types, their elements side by side; out: None (clipped in place), or per tensor None / a
    tensor of the same type, shape and strides that receives the clipped gradient.  A tensor that is written must not be there twice.
    Calls that use one table must not overlap in time."""

    def __init__(self, g: Sequence[torch.Tensor], out: Optional[Sequence[Optional[torch.Tensor]]] = None, device="cuda"):
        n = len(g)
        out = [None] * n if out is None else list(out)
        _want(len(out) == n, "GradBatch", "as many results as gradients")
        self.device = _gpu(device, "GradBatch")
        self.count = n
        self.keep = (list(g), out)
        self.host = (kfac_grad_item * max(n, 1))()
        index = self.device.index
        for i, (x, y) in enumerate(zip(g, out)):
            dtype, size = _KFAC_DTYPE.get(x.dtype), x.numel()
            if dtype is None or x.get_device() != index or not (x.is_contiguous() or _dense(x)):
                _want(size == 0 and dtype is not None, "GradBatch", f"gradient {i}: float32, bfloat16 or float16 on {self.device}, without gaps")
            if y is not None and not (y.dtype == x.dtype and y.get_device() == index and y.shape == x.shape and y.stride() == x.stride()):
                _want(False, "GradBatch", f"result {i}: the gradient's type, shape and strides")
            item = self.host[i]
            item.g, item.out, item.n, item.dtype = x.data_ptr(), None if y is None else y.data_ptr(), size, dtype
        self.apart = None         # whether a clipping call may write: no tensor that it writes overlaps another (found by the first one)
        self.norm = torch.zeros((), dtype=torch.float32, device=self.device)
        self.ws = alloc_workspace(int(load_library().kfac_grad_norm_workspace_bytes(self.host, n)), self.device)
        self.ws_bytes = 0 if self.ws is None else self.ws.numel()

    def _apart(self) -> bool:
        spans = []                # first byte, behind the last one, written
        for item, (g, _) in zip(self.host, zip(*self.keep)):
            size, here = item.n * g.element_size(), item.out in (None, item.g)
            if size:
                spans += [(item.g, item.g + size, here)] + ([] if here else [(item.out, item.out + size, True)])
        any_end = written_end = 0
        for first, end, written in sorted(spans):
            if first < (any_end if written else written_end):
                return False
            any_end = max(any_end, end)
            written_end = max(written_end, end) if written else written_end
        return True


def kfac_grad_norm_batched(batch: GradBatch, stream=None) -> torch.Tensor:
    """The norm over all of the table's gradients: batch.norm, a device float that the next call on the table overwrites."""
    rc = (_lib or load_library()).kfac_grad_norm_batched(batch.host, batch.count, batch.norm.data_ptr(), _ptr(batch.ws), batch.ws_bytes,
                                                         _stream_on(batch.device.index, "kfac_grad_norm_batched", stream))
    _check(rc, "kfac_grad_norm_batched")
    return batch.norm


def kfac_grad_clip_batched(batch: GradBatch, max_norm: float, given_norm: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """out = g min(1, max_norm / norm).  given_norm: None (the norm is that of the table's gradients), or the norm as one device
    float, such as the norm over all processes.  Returns the norm that was used."""
    where = "kfac_grad_clip_batched"
    if given_norm is not None and not (given_norm.dtype == torch.float32 and given_norm.numel() == 1 and given_norm.device == batch.device):
        _want(False, where, f"given_norm: one float32 on {batch.device}")
    if batch.apart is None:
        batch.apart = batch._apart()
    if not batch.apart:
        _want(False, where, "a tensor that is written overlaps another of the table")
    norm = batch.norm if given_norm is None else given_norm
    rc = (_lib or load_library()).kfac_grad_clip_batched(batch.host, batch.count, float(max_norm), _ptr(given_norm),
                                                         None if given_norm is not None else norm.data_ptr(), _ptr(batch.ws), batch.ws_bytes,
                                                         _stream_on(batch.device.index, where, stream))
    _check(rc, where)
    return norm


class ExpertRoute:
    """Where the tokens of a layer of experts go: the device tensors offsets (E + 1), order (T K; None: not wanted) and place (T, K)
    that kfac_expert_sort fills and the others read, all int32, and the sort's scratch.  Calls that use one object must not
    overlap a sort in time."""

    def __init__(self, tokens: int, choices: int, experts: int, device="cuda", offsets: Optional[torch.Tensor] = None,
                 order: Optional[torch.Tensor] = None, place: Optional[torch.Tensor] = None, want_order: bool = True):
        self.device = _gpu(device, "ExpertRoute")
        self.index = self.device.index
        self.tokens, self.choices, self.experts = int(tokens), int(choices), int(experts)
        self.desc = kfac_expert_desc(self.tokens, self.choices, self.experts, 0, 0, 0, 0, 0)
        rows = self.tokens * self.choices
        _want(self.tokens >= 0 and self.choices >= 1 and self.experts >= 1, "ExpertRoute", "tokens, choices, experts")
        i32 = dict(dtype=torch.int32, device=self.device)

        def given(t, shape, name):
            return torch.empty(shape, **i32) if t is None else _flat(t, torch.int32, shape, self.device, "ExpertRoute", name)

        self.offsets = given(offsets, (self.experts + 1,), "offsets")
        self.order = given(order, (rows,), "order") if want_order or order is not None else None
        self.place = given(place, (self.tokens, self.choices), "place")
        self.ws = alloc_workspace(int(load_library().kfac_expert_sort_workspace_bytes(ctypes.byref(self.desc))), self.device)
        self.ws_bytes = 0 if self.ws is None else self.ws.numel()
        self._descs = {}          # by the tensors' shapes, strides and types

    def _side(self, t, rows, where, name):
        _want(t.dim() == 2 and t.shape[0] == rows and t.shape[1] >= 1 and t.dtype in _KFAC_DTYPE and t.device == self.device, where,
              f"{name}: {rows} rows of float32, bfloat16 or float16 on {self.device}")
        _want(t.shape[1] == 1 or t.stride(1) == 1, where, f"{name}: elements of a row side by side")
        _want(rows <= 1 or t.stride(0) >= t.shape[1], where, f"{name}: rows apart from each other")
        return 0 if rows <= 1 else t.stride(0)

    def _rows(self, where, token_side, row_side, grad_side=None):
        """The descriptor of a call on these tensors: one in tokens' order, one or none in the experts', the gradient of such a one or none."""
        key = (token_side.shape, token_side.stride(), token_side.dtype, token_side.get_device())
        for t in (row_side, grad_side):
            key += (None,) if t is None else (t.shape, t.stride(), t.dtype, t.get_device())
        desc = self._descs.get(key)
        if desc is None:
            rows = self.tokens * self.choices
            ld = [self._side(token_side, self.tokens, where, "a tensor in tokens' order")]
            for t in (row_side, grad_side):
                ld.append(0 if t is None else self._side(t, rows, where, "a tensor in the experts' order"))
                _want(t is None or (t.shape[1] == token_side.shape[1] and t.dtype == token_side.dtype), where, "rows of one width and type")
            desc = self._descs[key] = ctypes.byref(kfac_expert_desc(self.tokens, self.choices, self.experts, token_side.shape[1],
                                                                    _KFAC_DTYPE[token_side.dtype], *ld))
        return desc

    def _weights(self, t, where, name):
        if t is None:
            return None
        if not (t.dtype == torch.float32 and t.shape == self.place.shape and t.is_contiguous() and t.get_device() == self.index):
            _want(False, where, f"{name}: contiguous float32 of shape {tuple(self.place.shape)} on {self.device}")
        return t.data_ptr()


def kfac_expert_sort(route: ExpertRoute, expert: torch.Tensor, stream=None) -> ExpertRoute:
    """expert: (T, K) int32, what is not in 0 .. E - 1 is no assignment.  Fills route.offsets, route.order and route.place."""
    if not (expert.dtype == torch.int32 and expert.shape == route.place.shape and expert.is_contiguous() and expert.get_device() == route.index):
        _want(False, "kfac_expert_sort", f"expert: contiguous int32 of shape {tuple(route.place.shape)} on {route.device}")
    rc = (_lib or load_library()).kfac_expert_sort(ctypes.byref(route.desc), expert.data_ptr(), route.offsets.data_ptr(), _ptr(route.order),
                                                   route.place.data_ptr(), _ptr(route.ws), route.ws_bytes,
                                                   _stream_on(route.index, "kfac_expert_sort", stream))
    _check(rc, "kfac_expert_sort")
    return route


def kfac_expert_dispatch(route: ExpertRoute, x: torch.Tensor, xs: torch.Tensor, stream=None) -> torch.Tensor:
    """x: (T, D), xs: (T K, D): every token's row to its places."""
    desc = route._rows("kfac_expert_dispatch", x, xs)
    rc = (_lib or load_library()).kfac_expert_dispatch(desc, x.data_ptr(), route.place.data_ptr(), xs.data_ptr(),
                                                       _stream_on(route.index, "kfac_expert_dispatch", stream))
    _check(rc, "kfac_expert_dispatch")
    return xs


def kfac_expert_combine(route: ExpertRoute, ys: torch.Tensor, weights: Optional[torch.Tensor], y: torch.Tensor, stream=None) -> torch.Tensor:
    """ys: (T K, D), weights: (T, K) float32 or None (all 1), y: (T, D).  Without weights also the gradient of kfac_expert_dispatch."""
    desc = route._rows("kfac_expert_combine", y, ys)
    rc = (_lib or load_library()).kfac_expert_combine(desc, ys.data_ptr(), route._weights(weights, "kfac_expert_combine", "weights"),
                                                      route.place.data_ptr(), y.data_ptr(), _stream_on(route.index, "kfac_expert_combine", stream))
    _check(rc, "kfac_expert_combine")
    return y


def kfac_expert_combine_backward(route: ExpertRoute, dy: torch.Tensor, ys: Optional[torch.Tensor], weights: Optional[torch.Tensor],
                                 dys: torch.Tensor, dweights: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """dy: (T, D), ys and dys: (T K, D), weights and dweights: (T, K) float32.  dweights = None: ys is not read and may be None."""
    where = "kfac_expert_combine_backward"
    _want(dweights is None or ys is not None, where, "dweights needs ys")
    desc = route._rows(where, dy, None if dweights is None else ys, dys)
    rc = (_lib or load_library()).kfac_expert_combine_backward(desc, dy.data_ptr(), None if dweights is None else ys.data_ptr(),
                                                               route._weights(weights, where, "weights"), route.place.data_ptr(), dys.data_ptr(),
                                                               route._weights(dweights, where, "dweights"), _stream_on(route.index, where, stream))
    _check(rc, where)
    return dys


class ExpertFactors:
    """Descriptor and scratch of the factor builds of one layer of experts (built once, reused every step): x of `rows` rows of `dim`
    elements of a torch dtype in the experts' order, `ld` elements from one row to the next (0: dim).  Where these are whole 16-byte vectors x
    has to be 16-byte aligned; others are copied first.  Calls that use one object must not overlap in time."""

    def __init__(self, rows: int, experts: int, dim: int, dtype: torch.dtype, has_bias: bool = False, packed: bool = False, ld: int = 0,
                 device="cuda"):
        self.device = _gpu(device, "ExpertFactors")
        self.index = self.device.index
        _want(dtype in _KFAC_DTYPE, "ExpertFactors", "float32, bfloat16 or float16")
        self.rows, self.experts, self.dim, self.dtype, self.ld = int(rows), int(experts), int(dim), dtype, int(ld) or int(dim)
        self.d = self.dim + int(bool(has_bias))
        self.shape = (self.experts, packed_elems(self.d)) if packed else (self.experts, self.d, self.d)
        self.desc = kfac_expert_factor_desc(self.rows, self.experts, self.dim, _KFAC_DTYPE[dtype], int(bool(has_bias)), int(bool(packed)), int(ld))
        self.on_grid = self.ld * dtype.itemsize % 16 == 0 and self.ld <= 1 << 18           # rows are read as they lie, not copied first
        self.ws = alloc_workspace(int(load_library().kfac_expert_factor_workspace_bytes(ctypes.byref(self.desc))), self.device)
        self.ws_bytes = 0 if self.ws is None else self.ws.numel()


def kfac_expert_factor(plan: ExpertFactors, x: torch.Tensor, offsets: torch.Tensor, scale: float = 0.0, out: Optional[torch.Tensor] = None,
                       running: Optional[torch.Tensor] = None, decay: float = 0.0, stream=None) -> torch.Tensor:
    """The factors of all experts, into `out` (plan.shape, float32), or folded into the running averages `running`."""
    where = "kfac_expert_factor"
    if not (x.dtype == plan.dtype and x.shape == (plan.rows, plan.dim) and x.get_device() == plan.index and
            (plan.dim == 1 or x.stride(1) == 1) and (plan.rows <= 1 or x.stride(0) == plan.ld)):
        _want(False, where, f"x: {plan.dtype} of shape {(plan.rows, plan.dim)} on {plan.device}, rows {plan.ld} elements apart")
    if plan.on_grid and x.data_ptr() % 16 and plan.rows:
        _want(False, where, f"x: rows {plan.ld} elements apart, which are whole 16-byte vectors, have to begin at 16-byte addresses")
    if not (offsets.dtype == torch.int32 and offsets.shape == (plan.experts + 1,) and offsets.is_contiguous() and offsets.get_device() == plan.index):
        _want(False, where, f"offsets: {plan.experts + 1} contiguous int32 on {plan.device}")
    _want((out is None) != (running is None), where, "either out or running")
    to = running if out is None else out
    if not (to.dtype == torch.float32 and to.shape == plan.shape and to.is_contiguous() and to.get_device() == plan.index):
        _want(False, where, f"contiguous float32 results of shape {plan.shape} on {plan.device}")
    rc = (_lib or load_library()).kfac_expert_factor(ctypes.byref(plan.desc), x.data_ptr(), offsets.data_ptr(), float(scale), _ptr(out), _ptr(running),
                                                     float(decay), _ptr(plan.ws), plan.ws_bytes, _stream_on(plan.index, where, stream))
    _check(rc, where)
    return to


def kfac_bn_sample_grads_workspace_bytes(N: int, C: int, HW: int) -> int:
    return int(load_library().kfac_bn_sample_grads_workspace_bytes(int(N), int(C), int(HW)))


def kfac_bn_sample_grads(xhat: torch.Tensor, gout: torch.Tensor, dtype: int, g: Optional[torch.Tensor] = None,
                         ws: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """xhat, gout: (N, H, W, C) or (N, HW, C) channels-last tensors of the given kfac dtype; returns g (N, 2C) fp32."""
    N, C = int(xhat.shape[0]), int(xhat.shape[-1])
    HW = int(xhat.numel() // (N * C))
    if g is None:
        g = torch.empty((N, 2 * C), dtype=torch.float32, device=xhat.device)
    if ws is None:
        ws = alloc_workspace(int(load_library().kfac_bn_sample_grads_workspace_bytes(N, C, HW)), xhat.device)
    ws_bytes = 0 if ws is None else ws.numel() * ws.element_size()
    rc = load_library().kfac_bn_sample_grads(_ptr(xhat), _ptr(gout), N, C, HW, int(dtype), _ptr(g), _ptr(ws), ws_bytes,
                                             _stream(stream))
    _check(rc, "kfac_bn_sample_grads")
    return g


class BnBatch:
    """A kfac_bn_item table (host memory), the per-sample gradient tensors (N, 2C) and the scratch, for many BN layers.
    xhat[i], gout[i]: channels-last (N, H, W, C) or (N, HW, C) tensors of kfac dtype dtype[i] (one value: all layers)."""

    def __init__(self, xhat: Sequence[torch.Tensor], gout: Sequence[torch.Tensor], dtype, device="cuda"):
        n = len(xhat)
        dtypes = list(dtype) if isinstance(dtype, (list, tuple)) else [int(dtype)] * n
        self.count = n
        self.g = []
        self.host = (kfac_bn_item * max(n, 1))()
        for i in range(n):
            N, C = int(xhat[i].shape[0]), int(xhat[i].shape[-1])
            HW = int(xhat[i].numel() // (N * C))
            self.g.append(torch.empty((N, 2 * C), dtype=torch.float32, device=device))
            self.host[i] = kfac_bn_item(xhat[i].data_ptr(), gout[i].data_ptr(), self.g[i].data_ptr(), N, C, HW, dtypes[i])
        self.keep = (list(xhat), list(gout))
        nbytes = int(load_library().kfac_bn_sample_grads_batched_workspace_bytes(self.host, n)) if n else 0
        self.ws = alloc_workspace(nbytes, device) if nbytes else None


def kfac_bn_sample_grads_batched(batch: BnBatch, stream=None):
    ws_bytes = 0 if batch.ws is None else batch.ws.numel() * batch.ws.element_size()
    rc = load_library().kfac_bn_sample_grads_batched(batch.host, batch.count, _ptr(batch.ws), ws_bytes, _stream(stream))
    _check(rc, "kfac_bn_sample_grads_batched")
    return batch.g


def kfac_bn_diag_precondition(g: torch.Tensor, grad: Optional[torch.Tensor], damping: float,
                              fisher_diag: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
                              stream=None) -> None:
    N, C2 = int(g.shape[0]), int(g.shape[1])
    rc = load_library().kfac_bn_diag_precondition(_ptr(g), N, C2, _ptr(grad), float(damping), _ptr(fisher_diag), _ptr(out),
                                                  _stream(stream))
    _check(rc, "kfac_bn_diag_precondition")


def kfac_inverse_workspace_bytes(dim: int) -> int:
    return int(load_library().kfac_inverse_workspace_bytes(int(dim)))


def kfac_damped_inverse(S: torch.Tensor, dim: int, damping: float, Minv: torch.Tensor,
                        info: Optional[torch.Tensor] = None, ws: Optional[torch.Tensor] = None,
                        stream=None) -> torch.Tensor:
    ws_bytes = 0 if ws is None else ws.numel() * ws.element_size()
    rc = load_library().kfac_damped_inverse(_ptr(S), int(dim), float(damping), _ptr(Minv), _ptr(info), _ptr(ws),
                                            ws_bytes, _stream(stream))
    _check(rc, "kfac_damped_inverse")
    return Minv


class InverseBatch:
    """A kfac_inverse_item table (host memory; built once, reused every step) and the scratch it points to."""

    def __init__(self, S: Sequence[torch.Tensor], Minv: Sequence[torch.Tensor], dampings: Sequence[float],
                 info: Optional[torch.Tensor] = None, device="cuda",
                 dampings_dev: Optional[Sequence[Optional[int]]] = None, ws=None, planes=None):
        """dampings_dev[i]: None, or the device address of a float that replaces dampings[i] when the work runs.
        planes: None, or per matrix None / a byte tensor of kfac_inverse_planes_bytes(dim) that receives the inverse as
        fp16 piece planes (what PrecondBatch takes as Ginv_planes / Ainv_planes).
        ws: None (scratch is allocated here), or one scratch tensor per matrix of kfac_inverse_workspace_bytes(dim)
        bytes, which tables that never run at the same time may share."""
        n = len(S)
        dims = [int(s.shape[0]) for s in S]
        self.order = sorted(range(n), key=lambda i: -dims[i])        # the ABI wants largest first
        self.count = n
        self.ws = list(ws) if ws is not None else [alloc_workspace(kfac_inverse_workspace_bytes(d), device) for d in dims]
        self.info = info if info is not None else torch.zeros(n, dtype=torch.int32, device=device)
        self.keep = (list(S), list(Minv), None if planes is None else list(planes))
        arr = (kfac_inverse_item * n)()
        for slot, i in enumerate(self.order):
            arr[slot] = kfac_inverse_item(S[i].data_ptr(), Minv[i].data_ptr(), _ptr(self.ws[i]),
                                          self.info.data_ptr() + 4 * i, dims[i], float(dampings[i]),
                                          None if dampings_dev is None else dampings_dev[i],
                                          None if planes is None else _ptr(planes[i]))
        self.host = arr


def kfac_inverse_planes_bytes(dim: int) -> int:
    return int(load_library().kfac_inverse_planes_bytes(int(dim)))


def kfac_damped_inverse_batched(batch: InverseBatch, stream=None) -> None:
    rc = load_library().kfac_damped_inverse_batched(batch.host, batch.count, _stream(stream))
    _check(rc, "kfac_damped_inverse_batched")


KFAC_REFRESH_GROWING, KFAC_REFRESH_LATE = 0, 1


class PiBatch:
    """A kfac_pi_item table (host memory) and the device array of per-factor dampings it fills: lam[2 i] for A_i,
    lam[2 i + 1] for G_i."""

    def __init__(self, A: Sequence[torch.Tensor], G: Sequence[torch.Tensor], device="cuda"):
        n = len(A)
        self.count = n
        self.keep = (list(A), list(G))
        self.host = (kfac_pi_item * max(n, 1))()
        for i in range(n):
            self.host[i] = kfac_pi_item(A[i].data_ptr(), G[i].data_ptr(), int(A[i].shape[0]), int(G[i].shape[0]))
        self.lam = torch.zeros(2 * max(n, 1), dtype=torch.float32, device=device)

    def address(self, layer: int, which: int) -> int:
        """Device address of lambda_A (which = 0) or lambda_G (which = 1) of a layer."""
        return self.lam.data_ptr() + 4 * (2 * layer + which)


def kfac_pi_damping_batched(batch: PiBatch, gamma: float, stream=None) -> torch.Tensor:
    rc = load_library().kfac_pi_damping_batched(batch.host, batch.count, float(gamma), _ptr(batch.lam), _stream(stream))
    _check(rc, "kfac_pi_damping_batched")
    return batch.lam[:2 * batch.count]


def kfac_warmup_damping_alpha(gamma0: float, gamma_target: float, t_warmup: float) -> float:
    return float(load_library().kfac_warmup_damping_alpha(float(gamma0), float(gamma_target), float(t_warmup)))


def kfac_warmup_damping_next(gamma: float, gamma_target: float, alpha: float) -> float:
    return float(load_library().kfac_warmup_damping_next(float(gamma), float(gamma_target), float(alpha)))


def kfac_bn_damping(gamma: float, rho_bn: float) -> float:
    return float(load_library().kfac_bn_damping(float(gamma), float(rho_bn)))


def kfac_refresh_interval(epoch: int, heuristic: int = KFAC_REFRESH_GROWING) -> int:
    return int(load_library().kfac_refresh_interval(int(epoch), int(heuristic)))


def kfac_precondition_workspace_bytes(dG: int, dA: int) -> int:
    return int(load_library().kfac_precondition_workspace_bytes(int(dG), int(dA)))


def kfac_precondition(Ginv: torch.Tensor, Ainv: torch.Tensor, gradW: torch.Tensor, dG: int, dA: int,
                      out: torch.Tensor, ws: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    ws_bytes = 0 if ws is None else ws.numel() * ws.element_size()
    rc = load_library().kfac_precondition(_ptr(Ginv), _ptr(Ainv), _ptr(gradW), int(dG), int(dA), _ptr(out), _ptr(ws),
                                          ws_bytes, _stream(stream))
    _check(rc, "kfac_precondition")
    return out


class PrecondBatch:
    """Host + device copies of a kfac_precond_item table (built once, reused every step).  ws: None (scratch is
    allocated here), or one scratch tensor per layer of kfac_precondition_workspace_bytes(d_G, d_A) bytes."""

    def __init__(self, Ginv: Sequence[torch.Tensor], Ainv: Sequence[torch.Tensor], gradW: Sequence[torch.Tensor],
                 out: Sequence[torch.Tensor], device="cuda", ws=None, Ginv_planes=None, Ainv_planes=None):
        """Ginv_planes / Ainv_planes: None, or per layer None / the planes tensor an InverseBatch filled for that inverse."""
        n = len(out)
        shapes = [tuple(g.shape) for g in gradW]
        self.order = sorted(range(n), key=lambda i: -shapes[i][1])       # large d_A first: best load balance
        self.count = n
        self.ws = (list(ws) if ws is not None else
                   [alloc_workspace(kfac_precondition_workspace_bytes(dG, dA), device) for dG, dA in shapes])
        self.keep = (list(Ginv), list(Ainv), list(gradW), list(out), Ginv_planes, Ainv_planes)
        arr = (kfac_precond_item * n)()
        for slot, i in enumerate(self.order):
            arr[slot] = kfac_precond_item(Ginv[i].data_ptr(), Ainv[i].data_ptr(), gradW[i].data_ptr(),
                                          out[i].data_ptr(), self.ws[i].data_ptr(), shapes[i][0], shapes[i][1],
                                          None if Ginv_planes is None else _ptr(Ginv_planes[i]),
                                          None if Ainv_planes is None else _ptr(Ainv_planes[i]))
        self.host = arr
        self.dev = torch.frombuffer(bytearray(bytes(arr)), dtype=torch.uint8).to(device)


def kfac_precondition_batched(batch: PrecondBatch, stream=None) -> None:
    rc = load_library().kfac_precondition_batched(batch.host, batch.dev.data_ptr(), batch.count, _stream(stream))
    _check(rc, "kfac_precondition_batched")


def kfac_kernel_timing_enable(enable: bool) -> None:
    _check(load_library().kfac_kernel_timing_enable(int(bool(enable))), "kfac_kernel_timing_enable")


def kfac_probe_mfma(dtype: int, workgroups: int, iters: int, out: torch.Tensor, stream=None) -> None:
    _check(load_library().kfac_probe_mfma(int(dtype), int(workgroups), int(iters), _ptr(out), _stream(stream)), "kfac_probe_mfma")


def kfac_probe_copy(src: torch.Tensor, dst: torch.Tensor, workgroups: int, stream=None) -> None:
    nbytes = src.numel() * src.element_size()
    _check(load_library().kfac_probe_copy(_ptr(src), _ptr(dst), nbytes, int(workgroups), _stream(stream)), "kfac_probe_copy")


def kfac_probe_read(src: torch.Tensor, sink: torch.Tensor, workgroups: int, stream=None) -> None:
    nbytes = src.numel() * src.element_size()
    _check(load_library().kfac_probe_read(_ptr(src), _ptr(sink), nbytes, int(workgroups), _stream(stream)), "kfac_probe_read")


def kfac_kernel_timing_report() -> dict:
    """{kernel name: (total milliseconds, launches)} since timing was enabled or last reported."""
    buf = ctypes.create_string_buffer(1 << 16)
    _check(load_library().kfac_kernel_timing_report(buf, len(buf)), "kfac_kernel_timing_report")
    out = {}
    for line in buf.value.decode().splitlines():
        name, ms, n = line.rsplit(" ", 2)
        out[name] = (float(ms), int(n))
    return out
