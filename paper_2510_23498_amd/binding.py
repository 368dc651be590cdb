"""ctypes binding of librampde.so (argument marshalling only).

The functions carry the names of the C entry points declared in include/rampde.h.
torch is used for device memory and the current stream; no step of the method runs
here.  If the library has not been built the first call raises: there is no fallback.
"""
from __future__ import annotations

import ctypes as C
import functools
import os
from dataclasses import dataclass
from typing import NamedTuple, Optional, Sequence

import numpy as np
import torch

from .build import LIB_PATH

F32, F16, BF16 = 0, 1, 2
SCALE_NONE, SCALE_NONE_SAFE, SCALE_DYNAMIC, SCALE_AUTO = 0, 1, 2, 3
VEL_MLP, VEL_CONV2, VEL_PARABOLIC, VEL_CNF = 0, 1, 2, 3
OK, EINVAL, EUNSUPPORTED, EWORKSPACE, ESCALE, EHIP = 0, 1, 2, 3, 4, 5
_LOW = {"f32": F32, "f16": F16, "bf16": BF16}
_SCALING = {"none": SCALE_NONE, "none_safe": SCALE_NONE_SAFE, "dynamic": SCALE_DYNAMIC, "auto": SCALE_AUTO}
_TORCH_LOW = {F16: torch.float16, BF16: torch.bfloat16}
_TYPES = {torch.float32: F32, torch.float16: F16, torch.bfloat16: BF16}
_FP8_MODES = {"rows": 0, "cols": 1, "blocks": 2}

EXPORTS = ("rampde_num_params", "rampde_workspace_bytes", "rampde_odeint_fwd", "rampde_odeint_bwd",
           "rampde_odeint_bwd_tgrid", "rampde_strerror", "rampde_version", "rampde_timing_enable", "rampde_timing_read",
           "rampde_recurrence_states", "rampde_recurrence_workspace_bytes", "rampde_recurrence_fwd", "rampde_recurrence_bwd",
           "rampde_dropout", "rampde_join_workspace_bytes", "rampde_join_fwd", "rampde_join_bwd", "rampde_fp8_value_bytes",
           "rampde_fp8_scale_bytes", "rampde_fp8_quantize", "rampde_fp8_workspace_bytes", "rampde_fp8_matmul",
           "rampde_fp8_matmul_short")

K_VELOCITY_GEMM, K_WGRAD_GEMM, K_COMBINE_STORE, K_ADJOINT_UPDATE, K_FUSED_FORWARD, K_FUSED_ADJOINT_STEP = range(6)
ROUND_INCREMENT, GROW_RAW_NORM, PER_LAYER_KERNELS, NAIVE_STATE, NO_WAITS, SKEWED_CLUSTERS = 1, 2, 4, 8, 16, 32


def no_waits_after(n: int) -> int:
    """RAMPDE_NO_WAITS_AFTER(n)"""
    return NO_WAITS | n << 16


class _Tableau(C.Structure):
    _fields_ = [("s", C.c_int), ("A", C.POINTER(C.c_double)), ("b", C.POINTER(C.c_double)),
                ("c", C.POINTER(C.c_double))]


class _Velocity(C.Structure):
    _fields_ = [("kind", C.c_int), ("n_layers", C.c_int), ("widths", C.POINTER(C.c_int)),
                ("C", C.c_int), ("H", C.c_int), ("W", C.c_int), ("time_input", C.c_int), ("n_intervals", C.c_int)]


class _Policy(C.Structure):
    _fields_ = [("low", C.c_int), ("scaling", C.c_int), ("k_max", C.c_int), ("flags", C.c_uint),
                ("step_group", C.c_int), ("row_tile", C.c_int), ("wgrad_tile", C.c_int), ("scale_group", C.c_int)]


class _Stats(C.Structure):
    _fields_ = [("status", C.c_int), ("failed_step", C.c_int), ("retries", C.c_int),
                ("s_first", C.c_float), ("s_last", C.c_float), ("s_min", C.c_float), ("s_max", C.c_float)]


class _KernelTime(C.Structure):
    _fields_ = [("ms", C.c_double), ("launches", C.c_int64), ("work", C.c_double)]


class _Recurrence(C.Structure):
    _fields_ = [("B", C.c_int64), ("T", C.c_int64), ("D", C.c_int64), ("share", C.c_int), ("low", C.c_int),
                ("x_stride", C.c_int64 * 2), ("z_stride", C.c_int64 * 2), ("h_stride", C.c_int64 * 2)]


class _Join(C.Structure):
    _fields_ = [("rows", C.c_int64), ("cols", C.c_int64), ("low", C.c_int), ("alpha", C.c_double), ("eps", C.c_double),
                ("p", C.c_double), ("seed", C.c_uint64), ("offset", C.c_uint64), ("ld_b", C.c_int64),
                ("ld_gate", C.c_int64), ("ld_x", C.c_int64), ("write_grads", C.c_int)]


class RampdeError(RuntimeError):
    def __init__(self, code: int, msg: str, stats=None):
        super().__init__(f"rampde error {code}: {msg}")
        self.code = code
        self.stats = stats


_lib = None


def load_library():
    """Load librampde.so (built in-tree by paper_2510_23498_amd.build); raises if absent."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is missing: run `python -m paper_2510_23498_amd.build` first "
                           "(there is no fallback path)")
    lib = C.CDLL(LIB_PATH)
    lib.rampde_num_params.restype = C.c_int64
    lib.rampde_num_params.argtypes = [C.POINTER(_Velocity)]
    lib.rampde_workspace_bytes.restype = C.c_size_t
    lib.rampde_workspace_bytes.argtypes = [C.POINTER(_Velocity), C.c_int64, C.c_int, C.POINTER(_Tableau),
                                           C.POINTER(_Policy), C.c_int]
    lib.rampde_odeint_fwd.restype = C.c_int
    lib.rampde_odeint_fwd.argtypes = [C.POINTER(_Velocity), C.c_void_p, C.c_void_p, C.c_int64,
                                      C.POINTER(C.c_double), C.c_int, C.POINTER(_Tableau), C.POINTER(_Policy),
                                      C.c_void_p, C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]
    lib.rampde_odeint_fwd_static.restype = C.c_int
    lib.rampde_odeint_fwd_static.argtypes = [C.POINTER(_Velocity), C.c_void_p, C.c_void_p, C.c_int64,
                                             C.POINTER(C.c_double), C.c_int, C.POINTER(_Tableau),
                                             C.POINTER(_Policy), C.c_void_p, C.c_void_p, C.c_void_p]
    lib.rampde_odeint_bwd.restype = C.c_int
    lib.rampde_odeint_bwd.argtypes = [C.POINTER(_Velocity), C.c_void_p, C.c_int64, C.POINTER(C.c_double), C.c_int,
                                      C.POINTER(_Tableau), C.POINTER(_Policy), C.c_void_p, C.c_void_p, C.c_void_p,
                                      C.c_void_p, C.c_void_p, C.POINTER(C.c_float), C.POINTER(_Stats), C.c_void_p,
                                      C.c_size_t, C.c_void_p]
    lib.rampde_odeint_bwd_tgrid.restype = C.c_int
    lib.rampde_odeint_bwd_tgrid.argtypes = [C.POINTER(_Velocity), C.c_void_p, C.c_int64, C.POINTER(C.c_double), C.c_int,
                                            C.POINTER(_Tableau), C.POINTER(_Policy), C.c_void_p, C.c_void_p, C.c_void_p,
                                            C.c_void_p, C.c_void_p, C.c_void_p, C.POINTER(C.c_float),
                                            C.POINTER(_Stats), C.c_void_p, C.c_size_t, C.c_void_p]
    lib.rampde_strerror.restype = C.c_char_p
    lib.rampde_strerror.argtypes = [C.c_int]
    lib.rampde_version.restype = C.c_int
    lib.rampde_timing_enable.restype = C.c_int
    lib.rampde_timing_enable.argtypes = [C.c_int]
    lib.rampde_timing_read.restype = C.c_int
    lib.rampde_timing_read.argtypes = [C.c_int, C.POINTER(_KernelTime)]
    p, i64, size, dbl, u64 = C.c_void_p, C.c_int64, C.c_size_t, C.c_double, C.c_uint64
    for name, res, args in (
            ("rampde_recurrence_states", i64, [C.POINTER(_Recurrence)]),
            ("rampde_recurrence_workspace_bytes", size, [C.POINTER(_Recurrence)]),
            ("rampde_recurrence_fwd", C.c_int, [C.POINTER(_Recurrence)] + [p] * 8 + [size, p]),
            ("rampde_recurrence_bwd", C.c_int, [C.POINTER(_Recurrence)] + [p] * 10 + [size, p]),
            ("rampde_dropout", C.c_int, [C.c_int, i64, p, dbl, u64, u64, p, p]),
            ("rampde_join_workspace_bytes", size, [C.POINTER(_Join)]),
            ("rampde_join_fwd", C.c_int, [C.POINTER(_Join)] + [p] * 10),
            ("rampde_join_bwd", C.c_int, [C.POINTER(_Join)] + [p] * 16 + [size, p]),
            ("rampde_fp8_value_bytes", i64, [i64, i64]),
            ("rampde_fp8_scale_bytes", i64, [i64, i64]),
            ("rampde_fp8_quantize", C.c_int, [C.c_int, C.c_int, i64, i64, p, i64] + [p] * 5),
            ("rampde_fp8_workspace_bytes", size, [i64, i64, i64]),
            ("rampde_fp8_matmul", C.c_int, [i64, i64, i64, p, p, p, p, C.c_int, C.c_int, p, i64, p, size, p]),
            ("rampde_fp8_matmul_short", C.c_int, [i64, i64, i64, p, p, p, p, C.c_int, p, i64, p, size, p])):
        fn = getattr(lib, name)
        fn.restype, fn.argtypes = res, args
    _lib = lib
    return lib


# ------------------------------------------------------------------ descriptors
class Velocity:
    """Host-side velocity descriptor (mirrors rampde_velocity)."""

    def __init__(self, kind: str, widths: Sequence[int] = (), C_: int = 0, H: int = 0, W: int = 0,
                 time_input: bool = True, n_intervals: int = 0):
        self.kind = kind
        self.n_intervals = int(n_intervals)
        self.widths = tuple(int(w) for w in widths)
        self.C, self.H, self.W = int(C_), int(H), int(W)
        self.time_input = bool(time_input)
        self._warr = (C.c_int * max(1, len(self.widths)))(*self.widths) if self.widths else None
        self.c = _Velocity()
        self.c.kind = {"mlp": VEL_MLP, "conv2": VEL_CONV2, "parabolic": VEL_PARABOLIC, "cnf": VEL_CNF}[kind]
        self.c.n_intervals = self.n_intervals
        self.c.n_layers = len(self.widths) - 1 if kind in ("mlp", "cnf") else 2
        self.c.widths = C.cast(self._warr, C.POINTER(C.c_int)) if self._warr is not None else None
        self.c.C, self.c.H, self.c.W = self.C, self.H, self.W
        self.c.time_input = 1 if self.time_input else 0

    @staticmethod
    def mlp(widths, time_input=True):
        return Velocity("mlp", widths=widths, time_input=time_input)

    @staticmethod
    def conv2(C_, H, W, time_input=True):
        return Velocity("conv2", C_=C_, H=H, W=W, time_input=time_input)

    @staticmethod
    def cnf(d, H, time_input=True):
        """state [z; l] of d + 1 columns; velocity d -> H -> d with the exact trace row"""
        return Velocity("cnf", widths=(d, H, d), time_input=time_input)

    @staticmethod
    def parabolic(C_, H, W, n_intervals=1):
        return Velocity("parabolic", C_=C_, H=H, W=W, time_input=False, n_intervals=n_intervals)

    @property
    def d(self):
        if self.kind == "cnf":
            return self.widths[0] + 1
        return self.widths[0] if self.kind == "mlp" else self.C * self.H * self.W

    def state_shape(self, B):
        if self.kind == "cnf":
            return (B, self.widths[0] + 1)
        return (B, self.widths[0]) if self.kind == "mlp" else (B, self.C, self.H, self.W)

    def ckpt_shape(self, B, N):
        if self.kind == "cnf":
            return (N + 1, B, self.widths[0] + 1)
        return (N + 1, B, self.widths[0]) if self.kind == "mlp" else (N + 1, B, self.H, self.W, self.C)


class Tableau:
    """Explicit Butcher tableau (mirrors rampde_tableau); A is s x s, strictly lower triangular."""

    def __init__(self, A, b, c):
        self.A = np.ascontiguousarray(np.asarray(A, dtype=np.float64))
        self.b = np.ascontiguousarray(np.asarray(b, dtype=np.float64))
        self.cc = np.ascontiguousarray(np.asarray(c, dtype=np.float64))
        self.s = int(self.b.shape[0])
        self.c = _Tableau(self.s, self.A.ctypes.data_as(C.POINTER(C.c_double)),
                          self.b.ctypes.data_as(C.POINTER(C.c_double)),
                          self.cc.ctypes.data_as(C.POINTER(C.c_double)))


@dataclass
class Policy:
    low: str = "f16"
    scaling: str = "auto"
    k_max: int = 16
    flags: int = 0
    step_group: int = 0
    row_tile: int = 0
    scale_group: int = 0
    wgrad_tile: int = 0

    @property
    def c(self):
        return _Policy(_LOW[self.low], _SCALING[self.scaling], int(self.k_max), int(self.flags),
                       int(self.step_group), int(self.row_tile), int(self.wgrad_tile), int(self.scale_group))

    @property
    def torch_low(self):
        return _TORCH_LOW[_LOW[self.low]]


@dataclass
class BwdInfo:
    status: int
    failed_step: int
    retries: int
    s_first: float
    s_last: float
    s_min: float
    s_max: float
    scale_hist: Optional[np.ndarray]


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else C.c_void_p(t.data_ptr())


def _stream_of(stream, device):
    """Handle of `stream`, or of the current one of the tensors' GPU"""
    # (without an object around the current stream's handle, which takes a fifth of the time of a small call)
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(device.index)
    if stream.device != device:
        raise ValueError(f"stream: on {stream.device}, the tensors are on {device}")
    return stream.cuda_stream


def _on(device, fn, *args) -> int:
    """fn on the tensors' GPU.  The library launches on the current one, and every GPU's default stream has the handle 0."""
    if device.index == torch._C._cuda_getDevice():
        return fn(*args)
    with torch.cuda.device(device):
        return fn(*args)


def _check_dev(t: torch.Tensor, dtype, numel, name, device=None):
    if not (t.is_cuda and t.is_contiguous() and t.dtype == dtype and t.numel() == numel and device in (None, t.device)):
        raise ValueError(f"{name}: need a contiguous cuda tensor of {dtype} with {numel} elements{f' on {device}' if device else ''}, "
                         f"got {t.dtype} {tuple(t.shape)} on {t.device}")


def rampde_strerror(code: int) -> str:
    return load_library().rampde_strerror(code).decode()


def rampde_version() -> int:
    return load_library().rampde_version()


def rampde_timing_enable(on: bool) -> None:
    load_library().rampde_timing_enable(1 if on else 0)


def rampde_timing_read(kernel_class: int):
    """(total ms, launches, algorithmic work) of the recorded launches of one kernel class."""
    kt = _KernelTime()
    rc = load_library().rampde_timing_read(kernel_class, C.byref(kt))
    if rc != OK:
        raise RampdeError(rc, rampde_strerror(rc))
    return kt.ms, int(kt.launches), kt.work


def rampde_num_params(vel: Velocity) -> int:
    return int(load_library().rampde_num_params(C.byref(vel.c)))


def rampde_workspace_bytes(vel: Velocity, B: int, N: int, tab: Tableau, pol: Policy, is_backward: bool) -> int:
    pc = pol.c
    return int(load_library().rampde_workspace_bytes(C.byref(vel.c), B, N, C.byref(tab.c), C.byref(pc),
                                                     1 if is_backward else 0))


def alloc_workspace(vel, B, N, tab, pol, is_backward, device="cuda"):
    nbytes = rampde_workspace_bytes(vel, B, N, tab, pol, is_backward)
    if nbytes == 0:
        raise RampdeError(EINVAL, "workspace query rejected the arguments")
    return torch.empty(nbytes, dtype=torch.uint8, device=device)


def rampde_odeint_fwd(vel: Velocity, theta: torch.Tensor, y0: torch.Tensor, tgrid, tab: Tableau, pol: Policy,
                      ckpt: Optional[torch.Tensor] = None, yN: Optional[torch.Tensor] = None,
                      workspace: Optional[torch.Tensor] = None, stream=None):
    """Forward pass (paper Algorithm 1).  Returns (yN fp32, ckpt low precision).  Asynchronous."""
    lib = load_library()
    B = int(y0.shape[0])
    tg = np.ascontiguousarray(np.asarray(tgrid, dtype=np.float64))
    N = int(tg.shape[0]) - 1
    P, device = rampde_num_params(vel), y0.device
    _check_dev(theta, torch.float32, P, "theta", device)
    _check_dev(y0, torch.float32, B * vel.d, "y0")
    if ckpt is None:
        ckpt = torch.empty(vel.ckpt_shape(B, N), dtype=pol.torch_low, device=y0.device)
    if yN is None:
        yN = torch.empty_like(y0)
    _check_dev(ckpt, pol.torch_low, (N + 1) * B * vel.d, "ckpt", device)
    _check_dev(yN, torch.float32, B * vel.d, "yN", device)
    if workspace is None:
        workspace = alloc_workspace(vel, B, N, tab, pol, False, y0.device)
    pc = pol.c
    rc = _on(device, lib.rampde_odeint_fwd, C.byref(vel.c), _ptr(theta), _ptr(y0), B, tg.ctypes.data_as(C.POINTER(C.c_double)), N,
             C.byref(tab.c), C.byref(pc), _ptr(ckpt), _ptr(yN), _ptr(workspace), workspace.numel(), _stream_of(stream, device))
    if rc != OK:
        raise RampdeError(rc, rampde_strerror(rc))
    return yN, ckpt


STATIC_SCRATCH_BYTES = 32 << 20


def rampde_odeint_fwd_static(vel: Velocity, theta: torch.Tensor, y0: torch.Tensor, tgrid, tab: Tableau, pol: Policy,
                             ckpt: torch.Tensor, yN: torch.Tensor, stream=None):
    """rampde_odeint_fwd on the library's static scratch array: the caller passes every output, nothing
    is allocated here or in the library.  Raises RampdeError(EWORKSPACE) when the problem needs more
    than STATIC_SCRATCH_BYTES of workspace."""
    lib = load_library()
    B = int(y0.shape[0])
    tg = np.ascontiguousarray(np.asarray(tgrid, dtype=np.float64))
    N = int(tg.shape[0]) - 1
    device = y0.device
    _check_dev(theta, torch.float32, rampde_num_params(vel), "theta", device)
    _check_dev(y0, torch.float32, B * vel.d, "y0")
    _check_dev(ckpt, pol.torch_low, (N + 1) * B * vel.d, "ckpt", device)
    _check_dev(yN, torch.float32, B * vel.d, "yN", device)
    pc = pol.c
    rc = _on(device, lib.rampde_odeint_fwd_static, C.byref(vel.c), _ptr(theta), _ptr(y0), B,
             tg.ctypes.data_as(C.POINTER(C.c_double)), N, C.byref(tab.c), C.byref(pc), _ptr(ckpt), _ptr(yN),
             _stream_of(stream, device))
    if rc != OK:
        raise RampdeError(rc, rampde_strerror(rc))
    return yN, ckpt


def rampde_odeint_bwd(vel: Velocity, theta: torch.Tensor, tgrid, tab: Tableau, pol: Policy, ckpt: torch.Tensor,
                      grad_yN: torch.Tensor, grad_ys: Optional[torch.Tensor] = None,
                      grad_y0: Optional[torch.Tensor] = None, grad_theta: Optional[torch.Tensor] = None,
                      workspace: Optional[torch.Tensor] = None, stream=None, want_info: bool = True,
                      grad_t: Optional[torch.Tensor] = None):
    """Discrete adjoint (paper Algorithm 2).  Returns (grad_y0, grad_theta, BwdInfo or None).

    grad_theta is accumulated into; when omitted a zero vector is created.  With `grad_t` (N+1 fp32
    on the device, accumulated into) the call goes to rampde_odeint_bwd_tgrid and also forms dL/dt.
    """
    lib = load_library()
    B = int(grad_yN.shape[0])
    tg = np.ascontiguousarray(np.asarray(tgrid, dtype=np.float64))
    N = int(tg.shape[0]) - 1
    P, device = rampde_num_params(vel), grad_yN.device
    _check_dev(theta, torch.float32, P, "theta", device)
    _check_dev(grad_yN, torch.float32, B * vel.d, "grad_yN")
    _check_dev(ckpt, pol.torch_low, (N + 1) * B * vel.d, "ckpt", device)
    if grad_ys is not None:
        _check_dev(grad_ys, torch.float32, (N + 1) * B * vel.d, "grad_ys", device)
    if grad_y0 is None:
        grad_y0 = torch.empty_like(grad_yN)
    if grad_theta is None:
        grad_theta = torch.zeros(P, dtype=torch.float32, device=grad_yN.device)
    _check_dev(grad_y0, torch.float32, B * vel.d, "grad_y0", device)
    _check_dev(grad_theta, torch.float32, P, "grad_theta", device)
    if workspace is None:
        workspace = alloc_workspace(vel, B, N, tab, pol, True, grad_yN.device)
    pc = pol.c
    stats = _Stats()
    G = int(pol.scale_group)
    groups = (B + G - 1) // G if 0 < G < B else 1
    # one row of N + 1 scales per scale group (a plain vector without groups)
    hist = np.zeros(N + 1 if groups == 1 else (groups, N + 1), dtype=np.float32) if want_info else None
    hist_p = hist.ctypes.data_as(C.POINTER(C.c_float)) if want_info else None
    stats_p = C.byref(stats) if want_info else None
    if grad_t is not None:
        _check_dev(grad_t, torch.float32, N + 1, "grad_t", device)
        rc = _on(device, lib.rampde_odeint_bwd_tgrid, C.byref(vel.c), _ptr(theta), B, tg.ctypes.data_as(C.POINTER(C.c_double)),
                 N, C.byref(tab.c), C.byref(pc), _ptr(ckpt), _ptr(grad_yN), _ptr(grad_ys), _ptr(grad_y0), _ptr(grad_theta),
                 _ptr(grad_t), hist_p, stats_p, _ptr(workspace), workspace.numel(), _stream_of(stream, device))
    else:
        rc = _on(device, lib.rampde_odeint_bwd, C.byref(vel.c), _ptr(theta), B, tg.ctypes.data_as(C.POINTER(C.c_double)), N,
                 C.byref(tab.c), C.byref(pc), _ptr(ckpt), _ptr(grad_yN), _ptr(grad_ys), _ptr(grad_y0), _ptr(grad_theta),
                 hist_p, stats_p, _ptr(workspace), workspace.numel(), _stream_of(stream, device))
    info = None
    if want_info:
        info = BwdInfo(stats.status, stats.failed_step, stats.retries, stats.s_first, stats.s_last, stats.s_min,
                       stats.s_max, hist)
    if rc != OK:
        raise RampdeError(rc, rampde_strerror(rc), info)
    return grad_y0, grad_theta, info


def rampde_odeint_bwd_tgrid(vel: Velocity, theta: torch.Tensor, tgrid, tab: Tableau, pol: Policy, ckpt: torch.Tensor,
                            grad_yN: torch.Tensor, grad_t: Optional[torch.Tensor] = None, **kw):
    """Discrete adjoint with the time-grid gradient (paper Sec. 3, update lines of t'; Algorithm 2).
    Returns (grad_y0, grad_theta, grad_t, BwdInfo or None); grad_t is accumulated into (zeros when omitted)."""
    if grad_t is None:
        grad_t = torch.zeros(len(tgrid), dtype=torch.float32, device=grad_yN.device)
    gy0, gth, info = rampde_odeint_bwd(vel, theta, tgrid, tab, pol, ckpt, grad_yN, grad_t=grad_t, **kw)
    return gy0, gth, grad_t, info


# ------------------------------------------------------------------ operators of a sequence encoder
# Descriptors and sizes go by shapes, strides and types alone and are kept per combination of them (a serving loop makes the same
# call over and over, and its kernels take less time than filling in a structure does).
def _raise(rc: int) -> None:
    if rc != OK:
        raise RampdeError(rc, rampde_strerror(rc))


def _at(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


def _type_of(t: torch.Tensor, name: str) -> int:
    low = _TYPES.get(t.dtype)
    if low is None or not t.is_cuda:
        raise ValueError(f"{name}: need a cuda tensor of float32, float16 or bfloat16, got {t.dtype} on {t.device}")
    return low


@functools.lru_cache(maxsize=4096)
def _rows_apart(shape, stride) -> bool:
    """Neighbouring elements in the last dimension, and rows that do not overlap in the others"""
    return (shape[-1] == 1 or stride[-1] == 1) and all(n == 1 or s >= shape[-1] for n, s in zip(shape[:-1], stride[:-1]))


def _check_like(t: Optional[torch.Tensor], dtype, shape, device, name, contiguous=True):
    """t is None, or of this type and shape on this device, and contiguous, or (contiguous=False) with rows as in _rows_apart"""
    if t is None or (t.dtype is dtype and t.shape == shape and t.device == device and
                     (t.is_contiguous() or (not contiguous and _rows_apart(t.shape, t.stride())))):
        return
    raise ValueError(f"{name}: need a {'contiguous' if contiguous else 'row-wise contiguous'} tensor of {dtype} and shape "
                     f"{tuple(shape)} on {device}, got {t.dtype} {tuple(t.shape)} (strides {t.stride()}) on {t.device}")


def _new(stream, make, *args, **kw) -> torch.Tensor:
    """A tensor that the work on `stream` may use at once: allocated as that stream's (its memory may be another's until then)"""
    if stream is None:
        return make(*args, **kw)
    with torch.cuda.stream(stream):
        return make(*args, **kw)


def _empty_like(stream, t: torch.Tensor) -> torch.Tensor:
    """Uninitialised, with the strides of t (also those of a slice)"""
    if t.is_contiguous():
        return torch.empty_like(t) if stream is None else _new(stream, torch.empty_like, t)
    return _new(stream, torch.empty_strided, t.shape, t.stride(), dtype=t.dtype, device=t.device)


_UNUSED = {}  # device -> 256 bytes for calls whose kernels use no workspace: never written or read


def _space(nbytes: int, workspace: Optional[torch.Tensor], device, stream) -> torch.Tensor:
    if workspace is None:
        if nbytes == 0:
            if device not in _UNUSED:
                _UNUSED[device] = torch.empty(256, dtype=torch.uint8, device=device)
            return _UNUSED[device]
        return _new(stream, torch.empty, nbytes, dtype=torch.uint8, device=device)
    if workspace.device != device or not workspace.is_contiguous():
        raise ValueError(f"workspace: need a contiguous tensor on {device}")
    return workspace


def _size(t: torch.Tensor) -> int:
    return t.numel() * t.element_size()


def _needed(nbytes: int, call=None, ref=None) -> int:
    """Bytes of workspace; a query that gives none has rejected the arguments, for the reason that `call` without buffers names"""
    if nbytes == 0:
        rc = EINVAL if call is None else call(ref, *[0] * (len(call.argtypes) - 1))
        raise RampdeError(rc, f"the arguments are rejected: {rampde_strerror(rc)}")
    return nbytes


@functools.lru_cache(maxsize=1024)
def _recurrence_plan(dtype, x_shape, x_stride, z_shape, z_stride, h_stride):
    """(descriptor, states to save, bytes of workspace that are used)"""
    if len(x_shape) != 3 or len(z_shape) != 3:
        raise ValueError(f"x and z: need [batch, steps, channels], got {tuple(x_shape)} and {tuple(z_shape)}")
    B, T, D = x_shape
    gates = z_shape[2]
    if min(B, T, D, gates) < 1 or D % gates or tuple(z_shape[:2]) != (B, T):
        raise ValueError(f"x {tuple(x_shape)} and z {tuple(z_shape)}: need the same samples and steps, and a number of gates that "
                         "divides the number of channels")
    if not (_rows_apart(x_shape, x_stride) and _rows_apart(z_shape, z_stride)):
        raise ValueError(f"x and z: channels have to be neighbours and rows apart, got strides {x_stride} and {z_stride}")
    share = D // gates
    if share & (share - 1) or share > 128:
        raise RampdeError(EUNSUPPORTED, f"{share} channels share a gate (x {tuple(x_shape)}, z {tuple(z_shape)}): need a power of two, "
                          "at most 128")
    r = _Recurrence(B, T, D, share, _TYPES[dtype], x_stride[:2], z_stride[:2], h_stride[:2] if h_stride else (0, 0))
    ref = C.byref(r)
    lib = load_library()
    nbytes = _needed(int(lib.rampde_recurrence_workspace_bytes(ref)), lib.rampde_recurrence_fwd, ref)
    return ref, int(lib.rampde_recurrence_states(ref)), 0 if nbytes == 256 else nbytes


def _recurrence(x: torch.Tensor, z: torch.Tensor, h: Optional[torch.Tensor]):
    _type_of(x, "x")
    if z.dtype is not x.dtype or z.device != x.device:
        raise ValueError(f"z: need {x.dtype} on {x.device} as x, got {z.dtype} on {z.device}")
    return _recurrence_plan(x.dtype, x.shape, x.stride(), z.shape, z.stride(), None if h is None else h.stride())


def rampde_recurrence_fwd(x: torch.Tensor, z: torch.Tensor, h0: Optional[torch.Tensor] = None,
                          lengths: Optional[torch.Tensor] = None, h: Optional[torch.Tensor] = None,
                          hT: Optional[torch.Tensor] = None, states: Optional[torch.Tensor] = None,
                          save_states: bool = False, workspace: Optional[torch.Tensor] = None, stream=None, want_h: bool = True):
    """Gated linear recurrence h_t = h_{t-1} + sigmoid(z_t) (x_t - h_{t-1}).

    x [B, T, D] and z [B, T, D / share] (share a power of two up to 128) may be slices (channels neighbouring); h0 [B, D] fp32;
    lengths [B] int32.  Returns (h, hT, states): states is None unless given or `save_states`, which the backward pass needs; h is
    None where neither it is given nor `want_h` (the last state alone is of interest, a third of the traffic less).  Asynchronous.
    """
    device = x.device
    if h is None:
        if want_h:
            h = _new(stream, torch.empty_like, x, memory_format=torch.contiguous_format)
    else:
        _check_like(h, x.dtype, x.shape, device, "h", contiguous=False)
    ref, n, nbytes = _recurrence(x, z, h)
    state = (x.shape[0], x.shape[2])
    _check_like(h0, torch.float32, state, device, "h0")
    if hT is not None:
        _check_like(hT, torch.float32, state, device, "hT")
    elif h0 is not None:
        hT = _empty_like(stream, h0)
    else:
        hT = _new(stream, torch.empty, state, dtype=torch.float32, device=device)
    if states is not None:
        _check_like(states, torch.float32, (n,), device, "states")
    elif save_states:
        states = _new(stream, torch.empty, n, dtype=torch.float32, device=device)
    _check_like(lengths, torch.int32, state[:1], device, "lengths")
    workspace = _space(nbytes, workspace, device, stream)
    _raise(_on(device, _lib.rampde_recurrence_fwd, ref, _at(x), _at(z), _at(h0), _at(lengths), _at(h), _at(hT), _at(states),
               _at(workspace), _size(workspace), _stream_of(stream, device)))
    return h, hT, states


def rampde_recurrence_bwd(x: torch.Tensor, z: torch.Tensor, states: torch.Tensor, dh: Optional[torch.Tensor],
                          dhT: Optional[torch.Tensor] = None, lengths: Optional[torch.Tensor] = None,
                          h0: Optional[torch.Tensor] = None, dx: Optional[torch.Tensor] = None,
                          dz: Optional[torch.Tensor] = None, dh0: Optional[torch.Tensor] = None,
                          workspace: Optional[torch.Tensor] = None, stream=None):
    """Gradients of the recurrence from those of its states (dh) and of its last state (dhT).  Returns (dx, dz, dh0); dx and
    dz, where given, have the strides of x and z.  dh0 is formed when it or h0 (not read: its states are saved) is given.
    """
    device = x.device
    _check_like(dh, x.dtype, x.shape, device, "dh", contiguous=False)
    ref, n, nbytes = _recurrence(x, z, dh)
    state = (x.shape[0], x.shape[2])
    _check_like(dhT, torch.float32, state, device, "dhT")
    _check_like(lengths, torch.int32, state[:1], device, "lengths")
    _check_like(states, torch.float32, (n,), device, "states")
    if dx is None:
        dx = _empty_like(stream, x)
    if dz is None:
        dz = _empty_like(stream, z)
    for t, like, name in ((dx, x, "dx"), (dz, z, "dz")):
        _check_like(t, like.dtype, like.shape, device, name, contiguous=False)
        if t.stride() != like.stride() and any(t.stride(i) != like.stride(i) for i in (0, 1) if t.shape[i] > 1):
            raise ValueError(f"{name}: strides {t.stride()} are not those of its input, {like.stride()}")
    if dh0 is None and h0 is not None:
        dh0 = _new(stream, torch.empty, state, dtype=torch.float32, device=device)
    _check_like(dh0, torch.float32, state, device, "dh0")
    workspace = _space(nbytes, workspace, device, stream)
    _raise(_on(device, _lib.rampde_recurrence_bwd, ref, _at(x), _at(z), _at(lengths), _at(states), _at(dh), _at(dhT), _at(dx),
               _at(dz), _at(dh0), _at(workspace), _size(workspace), _stream_of(stream, device)))
    return dx, dz, dh0


def rampde_dropout(x: torch.Tensor, p: float, seed: int, offset: int = 0, out: Optional[torch.Tensor] = None, stream=None):
    """x with a share p of its elements zeroed and the others divided by 1 - p; the mask is a function of (seed, offset, element)
    and is not stored: the gradient is the same call on the cotangent.  `out` may be x."""
    low, device = _type_of(x, "x"), x.device
    _check_like(x, x.dtype, x.shape, device, "x")
    if out is None:
        out = _empty_like(stream, x)
    else:
        _check_like(out, x.dtype, x.shape, device, "out")
    _raise(_on(device, load_library().rampde_dropout, low, x.numel(), _at(x), p, seed, offset, _at(out), _stream_of(stream, device)))
    return out


class Join(NamedTuple):
    """What rampde_join holds beside the shapes: residual scale, epsilon of the norms, dropout of the branch."""
    alpha: float = 1.0
    eps: float = 1e-6
    p: float = 0.0
    seed: int = 0
    offset: int = 0


def _join_descriptor(join: Join, dtype, y: torch.Tensor, b, gate, x, vectors) -> _Join:
    low = _TYPES.get(dtype)
    if low is None or not y.is_cuda:
        raise ValueError(f"need cuda tensors, b, gate, x and dx of float32, float16 or bfloat16: got {dtype} on {y.device}")
    shape, device = y.shape, y.device
    if len(shape) != 2 or min(shape) < 1:
        raise ValueError(f"y: need [rows, cols], got {tuple(shape)}")
    rows, cols = shape
    _check_like(y, torch.float32, shape, device, "y")
    pitch = [0, 0, 0]
    for i, (t, name) in enumerate(((b, "b"), (gate, "gate"), (x, "x or dx"))):
        if t is not None:
            _check_like(t, dtype, shape, device, name, contiguous=False)
            if rows > 1:
                pitch[i] = t.stride(0)
    for t in vectors:
        _check_like(t, torch.float32, (cols,), device, "w_post, scale, w_pre and their gradients")
    return _Join(rows, cols, low, join.alpha, join.eps, join.p, join.seed, join.offset, *pitch)


class JoinGrads(NamedTuple):
    dy: torch.Tensor
    db: Optional[torch.Tensor]
    dgate: Optional[torch.Tensor]
    dw_post: Optional[torch.Tensor]
    dscale: Optional[torch.Tensor]
    dw_pre: Optional[torch.Tensor]


def rampde_join_fwd(join: Join, y: torch.Tensor, b: Optional[torch.Tensor] = None, gate: Optional[torch.Tensor] = None,
                    w_post: Optional[torch.Tensor] = None, scale: Optional[torch.Tensor] = None,
                    w_pre: Optional[torch.Tensor] = None, y_out: Optional[torch.Tensor] = None,
                    x: Optional[torch.Tensor] = None, rstd: Optional[torch.Tensor] = None, low=None, want_x: bool = True,
                    save_rstd: bool = False, stream=None):
    """y' = y + alpha scale sigmoid(gate) dropout(N(b) w_post) and x = N(y') w_pre, N the root-mean-square norm of a row.

    y [rows, cols] fp32; b, gate, x of one type (`low` names it where there is no b: then x = N(y) w_pre alone).  Returns
    (y', x, rstd); rstd [2, rows] is None unless given or `save_rstd`, which the backward pass needs.
    """
    dtype = b.dtype if b is not None else x.dtype if x is not None else low if low is not None else torch.bfloat16
    device = y.device
    if x is None and want_x:
        x = _empty_like(stream, b) if b is not None and b.is_contiguous() else _new(stream, torch.empty, y.shape, dtype=dtype,
                                                                                   device=device)
    j = _join_descriptor(join, dtype, y, b, gate, x, (w_post, scale, w_pre))
    if y_out is not None:
        _check_like(y_out, torch.float32, y.shape, device, "y_out")
    elif b is not None:
        y_out = _empty_like(stream, y)
    if rstd is not None:
        _check_like(rstd, torch.float32, (2, y.shape[0]), device, "rstd")
    elif save_rstd:
        rstd = _new(stream, torch.empty, (2, y.shape[0]), dtype=torch.float32, device=device)
    _raise(_on(device, load_library().rampde_join_fwd, C.byref(j), _at(y), _at(b), _at(gate), _at(w_post), _at(scale), _at(w_pre),
               _at(y_out), _at(x), _at(rstd), _stream_of(stream, device)))
    return (y if b is None else y_out), x, rstd


def _like_of(stream, grad, t, name):
    """The gradient's tensor: as given, or one like its input's"""
    if t is None:
        if grad is not None:
            raise ValueError(f"{name}: there is no input that it would be the gradient of")
        return None
    if grad is None:
        return _empty_like(stream, t)
    _check_like(grad, t.dtype, t.shape, t.device, name, contiguous=False)
    if t.shape[0] > 1 and grad.stride(0) != t.stride(0):
        raise ValueError(f"{name}: row pitch {grad.stride(0)} is not that of its input, {t.stride(0)}")
    return grad


def rampde_join_bwd(join: Join, y_out: torch.Tensor, b: Optional[torch.Tensor], rstd: torch.Tensor,
                    dy_out: Optional[torch.Tensor] = None, dx: Optional[torch.Tensor] = None,
                    gate: Optional[torch.Tensor] = None, w_post: Optional[torch.Tensor] = None,
                    scale: Optional[torch.Tensor] = None, w_pre: Optional[torch.Tensor] = None,
                    dy: Optional[torch.Tensor] = None, dw_post: Optional[torch.Tensor] = None,
                    dscale: Optional[torch.Tensor] = None, dw_pre: Optional[torch.Tensor] = None,
                    db: Optional[torch.Tensor] = None, dgate: Optional[torch.Tensor] = None,
                    workspace: Optional[torch.Tensor] = None, stream=None) -> JoinGrads:
    """Gradients of rampde_join_fwd from those of y' (dy_out) and of x (dx).  dw_post, dscale and dw_pre are accumulated into;
    where they are omitted, they are created for the parameters that are given.  `dy` may be dy_out; db and dgate, where
    given, have the row pitch of b and gate."""
    lib = load_library()
    device = y_out.device
    dtype = b.dtype if b is not None else dx.dtype if dx is not None else torch.bfloat16
    j = _join_descriptor(join, dtype, y_out, b, gate, dx, (w_post, scale, w_pre, dw_post, dscale, dw_pre))
    rows, cols = y_out.shape
    _check_like(rstd, torch.float32, (2, rows), device, "rstd")
    _check_like(dy_out, torch.float32, y_out.shape, device, "dy_out")
    if dy is None:
        dy = _empty_like(stream, y_out)
    _check_like(dy, torch.float32, y_out.shape, device, "dy")
    if dw_post is None and dscale is None and dw_pre is None:
        j.write_grads = 1
        new = _new(stream, torch.empty, (3, cols), dtype=torch.float32, device=device).unbind()
    else:
        new = _new(stream, torch.zeros, (3, cols), dtype=torch.float32, device=device).unbind()
    dw_post, dscale, dw_pre = [(n if d is None else d) if w is not None or d is not None else None
                               for w, d, n in zip((w_post, scale, w_pre), (dw_post, dscale, dw_pre), new)]
    db, dgate = (_like_of(stream, d, t, name) for d, t, name in ((db, b, "db"), (dgate, gate, "dgate")))
    workspace = _space(_needed(int(lib.rampde_join_workspace_bytes(C.byref(j))), lib.rampde_join_fwd, C.byref(j)), workspace, device, stream)
    _raise(_on(device, lib.rampde_join_bwd, C.byref(j), _at(y_out), _at(b), _at(gate), _at(w_post), _at(scale), _at(w_pre),
               _at(rstd), _at(dy_out), _at(dx), _at(dy), _at(db), _at(dgate), _at(dw_post), _at(dscale), _at(dw_pre),
               _at(workspace), _size(workspace), _stream_of(stream, device)))
    return JoinGrads(dy, db, dgate, dw_post, dscale, dw_pre)


class Fp8:
    """A quantised operand of `rows` rows and `cols` columns: values [rows, cols up to a multiple of 128] and biased scale exponents
    [rows, blocks of 128 up to a multiple of 4], both uint8 (layout and meaning: include/rampde.h)."""

    def __init__(self, values: torch.Tensor, scales: torch.Tensor, cols: int):
        self.rows, self.cols, self.device = int(values.shape[0]), int(cols), values.device
        if self.rows < 1 or self.cols < 1:
            raise ValueError("empty operand")
        blocks = (self.cols + 127) // 128
        _check_like(values, torch.uint8, (self.rows, blocks * 128), self.device, "values")
        _check_like(scales, torch.uint8, (self.rows, (blocks + 3) // 4 * 4), self.device, "scales")
        self._values, self._scales, self._buffer = values, scales, None
        self._at = (values.data_ptr(), scales.data_ptr())

    @staticmethod
    def empty(rows: int, cols: int, device, stream=None):
        """Uninitialised, in one allocation: the scales behind the values"""
        blocks = (cols + 127) // 128
        return Fp8._empty(rows, cols, rows * blocks * 128, rows * ((blocks + 3) // 4 * 4), device, stream)

    @staticmethod
    def _empty(rows, cols, value_bytes, scale_bytes, device, stream):
        q = object.__new__(Fp8)
        q.rows, q.cols, q.device = rows, cols, device
        q._values = q._scales = None
        q._buffer = _new(stream, torch.empty, value_bytes + scale_bytes, dtype=torch.uint8, device=device)
        at = q._buffer.data_ptr()
        q._at = (at, at + value_bytes)
        return q

    @property
    def values(self) -> torch.Tensor:
        if self._values is None:
            self._values = self._buffer[:self._at[1] - self._at[0]].view(self.rows, -1)
        return self._values

    @property
    def scales(self) -> torch.Tensor:
        if self._scales is None:
            self._scales = self._buffer[self._at[1] - self._at[0]:].view(self.rows, -1)
        return self._scales

    def dequantize(self) -> torch.Tensor:
        """The values that the operand stands for, fp32 (a convenience for inspection, not a kernel)"""
        scale = torch.exp2(self.scales.double() - 127).repeat_interleave(128, 1)[:, :self.cols]
        return (self.values.view(torch.float8_e4m3fn).double()[:, :self.cols] * scale).float()


@functools.lru_cache(maxsize=1024)
def _quantize_plan(shape, stride, mode):
    """(mode's code, R, K, row pitch, sizes of the operand, sizes of the transpose or None); sizes as Fp8._empty takes them"""
    if len(shape) != 2 or min(shape) < 1:
        raise ValueError(f"src: need [rows, cols], got {tuple(shape)}")
    if not _rows_apart(shape, stride):
        raise ValueError(f"src: need a row-wise contiguous tensor, got {tuple(shape)} (strides {stride})")
    R, K = shape
    lib = load_library()

    def sizes(rows, cols):
        return rows, cols, int(lib.rampde_fp8_value_bytes(rows, cols)), int(lib.rampde_fp8_scale_bytes(rows, cols))
    code = _FP8_MODES.get(mode)
    if code is None:
        raise ValueError(f"mode: need one of {', '.join(_FP8_MODES)}, got {mode!r}")
    return code, R, K, stride[0] if R > 1 else 0, sizes(K, R) if code == 1 else sizes(R, K), sizes(K, R) if code == 2 else None


def rampde_fp8_quantize(src: torch.Tensor, mode: str = "rows", out: Optional[Fp8] = None, out_t: Optional[Fp8] = None, stream=None):
    """src [R, K] in 8-bit floating point with a power-of-two scale for every 128 values.  mode "rows": an operand of R rows, blocks
    along them; "cols": the transpose, an operand of K rows; "blocks": blocks of 128 x 128, returns (operand, its transpose)."""
    low, device = _type_of(src, "src"), src.device
    code, R, K, ld, shape, shape_t = _quantize_plan(src.shape, src.stride(), mode)
    if out is None:
        out = Fp8._empty(*shape, device, stream)
    elif (out.rows, out.cols) != shape[:2] or out.device != device:
        raise ValueError(f"out: need an operand of shape {shape[:2]} on {device}")
    if out_t is None:
        if shape_t is not None:
            out_t = Fp8._empty(*shape_t, device, stream)
    elif shape_t is None or (out_t.rows, out_t.cols) != shape_t[:2] or out_t.device != device:
        raise ValueError(f"out_t: need {'no operand' if shape_t is None else f'an operand of shape {shape_t[:2]} on {device}'}")
    t_values, t_scales = (None, None) if out_t is None else out_t._at
    _raise(_on(device, _lib.rampde_fp8_quantize, low, code, R, K, src.data_ptr(), ld, *out._at, t_values, t_scales,
               _stream_of(stream, device)))
    return out if out_t is None else (out, out_t)


@functools.lru_cache(maxsize=1024)
def _fp8_workspace(M: int, N: int, K: int) -> int:
    nbytes = _needed(int(load_library().rampde_fp8_workspace_bytes(M, N, K)))
    return 0 if nbytes == 256 else nbytes


def rampde_fp8_matmul(a: Fp8, b: Fp8, dtype=torch.bfloat16, out: Optional[torch.Tensor] = None, accumulate: bool = False,
                      workspace: Optional[torch.Tensor] = None, stream=None, short_sums: bool = False) -> torch.Tensor:
    """a b^T of two quantised operands, summed in fp32 and rounded once to `dtype`; with `accumulate` added to `out` (fp32).
    `short_sums` (results of 16 bits): rampde_fp8_matmul_short, faster, the sums of 8 products keep 13 binary places."""
    device = a.device
    if a.cols != b.cols or b.device != device:
        raise ValueError(f"operands: need the same number of columns on one GPU, got {a.cols} on {device} and {b.cols} on {b.device}")
    M, N, K = a.rows, b.rows, a.cols
    if out is None:
        if accumulate:
            raise ValueError("accumulate: need `out`")
        out = _new(stream, torch.empty, (M, N), dtype=dtype, device=device)
    else:
        _check_like(out, out.dtype, (M, N), device, "out", contiguous=False)
    c_type = _type_of(out, "out")
    workspace = _space(_fp8_workspace(M, N, K), workspace, device, stream)
    ldc, at, size, st = out.stride(0) if M > 1 else 0, _at(workspace), _size(workspace), _stream_of(stream, device)
    if short_sums:
        if accumulate or c_type == F32:
            raise ValueError("short_sums: results of 16 bits, not accumulated")
        _raise(_on(device, _lib.rampde_fp8_matmul_short, M, N, K, *a._at, *b._at, c_type, _at(out), ldc, at, size, st))
    else:
        _raise(_on(device, _lib.rampde_fp8_matmul, M, N, K, *a._at, *b._at, c_type, 1 if accumulate else 0, _at(out), ldc, at, size, st))
    return out
