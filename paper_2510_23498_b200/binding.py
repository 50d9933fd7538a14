"""ctypes binding of the C ABI in include/mpode.h: same names, argument marshalling only.

PyTorch is used for device memory and streams, nothing else: every step of Alg. 1 / Alg. 2 runs in the
library's kernels.  There is no CPU fallback: if the shared library is missing and cannot be built, importing
the entry points raises.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import Optional, Sequence

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "libmpode.so")

# enums of mpode.h
OK, ERR_INVALID_ARG, ERR_UNSUPPORTED, ERR_WORKSPACE_TOO_SMALL, ERR_CUDA, ERR_BAD_STATE, ERR_NONFINITE_INPUT, \
    ERR_SCALE_FAILED, WARN_NONFINITE_GRAD = range(9)
DTYPES = {"f32": 0, "bf16": 1, "f16": 2}
SCALINGS = {"none": 0, "none_safe": 1, "dynamic": 2}
ACTS = {"none": 0, "tanh": 1, "softplus": 2, "relu": 3}
KINDS = {"mlp": 0, "linear": 0, "conv": 1, "cnf": 2, "scalar_poly": 3, "parabolic": 4, "cnf_hyper": 5}
NORMS = {"none": 0, "rms": 1, "meanvar": 2}
NO_OVERRIDE = -2147483648

EXPORTS = [
    "mpode_tableau_euler", "mpode_tableau_rk4", "mpode_create", "mpode_destroy", "mpode_param_count",
    "mpode_state_width", "mpode_workspace_bytes", "mpode_trajectory_bytes", "mpode_forward", "mpode_backward",
    "mpode_io_bytes", "mpode_forward_host", "mpode_backward_host", "mpode_get_stats", "mpode_status_string",
    "mpode_last_error", "mpode_set_profiling", "mpode_collect_profile", "mpode_backward_static_workspace",
    "mpode_debug_waits", "mpode_backward_ex", "mpode_operator_error", "mpode_recurrence_forward", "mpode_recurrence_backward",
    "mpode_residual_workspace_bytes", "mpode_residual_forward", "mpode_residual_backward", "mpode_dropout",
]
STATIC_WORKSPACE_BYTES = 32 * 1024 * 1024


class VelocityDesc(C.Structure):
    _fields_ = [("kind", C.c_int), ("d", C.c_int), ("n_layers", C.c_int), ("widths", C.POINTER(C.c_int)),
                ("act", C.c_int), ("append_time", C.c_int), ("has_bias", C.c_int),
                ("H", C.c_int), ("W", C.c_int), ("C", C.c_int), ("n_intervals", C.c_int), ("instance_norm", C.c_int)]


class Tableau(C.Structure):
    _fields_ = [("stages", C.c_int), ("a", C.POINTER(C.c_double)), ("b", C.POINTER(C.c_double)),
                ("c", C.POINTER(C.c_double))]


class Policy(C.Structure):
    _fields_ = [("low", C.c_int), ("scaling", C.c_int), ("k_max", C.c_int), ("growth_rule", C.c_int),
                ("round_increment", C.c_int), ("init_scale_exp_override", C.c_int), ("time_gradient", C.c_int)]


class ScaleLog(C.Structure):
    _fields_ = [("n_steps", C.c_int), ("exp_used", C.POINTER(C.c_int)), ("attempts", C.POINTER(C.c_int)),
                ("doubled", C.POINTER(C.c_ubyte)), ("first_failed_step", C.c_int)]


class Stats(C.Structure):
    _fields_ = [("kernel_launches", C.c_longlong), ("retries", C.c_longlong), ("host_syncs", C.c_longlong),
                ("tc_contractions", C.c_longlong), ("simt_contractions", C.c_longlong), ("fused_launches", C.c_longlong),
                ("whole_solve_launches", C.c_longlong), ("step_waits", C.c_longlong)]


class RecurrenceDesc(C.Structure):
    _fields_ = [("low", C.c_int), ("n_seq", C.c_int), ("n_steps", C.c_int), ("width", C.c_int), ("coupled", C.c_int),
                ("zero_behind", C.c_int), ("in_seq_stride", C.c_longlong), ("in_step_stride", C.c_longlong), ("out_seq_stride", C.c_longlong),
                ("out_step_stride", C.c_longlong)]


class ResidualDesc(C.Structure):
    _fields_ = [("low", C.c_int), ("width", C.c_int), ("post_norm", C.c_int), ("pre_norm", C.c_int), ("eps", C.c_float), ("h", C.c_float),
                ("p_drop", C.c_float), ("site", C.c_uint), ("ld_y", C.c_longlong), ("ld_u", C.c_longlong), ("ld_gate", C.c_longlong),
                ("ld_z", C.c_longlong)]


_lib = None


def load_library(build_if_missing: bool = True) -> C.CDLL:
    """Load libmpode.so (building it with nvcc first if it is absent).  Raises if neither works."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(_LIB_PATH):
        if not build_if_missing:
            raise RuntimeError("libmpode.so is missing; run `python -m paper_2510_23498_b200.build`")
        from . import build as _build
        _build.build()
    lib = C.CDLL(_LIB_PATH)
    vp, sz, i32 = C.c_void_p, C.c_size_t, C.c_int
    lib.mpode_tableau_euler.restype = C.POINTER(Tableau)
    lib.mpode_tableau_rk4.restype = C.POINTER(Tableau)
    lib.mpode_create.argtypes = [C.POINTER(vp), C.POINTER(VelocityDesc), i32, i32, C.POINTER(Policy)]
    lib.mpode_create.restype = i32
    lib.mpode_destroy.argtypes = [vp]
    lib.mpode_destroy.restype = None
    for name in ("mpode_param_count", "mpode_state_width", "mpode_workspace_bytes", "mpode_io_bytes"):
        getattr(lib, name).argtypes = [vp]
        getattr(lib, name).restype = sz
    lib.mpode_trajectory_bytes.argtypes = [vp, i32]
    lib.mpode_trajectory_bytes.restype = sz
    lib.mpode_forward.argtypes = [vp, vp, vp, vp, C.POINTER(C.c_float), i32, C.POINTER(Tableau), vp, vp, vp, vp, sz]
    lib.mpode_forward.restype = i32
    lib.mpode_backward.argtypes = [vp, vp, vp, vp, vp, i32, C.POINTER(ScaleLog), vp, sz]
    lib.mpode_backward.restype = i32
    lib.mpode_backward_ex.argtypes = [vp, vp, vp, vp, vp, vp, i32, C.POINTER(C.c_float), C.POINTER(ScaleLog), vp, sz]
    lib.mpode_backward_ex.restype = i32
    lib.mpode_backward_static_workspace.argtypes = [vp, vp, vp, vp, vp, i32, C.POINTER(ScaleLog)]
    lib.mpode_backward_static_workspace.restype = i32
    lib.mpode_forward_host.argtypes = [vp, vp, vp, vp, C.POINTER(C.c_float), i32, C.POINTER(Tableau), vp, vp, vp, vp,
                                       vp, sz]
    lib.mpode_forward_host.restype = i32
    lib.mpode_backward_host.argtypes = [vp, vp, vp, vp, vp, C.POINTER(ScaleLog), vp, vp, sz]
    lib.mpode_backward_host.restype = i32
    lib.mpode_get_stats.argtypes = [vp, C.POINTER(Stats)]
    lib.mpode_get_stats.restype = None
    lib.mpode_debug_waits.argtypes = [vp, C.c_ulonglong, i32]
    lib.mpode_debug_waits.restype = None
    lib.mpode_set_profiling.argtypes = [vp, i32]
    lib.mpode_set_profiling.restype = None
    lib.mpode_collect_profile.argtypes = [vp, C.POINTER(C.c_double), C.POINTER(C.c_longlong), C.POINTER(C.c_double)]
    lib.mpode_collect_profile.restype = i32
    lib.mpode_status_string.argtypes = [i32]
    lib.mpode_status_string.restype = C.c_char_p
    lib.mpode_last_error.argtypes = [vp]
    lib.mpode_last_error.restype = C.c_char_p
    lib.mpode_operator_error.argtypes = []
    lib.mpode_operator_error.restype = C.c_char_p
    lib.mpode_recurrence_forward.argtypes = [C.POINTER(RecurrenceDesc)] + [vp] * 7
    lib.mpode_recurrence_forward.restype = i32
    lib.mpode_recurrence_backward.argtypes = [C.POINTER(RecurrenceDesc)] + [vp] * 12
    lib.mpode_recurrence_backward.restype = i32
    lib.mpode_residual_workspace_bytes.argtypes = [C.POINTER(ResidualDesc), i32]
    lib.mpode_residual_workspace_bytes.restype = sz
    lib.mpode_residual_forward.argtypes = [C.POINTER(ResidualDesc), vp, i32] + [vp] * 10
    lib.mpode_residual_forward.restype = i32
    lib.mpode_residual_backward.argtypes = [C.POINTER(ResidualDesc), vp, i32] + [vp] * 10 + [i32] + [vp] * 6 + [i32, vp, vp, sz]
    lib.mpode_residual_backward.restype = i32
    lib.mpode_dropout.argtypes = [i32, vp, C.c_longlong, i32, vp, C.c_longlong, vp, C.c_longlong, C.c_float, vp, C.c_uint, vp]
    lib.mpode_dropout.restype = i32
    _lib = lib
    return lib


class MpodeError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__("mpode status %d: %s" % (status, message))
        self.status = status


def make_tableau(a: Sequence[Sequence[float]], b: Sequence[float], c: Sequence[float]):
    """Build a Tableau struct; keeps the backing arrays alive on the returned object."""
    s = len(b)
    aa = (C.c_double * (s * s))(*[float(a[j][l]) for j in range(s) for l in range(s)])
    bb = (C.c_double * s)(*[float(x) for x in b])
    cc = (C.c_double * s)(*[float(x) for x in c])
    t = Tableau(s, C.cast(aa, C.POINTER(C.c_double)), C.cast(bb, C.POINTER(C.c_double)),
                C.cast(cc, C.POINTER(C.c_double)))
    t._keep = (aa, bb, cc)
    return t


NAMED_TABLEAUX = {
    "euler": ([[0.0]], [1.0], [0.0]),
    "midpoint": ([[0, 0], [0.5, 0]], [0.0, 1.0], [0.0, 0.5]),
    "heun": ([[0, 0], [1.0, 0]], [0.5, 0.5], [0.0, 1.0]),
    "kutta3": ([[0, 0, 0], [0.5, 0, 0], [-1.0, 2.0, 0]], [1 / 6, 2 / 3, 1 / 6], [0.0, 0.5, 1.0]),
    "rk4": ([[0, 0, 0, 0], [0.5, 0, 0, 0], [0, 0.5, 0, 0], [0, 0, 1.0, 0]], [1 / 6, 1 / 3, 1 / 3, 1 / 6],
            [0.0, 0.5, 0.5, 1.0]),
    "rk38": ([[0, 0, 0, 0], [1 / 3, 0, 0, 0], [-1 / 3, 1.0, 0, 0], [1.0, -1.0, 1.0, 0]],
             [1 / 8, 3 / 8, 3 / 8, 1 / 8], [0.0, 1 / 3, 2 / 3, 1.0]),
}


def _ptr(t) -> int:
    """Device (or pinned host) address of a torch tensor, or 0."""
    return 0 if t is None else t.data_ptr()


class Context:
    """Thin owner of one mpode_ctx plus the torch-allocated workspace and trajectory."""

    def __init__(self, vel: dict, batch: int, max_steps: int, low: str = "bf16", scaling: str = "none",
                 k_max: int = 10, growth_rule: int = 0, round_increment: int = 0,
                 init_scale_exp_override: Optional[int] = None, device: str = "cuda:0", time_gradient: bool = False):
        import torch
        self.torch = torch
        self.lib = load_library()
        self.device = torch.device(device)
        self.low = low
        kind = vel["kind"]
        widths = vel.get("widths")
        if kind == "cnf_hyper":
            widths = [int(vel["hidden"]), int(vel["w"])]
        self._widths = (C.c_int * len(widths))(*widths) if widths else None
        desc = VelocityDesc(KINDS[kind], int(vel["d"]), (len(widths) - 1) if widths else 0,
                            C.cast(self._widths, C.POINTER(C.c_int)) if widths else None,
                            ACTS[vel.get("act", "none")], int(bool(vel.get("append_time", False))),
                            int(bool(vel.get("bias", kind != "linear"))), int(vel.get("H", 0)), int(vel.get("W", 0)),
                            int(vel.get("C", 0)), int(vel.get("n_intervals", 0)), int(bool(vel.get("norm", True))))
        pol = Policy(DTYPES[low], SCALINGS[scaling], k_max, growth_rule, round_increment,
                     NO_OVERRIDE if init_scale_exp_override is None else int(init_scale_exp_override), 1 if time_gradient else 0)
        self.time_gradient = bool(time_gradient)
        h = C.c_void_p()
        st = self.lib.mpode_create(C.byref(h), C.byref(desc), batch, max_steps, C.byref(pol))
        if st != OK:
            raise MpodeError(st, self.lib.mpode_status_string(st).decode())
        self.h = h
        self.batch = batch
        self.max_steps = max_steps
        self.p = int(self.lib.mpode_param_count(h))
        self.D = int(self.lib.mpode_state_width(h))
        self.d = int(vel["d"])
        self.workspace_bytes = int(self.lib.mpode_workspace_bytes(h))
        with torch.cuda.device(self.device):
            self.workspace = torch.empty(self.workspace_bytes + 256, dtype=torch.uint8, device=self.device)
        self.low_torch = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}[low]
        self.traj = None
        self.io = None

    def close(self):
        if getattr(self, "h", None):
            self.lib.mpode_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _check(self, st: int, allow=()):
        if st != OK and st not in allow:
            raise MpodeError(st, self.lib.mpode_last_error(self.h).decode() or self.lib.mpode_status_string(st).decode())
        return st

    def _stream(self) -> int:
        return int(self.torch.cuda.current_stream(self.device).cuda_stream)

    def _tableau(self, tab):
        if isinstance(tab, str):
            if tab == "euler":
                return self.lib.mpode_tableau_euler()
            if tab == "rk4":
                return self.lib.mpode_tableau_rk4()
            self._tab_keep = make_tableau(*NAMED_TABLEAUX[tab])
            return C.pointer(self._tab_keep)
        self._tab_keep = tab
        return C.pointer(tab)

    def forward(self, theta, y0, tgrid: np.ndarray, tab="rk4", probe=None, traj=None):
        """mpode_forward on device tensors.  Returns (traj [(N+1), B, d] low, yT [B, D] fp32).  `traj` may be a preallocated
        contiguous tensor of that shape (e.g. a view at an odd offset of a larger buffer)."""
        torch = self.torch
        n = int(len(tgrid) - 1)
        tg = np.ascontiguousarray(tgrid, dtype=np.float32)
        if traj is not None:
            assert tuple(traj.shape) == (n + 1, self.batch, self.d) and traj.dtype == self.low_torch and traj.is_contiguous()
            self.traj = traj
        elif self.traj is None or tuple(self.traj.shape) != (n + 1, self.batch, self.d) or self.traj.dtype != self.low_torch:
            self.traj = None                 # release the old buffer first: two trajectories must never be alive together
            self.traj = torch.empty((n + 1, self.batch, self.d), dtype=self.low_torch, device=self.device)
        yT = torch.empty((self.batch, self.D), dtype=torch.float32, device=self.device)
        self._keep = (theta, y0, probe, tg)
        st = self.lib.mpode_forward(self.h, self._stream(), _ptr(theta), _ptr(y0),
                                    tg.ctypes.data_as(C.POINTER(C.c_float)), n, self._tableau(tab), _ptr(probe),
                                    _ptr(self.traj), _ptr(yT), _ptr(self.workspace), self.workspace_bytes)
        self._check(st)
        return self.traj, yT

    def backward(self, dL_dyT, accumulate_into=None, want_log: bool = True, running_cot=None, want_dt: bool = False):
        """mpode_backward (mpode_backward_ex when a running-cost cotangent [N, B, D] or dL/dt is asked for).
        Returns (dL/dy0 [B, D], dL/dtheta [p], log dict or None, status); with want_dt the log dict carries "dL_dt"."""
        torch = self.torch
        n = self.traj.shape[0] - 1
        a0 = torch.empty((self.batch, self.D), dtype=torch.float32, device=self.device)
        g = accumulate_into if accumulate_into is not None else torch.empty(self.p, dtype=torch.float32, device=self.device)
        log = None
        if want_log:
            e = (C.c_int * n)()
            k = (C.c_int * n)()
            dbl = (C.c_ubyte * n)()
            log = ScaleLog(n, C.cast(e, C.POINTER(C.c_int)), C.cast(k, C.POINTER(C.c_int)),
                           C.cast(dbl, C.POINTER(C.c_ubyte)), -1)
        dt_arr = None
        if running_cot is not None or want_dt:
            dt_arr = np.zeros(n + 1, dtype=np.float32) if want_dt else None
            st = self.lib.mpode_backward_ex(self.h, self._stream(), _ptr(dL_dyT), _ptr(running_cot), _ptr(a0), _ptr(g),
                                            1 if accumulate_into is not None else 0,
                                            dt_arr.ctypes.data_as(C.POINTER(C.c_float)) if want_dt else None,
                                            C.byref(log) if log else None, _ptr(self.workspace), self.workspace_bytes)
        else:
            st = self.lib.mpode_backward(self.h, self._stream(), _ptr(dL_dyT), _ptr(a0), _ptr(g),
                                         1 if accumulate_into is not None else 0, C.byref(log) if log else None,
                                         _ptr(self.workspace), self.workspace_bytes)
        out_log = None
        if log is not None:
            out_log = dict(exp_used=list(e), attempts=list(k), doubled=[int(x) for x in dbl],
                           first_failed_step=int(log.first_failed_step))
        if dt_arr is not None:
            out_log = dict(out_log or {}, dL_dt=dt_arr)
        if st == ERR_SCALE_FAILED:
            return a0, g, out_log, st
        self._check(st, allow=(WARN_NONFINITE_GRAD,))
        return a0, g, out_log, st

    def backward_static_workspace(self, dL_dyT, out_a0=None, out_g=None, accumulate: bool = False, log_arrays=None):
        """mpode_backward_static_workspace: the backward pass on the library's own static device workspace (for callers
        that cannot allocate device memory).  With `out_a0` / `out_g` given (preallocated tensors) this wrapper allocates
        nothing either; `log_arrays` = (exp_used, attempts, doubled) ctypes arrays of n_steps entries receive the scale log.
        Returns (dL/dy0, dL/dtheta, status)."""
        torch = self.torch
        a0 = out_a0 if out_a0 is not None else torch.empty((self.batch, self.D), dtype=torch.float32, device=self.device)
        g = out_g if out_g is not None else torch.empty(self.p, dtype=torch.float32, device=self.device)
        log = None
        if log_arrays is not None:
            e, k, dbl = log_arrays
            log = ScaleLog(len(e), C.cast(e, C.POINTER(C.c_int)), C.cast(k, C.POINTER(C.c_int)), C.cast(dbl, C.POINTER(C.c_ubyte)), -1)
        st = self.lib.mpode_backward_static_workspace(self.h, self._stream(), _ptr(dL_dyT), _ptr(a0), _ptr(g),
                                                      1 if accumulate else 0, C.byref(log) if log is not None else None)
        self._check(st, allow=(WARN_NONFINITE_GRAD,))
        return a0, g, st

    # ---- host-buffer entry points (pinned torch tensors or numpy arrays as HOST pointers)
    def ensure_io(self):
        if self.io is None:
            nbytes = int(self.lib.mpode_io_bytes(self.h))
            self.io = self.torch.empty(nbytes + 256, dtype=self.torch.uint8, device=self.device)
        return self.io

    def forward_host(self, theta_h, y0_h, tgrid: np.ndarray, yT_h, tab="rk4", probe_h=None):
        torch = self.torch
        n = int(len(tgrid) - 1)
        tg = np.ascontiguousarray(tgrid, dtype=np.float32)
        if self.traj is None or self.traj.shape[0] != n + 1:
            self.traj = torch.empty((n + 1, self.batch, self.d), dtype=self.low_torch, device=self.device)
        self.ensure_io()
        self._keep = (theta_h, y0_h, probe_h, tg)
        st = self.lib.mpode_forward_host(self.h, self._stream(), _ptr(theta_h), _ptr(y0_h),
                                         tg.ctypes.data_as(C.POINTER(C.c_float)), n, self._tableau(tab),
                                         _ptr(probe_h), _ptr(self.traj), _ptr(yT_h), _ptr(self.io),
                                         _ptr(self.workspace), self.workspace_bytes)
        self._check(st)

    def backward_host(self, dL_dyT_h, dL_dy0_h, dL_dtheta_h):
        st = self.lib.mpode_backward_host(self.h, self._stream(), _ptr(dL_dyT_h), _ptr(dL_dy0_h), _ptr(dL_dtheta_h),
                                          None, _ptr(self.io), _ptr(self.workspace), self.workspace_bytes)
        return self._check(st, allow=(WARN_NONFINITE_GRAD,))

    def set_profiling(self, on: bool):
        self.lib.mpode_set_profiling(self.h, 1 if on else 0)

    def collect_profile(self) -> dict:
        ms = (C.c_double * 4)()
        n = (C.c_longlong * 4)()
        fl = (C.c_double * 4)()
        self._check(self.lib.mpode_collect_profile(self.h, ms, n, fl))
        names = ("forward", "dgrad", "wgrad", "fused_backward")
        return {names[k]: dict(ms=float(ms[k]), launches=int(n[k]), flops=float(fl[k])) for k in range(4)}

    def stats(self) -> dict:
        s = Stats()
        self.lib.mpode_get_stats(self.h, C.byref(s))
        return dict(kernel_launches=int(s.kernel_launches), retries=int(s.retries), host_syncs=int(s.host_syncs),
                    tc_contractions=int(s.tc_contractions), simt_contractions=int(s.simt_contractions),
                    fused_launches=int(s.fused_launches), whole_solve_launches=int(s.whole_solve_launches),
                    step_waits=int(s.step_waits))

    def debug_waits(self, wait_limit_ns: int = 0, starve_forward: bool = False):
        """Test hook of the bounded device-side waits (see mpode_debug_waits)."""
        self.lib.mpode_debug_waits(self.h, int(wait_limit_ns), 1 if starve_forward else 0)


# ---- operators of sequence and residual networks (mpode_recurrence_*, mpode_residual_*, mpode_dropout).  They need no Context: results go to new
# tensors or to the caller's, on the current stream of the inputs' device.  A call for one token runs a few microseconds on the GPU, so what the host does
# for it is kept short: shapes and strides are compared as they are, and a device guard is entered only where another device is current.
_torch = None
_LOW = {}
_raw_stream = None


def _load():
    """(library, torch), loaded once."""
    global _torch, _raw_stream
    if _torch is None:
        import torch
        # the current stream's handle without the Stream object around it (3 us less a call)
        _raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda device: torch.cuda.current_stream(device).cuda_stream)
        _LOW.update({torch.float32: 0, torch.bfloat16: 1, torch.float16: 2})
        load_library()
        _torch = torch
    return _lib, _torch


def _refuse(message: str):
    raise MpodeError(ERR_INVALID_ARG, message)


def _int32(**sizes):
    """Sizes that the C structures hold in 32 bits (ctypes would cut them off)."""
    for name, n in sizes.items():
        if not -0x80000000 <= n <= 0x7fffffff:
            raise MpodeError(ERR_UNSUPPORTED, "%s %d does not fit 32 bits" % (name, n))


def _site(n) -> int:
    n = int(n)
    if not -0x80000000 <= n <= 0xffffffff:
        _refuse("site %d does not fit 32 bits" % n)
    return n


def _low_of(t) -> int:
    low = _LOW.get(t.dtype)
    if low is None:
        _refuse("dtype %s is not one of float32, bfloat16, float16" % t.dtype)
    return low


def _run(entry, desc, tensors, args):
    """entry(desc, stream, *args) on the CUDA device of the first tensor, where all of them have to be."""
    lib, torch = _load()
    device = tensors[0].get_device()
    if device < 0:
        _refuse("the tensors have to be on a CUDA device")
    for t in tensors:
        if t is not None and t.get_device() != device:
            _refuse("tensors on %s and %s" % (tensors[0].device, t.device))
    if torch.cuda.current_device() == device:
        st = entry(desc, _raw_stream(device), *args)
    else:
        with torch.cuda.device(device):
            st = entry(desc, _raw_stream(device), *args)
    if st != OK:
        raise MpodeError(st, lib.mpode_operator_error().decode() or lib.mpode_status_string(st).decode())


def _expect(name: str, t, shape, dtype):
    if t is not None and (t.shape != shape or t.dtype != dtype or not t.is_contiguous()):
        _refuse("%s has to be a contiguous %s tensor of shape %s, not %s %s" % (name, dtype, tuple(shape), t.dtype, tuple(t.shape)))


def _layout(name: str, t, shape, dtype):
    """(sequence stride, step stride) of a [n_seq, n_steps, width] tensor whose channels lie side by side; the width where a dimension has one entry."""
    if t.shape != shape or t.dtype != dtype:
        _refuse("%s has to be a %s tensor of shape %s, not %s %s" % (name, dtype, tuple(shape), t.dtype, tuple(t.shape)))
    n, steps, width = shape
    a, b, c = t.stride()
    if c != 1 and width > 1:
        _refuse("the channels of %s have to lie side by side" % name)
    if n <= 1:
        a = width
    if steps <= 1:
        b = width
    if a == 0 or b == 0:
        _refuse("%s is broadcast along a dimension" % name)
    return a, b


def _same_layout(name: str, t, shape, dtype, layout):
    if t is not None and _layout(name, t, shape, dtype) != layout:
        _refuse("%s has to have the strides %s" % (name, layout))


def _like(t):
    """A tensor of the strides of t (a slice's gaps included)."""
    return _torch.empty_like(t) if t.is_contiguous() else _torch.empty_strided(t.shape, t.stride(), dtype=t.dtype, device=t.device)


def _sequences(x):
    if x.dim() != 3:
        _refuse("x has to be [n_seq, n_steps, width]")
    n, steps, width = x.shape
    if n > 0x7fffffff or steps > 0x7fffffff or width > 0x7fffffff:
        _int32(n_seq=n, n_steps=steps, width=width)
    return x.shape


def recurrence_forward(x, gate, y0=None, lengths=None, coupled: bool = True, y=None, yT=None):
    """mpode_recurrence_forward on x, gate [n_seq, n_steps, width] (any strides with the channels side by side, the same for both).
    Returns (y, yT): the stored trajectory (zero behind a sequence's length when allocated here, left alone there when given) and the float32 state
    behind the last step.  yT may be y0."""
    lib, torch = _load()
    shape = _sequences(x)
    n, steps, width = shape
    low, dtype = _low_of(x), x.dtype
    inner = _layout("x", x, shape, dtype)
    if gate.shape != shape or gate.dtype != dtype or gate.stride() != x.stride():
        _same_layout("gate", gate, shape, dtype, inner)
    zero_behind = 0
    if y is None:
        y = torch.empty_like(x)                                                   # (time-major inputs get a time-major trajectory)
        outer = inner if y.stride() == x.stride() else _layout("y", y, shape, dtype)
        if lengths is not None:
            zero_behind = 1
    else:
        outer = _layout("y", y, shape, dtype)
    states = (n, width)
    _expect("y0", y0, states, torch.float32)
    if yT is None:
        yT = x.new_empty(states, dtype=torch.float32) if y0 is None else torch.empty_like(y0)
    else:
        _expect("yT", yT, states, torch.float32)
    _expect("lengths", lengths, (n,), torch.int32)
    _run(lib.mpode_recurrence_forward, RecurrenceDesc(low, n, steps, width, 1 if coupled else 0, zero_behind, *inner, *outer),
         (x, gate, y0, lengths, y, yT), (x.data_ptr(), gate.data_ptr(), _ptr(y0), _ptr(lengths), y.data_ptr(), yT.data_ptr()))
    return y, yT


def recurrence_backward(x, gate, y, dL_dy, dL_dyT=None, y0=None, lengths=None, coupled: bool = True, dL_dx=None, dL_dgate=None, dL_dy0=None, flag=None):
    """mpode_recurrence_backward from the stored trajectory y.  dL_dy (or None) has the strides of y, dL_dx and dL_dgate those of x.
    Returns (dL_dx, dL_dgate, dL_dy0); the first two are zero behind a sequence's length when allocated here, left alone there when given.
    flag: int32 tensor of one element, set to 1 when a low-format gradient is not finite."""
    lib, torch = _load()
    shape = _sequences(x)
    n, steps, width = shape
    low, dtype = _low_of(x), x.dtype
    inner, outer = _layout("x", x, shape, dtype), _layout("y", y, shape, dtype)
    _same_layout("gate", gate, shape, dtype, inner)
    _same_layout("dL_dy", dL_dy, shape, dtype, outer)
    new = dL_dx is None and dL_dgate is None
    if new:
        dL_dx, dL_dgate = _like(x), _like(x)
    elif dL_dx is None or dL_dgate is None:
        _refuse("dL_dx and dL_dgate are given together or not at all")
    else:
        _same_layout("dL_dx", dL_dx, shape, dtype, inner)
        _same_layout("dL_dgate", dL_dgate, shape, dtype, inner)
    states = (n, width)
    if dL_dy0 is None:
        dL_dy0 = x.new_empty(states, dtype=torch.float32) if dL_dyT is None else torch.empty_like(dL_dyT)
    else:
        _expect("dL_dy0", dL_dy0, states, torch.float32)
    _expect("y0", y0, states, torch.float32)
    _expect("dL_dyT", dL_dyT, states, torch.float32)
    _expect("lengths", lengths, (n,), torch.int32)
    _expect("flag", flag, (1,), torch.int32)
    _run(lib.mpode_recurrence_backward, RecurrenceDesc(low, n, steps, width, 1 if coupled else 0, 1 if new and lengths is not None else 0, *inner, *outer),
         (x, gate, y, dL_dy, dL_dyT, y0, lengths, dL_dx, dL_dgate, dL_dy0, flag),
         (_ptr(x), _ptr(gate), _ptr(y0), _ptr(lengths), _ptr(y), _ptr(dL_dy), _ptr(dL_dyT), _ptr(dL_dx), _ptr(dL_dgate), _ptr(dL_dy0), _ptr(flag)))
    return dL_dx, dL_dgate, dL_dy0


def _rows(name: str, t, shape, dtype) -> int:
    """Row length of a [rows, width] tensor whose columns lie side by side."""
    if t is None:
        return 0
    if t.shape != shape or t.dtype != dtype:
        _refuse("%s has to be a %s tensor of shape %s, not %s %s" % (name, dtype, tuple(shape), t.dtype, tuple(t.shape)))
    ld, one = t.stride()
    if one != 1 and shape[1] > 1:
        _refuse("the columns of %s have to lie side by side" % name)
    if shape[0] <= 1:
        return shape[1]
    if ld < shape[1]:
        _refuse("the rows of %s overlap" % name)
    return ld


def _same_rows(name: str, t, shape, dtype, ld: int):
    if t is not None and _rows(name, t, shape, dtype) != ld:
        _refuse("%s has to have the row length %d" % (name, ld))


class ResidualStep:
    """mpode_residual_forward / mpode_residual_backward with a fixed width and settings.  The object holds the settings only: nothing of one call is
    kept for the next, and a call's scratch memory comes from torch's allocator, so that calls on several streams do not meet in it."""

    def __init__(self, width: int, low: str = "bf16", post_norm: str = "rms", pre_norm: str = "rms", eps: float = 1e-5, h: float = 1.0,
                 p: float = 0.0, site: int = 0):
        _, torch = _load()
        self.width, self.p, self.h, self.eps, self.site = int(width), float(p), float(h), float(eps), _site(site)
        _int32(width=self.width)
        self.low, self.post_norm, self.pre_norm = DTYPES[low], NORMS[post_norm], NORMS[pre_norm]
        self.low_torch = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}[low]

    def _desc(self, ld_y, ld_u, ld_gate, ld_z):
        return ResidualDesc(self.low, self.width, self.post_norm, self.pre_norm, self.eps, self.h, self.p, self.site, ld_y, ld_u, ld_gate, ld_z)

    def _shape(self, y, w_post, scale, w_pre, rng):
        if y.dim() != 2 or y.shape[1] != self.width:
            _refuse("the state has to be [rows, %d]" % self.width)
        if y.shape[0] > 0x7fffffff:
            _int32(rows=y.shape[0])
        one, f32 = (self.width,), _torch.float32
        _expect("w_post", w_post, one, f32)
        _expect("scale", scale, one, f32)
        _expect("w_pre", w_pre, one, f32)
        _expect("rng", rng, (2,), _torch.int64)
        return y.shape

    def forward(self, y, u=None, gate=None, w_post=None, scale=None, w_pre=None, rng=None, y_out=None, z=None, want_z: bool = True):
        """Returns (y', z, stats): the state behind the step (y itself without u), the next block's input (None with want_z=False) and the statistics
        that backward needs.  y_out may be y."""
        lib, torch = _load()
        f32, low = torch.float32, self.low_torch
        shape = self._shape(y, w_post, scale, w_pre, rng)
        ld_y = _rows("y", y, shape, f32)
        if y_out is not None:
            _same_rows("y_out", y_out, shape, f32, ld_y)
        elif u is not None:
            y_out = _like(y)
        if want_z and z is None:
            z = torch.empty_like(u) if u is not None and u.is_contiguous() else y.new_empty(shape, dtype=low)
        stats = y.new_empty((shape[0], 4))
        desc = self._desc(ld_y, _rows("u", u, shape, low), _rows("gate", gate, shape, low), _rows("z", z, shape, low))
        _run(lib.mpode_residual_forward, desc, (y, u, gate, w_post, scale, w_pre, rng, y_out, z),
             (shape[0], _ptr(y), _ptr(u), _ptr(gate), _ptr(w_post), _ptr(scale), _ptr(w_pre), _ptr(rng), _ptr(y_out), _ptr(z), _ptr(stats)))
        return (y if y_out is None else y_out), z, stats

    def backward(self, y_new, u=None, stats=None, dL_dy=None, dL_dz=None, gate=None, w_post=None, scale=None, w_pre=None, rng=None, scale_exp: int = 0,
                 accumulate_into: Optional[dict] = None, want_weights: bool = True, flag=None):
        """dL_dy: adjoint of y' (float32), dL_dz: cotangent of z (low format, times 2^scale_exp).  Returns a dict with "dy" (adjoint of y), "du" and "dgate" (low
        format, times 2^scale_exp; None without u, gate) and the gradients "dw_post", "dscale", "dw_pre" of the weights that were given (added to the
        tensors of that name in accumulate_into when given).  flag: int32 tensor of one element, set to 1 when du or dgate is not finite."""
        lib, torch = _load()
        f32, low = torch.float32, self.low_torch
        shape = self._shape(y_new, w_post, scale, w_pre, rng)
        rows = shape[0]
        _int32(scale_exp=int(scale_exp))
        _expect("stats", stats, (rows, 4), f32)
        _expect("flag", flag, (1,), torch.int32)
        ld_y, ld_u, ld_gate = _rows("y_new", y_new, shape, f32), _rows("u", u, shape, low), _rows("gate", gate, shape, low)
        _same_rows("dL_dy", dL_dy, shape, f32, ld_y)
        out = {"dy": _like(y_new), "du": None if u is None else _like(u), "dgate": None if gate is None else _like(gate)}
        for key, w in (("dw_post", w_post), ("dscale", scale), ("dw_pre", w_pre)):
            g = None
            if want_weights and w is not None:
                if accumulate_into is None:
                    g = torch.empty_like(w)
                else:
                    g = accumulate_into[key]
                    _expect(key, g, (self.width,), f32)
            out[key] = g
        grads = (out["dw_post"], out["dscale"], out["dw_pre"])
        desc = self._desc(ld_y, ld_u, ld_gate, _rows("dL_dz", dL_dz, shape, low))
        ws, nbytes = None, 0
        if rows > 0 and not (grads[0] is None and grads[1] is None and grads[2] is None):
            nbytes = lib.mpode_residual_workspace_bytes(desc, rows)
            ws = y_new.new_empty(nbytes // 4)
        _run(lib.mpode_residual_backward, desc, (y_new, u, stats, dL_dy, dL_dz, gate, w_post, scale, w_pre, rng, flag) + grads,
             (rows, _ptr(y_new), _ptr(u), _ptr(gate), _ptr(w_post), _ptr(scale), _ptr(w_pre), _ptr(rng), _ptr(stats), _ptr(dL_dy), _ptr(dL_dz),
              int(scale_exp), _ptr(out["dy"]), _ptr(out["du"]), _ptr(out["dgate"]), _ptr(grads[0]), _ptr(grads[1]), _ptr(grads[2]),
              0 if accumulate_into is None else 1, _ptr(flag), _ptr(ws), nbytes))
        return out


def dropout(x, p: float, rng, site: int = 0, out=None, flag=None):
    """mpode_dropout on the rows of x [..., width] (2-D with any row length, or contiguous); on a cotangent it is the backward pass.
    rng: int64 tensor {seed, step} on the device.  out may be x."""
    lib, torch = _load()
    low, dim = _low_of(x), x.dim()
    if dim == 0:
        _refuse("x has to have rows")
    if out is None:
        out = torch.empty_like(x)
    elif out.shape != x.shape or out.dtype != x.dtype:
        _refuse("out has to be of the shape and type of x")
    if dim == 2:
        shape = x.shape
        ld_x, ld_out = _rows("x", x, shape, x.dtype), _rows("out", out, shape, x.dtype)
    else:
        if not x.is_contiguous() or not out.is_contiguous():
            _refuse("x and out have to be contiguous, or 2-D with their columns side by side")
        shape = (x.numel() // max(x.shape[-1], 1), x.shape[-1])
        ld_x = ld_out = shape[1]
    if shape[1] > 0x7fffffff:
        _int32(width=shape[1])
    _expect("rng", rng, (2,), torch.int64)
    _expect("flag", flag, (1,), torch.int32)
    _run(lib.mpode_dropout, low, (x, rng, out, flag), (shape[0], shape[1], _ptr(x), ld_x, _ptr(out), ld_out, p, _ptr(rng), _site(site), _ptr(flag)))
    return out
