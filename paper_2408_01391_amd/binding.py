"""Thin ctypes binding of libftkmeans (argument marshalling only).

PyTorch provides device memory and the current stream; every step of the hot path runs
inside the HIP library.  There is no CPU fallback: if the library is missing or a call
fails, an exception is raised.  The calls compute values: torch records nothing of them, and results come without
``requires_grad`` whatever the operands' is (gradients are calls of their own).
"""
from __future__ import annotations

import ctypes
import itertools
import operator
from pathlib import Path

import torch

FT_OFF, FT_DETECT, FT_CORRECT, FT_STRICT = 0, 1, 2, 3
F32, F64, BF16, F16 = 0, 1, 2, 3

_LIB_PATH = Path(__file__).resolve().parent / "libftkmeans.so"
_lib = None

STAT_FIELDS = ("tiles_checked", "injected", "detected", "corrected", "recomputed",
               "uncorrectable", "refined", "max_residual_ppm")


class Geometry(ctypes.Structure):
    _fields_ = [(n, ctypes.c_uint32) for n in
                ("workgroups", "waves_per_workgroup", "tiles_per_wave", "regs_per_tile", "lanes", "bits")]


class FtkError(RuntimeError):
    def __init__(self, code, text):
        super().__init__("ftkmeans error %d: %s" % (code, text))
        self.code = code


def load():
    """Load the shared library (built by ``__graft_entry__.build()``)."""
    global _lib
    if _lib is not None:
        return _lib
    if not _LIB_PATH.exists():
        raise FileNotFoundError(
            "%s not found: build it with `python __graft_entry__.py` (hipcc, gfx950)" % _LIB_PATH)
    L = ctypes.CDLL(str(_LIB_PATH))
    vp, i64, i32, u64, sz = (ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32, ctypes.c_uint64,
                             ctypes.c_size_t)
    L.ftk_workspace_bytes.argtypes = [i32, i64, i32, i32, i32]
    L.ftk_workspace_bytes.restype = sz
    L.ftk_assign_geometry.argtypes = [i32, i64, i32, i32, i32, ctypes.POINTER(Geometry)]
    L.ftk_assign_geometry.restype = i32
    L.ftk_ft_thresholds.argtypes = [i32, i64, i32, i32, i32, ctypes.POINTER(ctypes.c_double),
                                    ctypes.POINTER(ctypes.c_double)]
    L.ftk_ft_thresholds.restype = i32
    L.ftk_plan_padded_rows.argtypes = [i32, i64, i32, i32, ctypes.POINTER(i64), ctypes.POINTER(i64)]
    L.ftk_plan_padded_rows.restype = i32
    L.ftk_kmeans_assign.argtypes = [i32, vp, vp, i64, i32, i32, vp, vp, i32, vp, i32, vp, vp, sz, vp]
    L.ftk_kmeans_assign.restype = i32
    L.ftk_kmeans_assign_static.argtypes = [i32, vp, vp, i64, i32, i32, vp, vp, i32, vp, i32, vp, vp]
    L.ftk_kmeans_assign_static.restype = i32
    L.ftk_static_scratch_bytes.argtypes = []
    L.ftk_static_scratch_bytes.restype = sz
    L.ftk_kmeans_assign_fast.argtypes = [i32, vp, vp, i64, i32, i32, vp, vp, i32, vp, i32, vp, vp, sz, vp]
    L.ftk_kmeans_assign_fast.restype = i32
    L.ftk_fast_plan.argtypes = [i32, i64, i32, i32, i32, vp, vp, vp]
    L.ftk_fast_plan.restype = i32
    L.ftk_absmax.argtypes = [i32, vp, i64, vp, vp]
    L.ftk_absmax.restype = i32
    L.ftk_kmeans_update.argtypes = [i32, vp, vp, i64, i32, i32, vp, vp, vp, vp, sz, vp]
    L.ftk_kmeans_update.restype = i32
    L.ftk_kmeans_step_batched.argtypes = [i32, vp, i64, i32, i32, vp, vp, vp, vp, vp, i64, vp, sz, vp]
    L.ftk_kmeans_step_batched.restype = i32
    L.ftk_kmeans_update_ft.argtypes = [i32, vp, vp, i64, i32, i32, vp, vp, vp, i32, vp, i32, vp, vp, sz, vp]
    L.ftk_kmeans_update_ft.restype = i32
    L.ftk_update_geometry.argtypes = [i32, i64, i32, i32, i32, ctypes.POINTER(Geometry)]
    L.ftk_update_geometry.restype = i32
    L.ftk_kmeans_fit.argtypes = [i32, vp, i64, i32, i32, i32, u64, vp, vp, vp, vp, vp, i32, vp, vp, sz, vp]
    L.ftk_kmeans_fit.restype = i32
    L.ftk_kmeans_fit_fast.argtypes = [i32, vp, i64, i32, i32, i32, u64, vp, vp, vp, vp, vp, i32, vp, vp, sz, vp]
    L.ftk_kmeans_fit_fast.restype = i32
    L.ftk_seeded_indices.argtypes = [u64, i64, i32, vp]
    L.ftk_seeded_indices.restype = i32
    L.ftk_profile_enable.argtypes = [i32]
    L.ftk_profile_enable.restype = i32
    L.ftk_profile_read.argtypes = [ctypes.POINTER(ctypes.c_double), ctypes.POINTER(ctypes.c_int64)]
    L.ftk_profile_read.restype = i32
    L.ftk_tuning_override.argtypes = [i32, i32, i32]
    L.ftk_tuning_override.restype = i32
    L.ftk_route_rows.argtypes = [i64, i32, i32, i32]
    L.ftk_route_rows.restype = i64
    L.ftk_route_workspace_bytes.argtypes = [i64, i32, i32]
    L.ftk_route_workspace_bytes.restype = sz
    L.ftk_route_plan.argtypes = [vp, i64, i32, i32, i32, i64, vp, vp, vp, vp, vp, sz, vp]
    L.ftk_route_plan.restype = i32
    L.ftk_route_gather.argtypes = [i32, vp, i64, i64, i32, i32, vp, vp, i64, vp, vp, i64, vp]
    L.ftk_route_gather.restype = i32
    L.ftk_route_dispatch.argtypes = [i32, vp, i64, i32, vp, i64, i32, i32, i32, i64, vp, vp, vp, vp, vp, i64, vp, sz, vp]
    L.ftk_route_dispatch.restype = i32
    L.ftk_route_combine.argtypes = [i32, vp, i64, i64, vp, vp, i64, i32, i32, vp, i64, vp]
    L.ftk_route_combine.restype = i32
    L.ftk_route_combine_grad.argtypes = [i32, vp, i64, vp, i64, vp, vp, i64, vp, i64, i32, i32, vp, i64, vp, vp]
    L.ftk_route_combine_grad.restype = i32
    L.ftk_mx4_quantize.argtypes = [i32, vp, i64, i64, i32, i32, vp, vp, vp]
    L.ftk_mx4_quantize.restype = i32
    L.ftk_mx4_dequantize.argtypes = [i32, vp, vp, i64, i32, vp, i64, vp]
    L.ftk_mx4_dequantize.restype = i32
    L.ftk_mx4_matmul.argtypes = [i32, vp, vp, i64, vp, vp, i64, i32, i32, i32, vp, vp, i32, vp, i64, vp]
    L.ftk_mx4_matmul.restype = i32
    L.ftk_mx4_linear.argtypes = [i32, vp, i64, i64, vp, vp, i64, i32, i32, i32, vp, vp, i32, vp, i64, vp, sz, vp]
    L.ftk_mx4_linear.restype = i32
    L.ftk_mx4_workspace_bytes.argtypes = [i64, i32, i64, i32]
    L.ftk_mx4_workspace_bytes.restype = i64
    L.ftk_mx4_outer.argtypes = [i32, vp, vp, vp, vp, i64, i32, i32, i32, vp, vp, vp]
    L.ftk_mx4_outer.restype = i32
    L.ftk_route_gate_workspace_bytes.argtypes = [i64, i32]
    L.ftk_route_gate_workspace_bytes.restype = sz
    L.ftk_route_gate.argtypes = [i32, vp, i64, i64, i32, i32, i32, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    L.ftk_route_gate.restype = i32
    L.ftk_route_gate_grad.argtypes = [i32, vp, i64, i64, i32, i32, i32, vp, vp, vp, vp, vp, vp, vp, i64, vp]
    L.ftk_route_gate_grad.restype = i32
    L.ftk_xent_workspace_bytes.argtypes = [i32, i64, i64, i32, i32]
    L.ftk_xent_workspace_bytes.restype = i64
    L.ftk_xent.argtypes = [i32, vp, i64, i64, vp, i64, i64, i32, vp, ctypes.c_double, vp, vp, vp, vp, sz, vp]
    L.ftk_xent.restype = i32
    L.ftk_xent_grad.argtypes = [i32, vp, i64, i64, vp, i64, i64, i32, vp, ctypes.c_double, vp, vp, vp, vp, i64, vp, i64, vp, vp, sz, vp]
    L.ftk_xent_grad.restype = i32
    L.ftk_adamw_step.argtypes = [i32, i32, i32, vp, i32, vp, vp]
    L.ftk_adamw_step.restype = i32
    L.ftk_adamw_moments.argtypes = [i32, vp, i32, vp, vp, vp]
    L.ftk_adamw_moments.restype = i32
    L.ftk_last_error.restype = ctypes.c_char_p
    L.ftk_version.restype = ctypes.c_char_p
    _lib = L
    return L


EXPORTS = ("ftk_workspace_bytes", "ftk_assign_geometry", "ftk_plan_padded_rows", "ftk_ft_thresholds", "ftk_kmeans_assign_static", "ftk_static_scratch_bytes", "ftk_kmeans_assign", "ftk_kmeans_assign_fast", "ftk_fast_plan", "ftk_absmax",
           "ftk_kmeans_update", "ftk_kmeans_update_ft", "ftk_kmeans_step_batched", "ftk_update_geometry", "ftk_kmeans_fit", "ftk_kmeans_fit_fast", "ftk_seeded_indices", "ftk_profile_enable",
           "ftk_route_rows", "ftk_route_workspace_bytes", "ftk_route_plan", "ftk_route_gather", "ftk_route_dispatch",
           "ftk_route_combine", "ftk_route_combine_grad", "ftk_mx4_quantize", "ftk_mx4_dequantize", "ftk_mx4_matmul",
           "ftk_mx4_linear", "ftk_mx4_workspace_bytes", "ftk_mx4_outer",
           "ftk_route_gate_workspace_bytes", "ftk_route_gate", "ftk_route_gate_grad", "ftk_xent_workspace_bytes", "ftk_xent",
           "ftk_xent_grad", "ftk_adamw_step", "ftk_adamw_moments",
           "ftk_profile_read", "ftk_tuning_override", "ftk_last_error", "ftk_version")


def _check(rc):
    if rc != 0:
        raise FtkError(rc, load().ftk_last_error().decode())


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return F32
    if t.dtype == torch.float64:
        return F64
    raise TypeError("float32 or float64 tensor expected, got %s" % t.dtype)


def _dev2d(t: torch.Tensor, name: str) -> torch.Tensor:
    if not t.is_cuda:
        raise ValueError("%s must live on the GPU" % name)
    if t.dim() != 2 or not t.is_contiguous():
        raise ValueError("%s must be a contiguous 2-D tensor" % name)
    return t


def _stream() -> int:
    # the current stream's handle, without the Stream object that torch.cuda.current_stream() makes (3 of 12 us of a small call)
    return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())


def _ptr(t):
    return None if t is None else t.data_ptr()


def ft_thresholds(dtype_code: int, N: int, D: int, K: int, ft_mode: int = FT_CORRECT):
    """(detect_coef, band_coef): detection threshold and exact-settlement band of point i are these
    times ||x_i|| max||c|| + max||c||^2/2, in score units (half a squared distance)."""
    a, b = ctypes.c_double(0.0), ctypes.c_double(0.0)
    _check(load().ftk_ft_thresholds(dtype_code, N, D, K, ft_mode, ctypes.byref(a), ctypes.byref(b)))
    return a.value, b.value


def plan_padded_rows(dtype_code: int, N: int, D: int, K: int):
    """(largest padded centroid-row count over all kernel variants, rows the workspace reserves)"""
    a, b = ctypes.c_int64(0), ctypes.c_int64(0)
    _check(load().ftk_plan_padded_rows(dtype_code, N, D, K, ctypes.byref(a), ctypes.byref(b)))
    return a.value, b.value


def workspace_bytes(dtype_code: int, N: int, D: int, K: int, ft_mode: int = FT_OFF) -> int:
    n = load().ftk_workspace_bytes(dtype_code, N, D, K, ft_mode)
    if n == 0:
        raise FtkError(1, load().ftk_last_error().decode())
    return n


def _mode_workspace(X: torch.Tensor, K: int, *modes: int) -> torch.Tensor:
    n = max(workspace_bytes(_dtype_code(X), X.shape[0], X.shape[1], K, m) for m in modes)
    return torch.empty(n + 256, dtype=torch.uint8, device=X.device)


def new_workspace(X: torch.Tensor, K: int, ft_mode: int = FT_CORRECT) -> torch.Tensor:
    """A workspace for calls of ``ft_mode`` and, at their full speed, for unprotected ones beside them (a
    protected mode alone needs no more than ``workspace_bytes`` reports for it)."""
    return _mode_workspace(X, K, ft_mode, FT_OFF)


def _ws_args(ws: torch.Tensor):
    """(first aligned address, bytes from there on) of a workspace, a contiguous device tensor of any type."""
    if not ws.is_cuda:
        raise ValueError("workspace must live on the GPU")
    if not ws.is_contiguous():
        raise ValueError("workspace must be contiguous")
    base = ws.data_ptr()
    aligned = (base + 255) // 256 * 256
    return aligned, max(0, ws.numel() * ws.element_size() - (aligned - base))


def assign_geometry(dtype_code: int, N: int, D: int, K: int, ft_mode: int = FT_OFF) -> Geometry:
    g = Geometry()
    _check(load().ftk_assign_geometry(dtype_code, N, D, K, ft_mode, ctypes.byref(g)))
    return g


def new_stats(device) -> torch.Tensor:
    return torch.zeros(len(STAT_FIELDS), dtype=torch.int64, device=device)


def stats_dict(stats: torch.Tensor) -> dict:
    return dict(zip(STAT_FIELDS, (int(v) for v in stats.cpu().tolist())))


def make_faults(rows, device) -> torch.Tensor:
    """rows: iterable of (workgroup, wave, tile, reg, lane, bit) -> device tensor [n, 6] uint32-as-int32."""
    t = torch.tensor(list(rows), dtype=torch.int64).reshape(-1, 6)
    return t.to(torch.int32).contiguous().to(device)


def kmeans_assign(X, C, labels=None, mindist=None, ft_mode=FT_OFF, faults=None, stats=None,
                  workspace=None, want_mindist=True):
    """Assignment step (Eq. 1).  Returns (labels int32 [N], mindist [N] or None)."""
    _dev2d(X, "X"), _dev2d(C, "C")
    if X.dtype != C.dtype or X.shape[1] != C.shape[1]:
        raise ValueError("X [N,D] and C [K,D] must share dtype and D")
    N, D = X.shape
    K = C.shape[0]
    if labels is None:
        labels = torch.empty(N, dtype=torch.int32, device=X.device)
    if mindist is None and want_mindist:
        mindist = torch.empty(N, dtype=X.dtype, device=X.device)
    if workspace is None:
        workspace = _mode_workspace(X, K, ft_mode)
    wp, wn = _ws_args(workspace)
    nf = 0 if faults is None else faults.shape[0]
    _check(load().ftk_kmeans_assign(_dtype_code(X), X.data_ptr(), C.data_ptr(), N, D, K,
                                    labels.data_ptr(), _ptr(mindist), ft_mode, _ptr(faults), nf,
                                    _ptr(stats), wp, wn, _stream()))
    return labels, mindist


def static_scratch_bytes() -> int:
    return load().ftk_static_scratch_bytes()


def kmeans_assign_static(X, C, labels, mindist=None, ft_mode=FT_OFF, faults=None, stats=None):
    """Assignment step through the entry point that allocates nothing: outputs are the caller's
    tensors, scratch is the library's static device array.  Returns (labels, mindist)."""
    _dev2d(X, "X"), _dev2d(C, "C")
    if X.dtype != C.dtype or X.shape[1] != C.shape[1]:
        raise ValueError("X [N,D] and C [K,D] must share dtype and D")
    N, D = X.shape
    K = C.shape[0]
    nf = 0 if faults is None else faults.shape[0]
    _check(load().ftk_kmeans_assign_static(_dtype_code(X), X.data_ptr(), C.data_ptr(), N, D, K,
                                           labels.data_ptr(), _ptr(mindist), ft_mode, _ptr(faults), nf,
                                           _ptr(stats), _stream()))
    return labels, mindist


def fast_plan(dtype_code: int, N: int, D: int, K: int, ft_mode: int = FT_OFF):
    """(geometry, detect_coef, band_coef) of the split-bf16 path: what assign_geometry and
    ft_thresholds report for the fp32 path."""
    g = Geometry()
    a, b = ctypes.c_double(0.0), ctypes.c_double(0.0)
    _check(load().ftk_fast_plan(dtype_code, N, D, K, ft_mode, ctypes.byref(g), ctypes.byref(a), ctypes.byref(b)))
    return g, a.value, b.value


def kmeans_assign_fast(X, C, labels=None, mindist=None, workspace=None, want_mindist=True, ft_mode=FT_OFF,
                       faults=None, stats=None):
    """Assignment step on the split-bf16 matrix path (fp32 data, D <= 128).  Returns (labels, mindist)."""
    _dev2d(X, "X"), _dev2d(C, "C")
    if X.dtype != C.dtype or X.shape[1] != C.shape[1]:
        raise ValueError("X [N,D] and C [K,D] must share dtype and D")
    N, D = X.shape
    K = C.shape[0]
    if labels is None:
        labels = torch.empty(N, dtype=torch.int32, device=X.device)
    if mindist is None and want_mindist:
        mindist = torch.empty(N, dtype=X.dtype, device=X.device)
    if workspace is None:
        workspace = _mode_workspace(X, K, ft_mode)
    wp, wn = _ws_args(workspace)
    nf = 0 if faults is None else faults.shape[0]
    _check(load().ftk_kmeans_assign_fast(_dtype_code(X), X.data_ptr(), C.data_ptr(), N, D, K,
                                         labels.data_ptr(), _ptr(mindist), ft_mode, _ptr(faults), nf,
                                         _ptr(stats), wp, wn, _stream()))
    return labels, mindist


def tuning_override(assign_variant: int = -1, generic_tiles: int = -1, update_path: int = -1):
    """Force kernel choices for later calls (-1 = built-in rule); for the shape-sweep tool and tests."""
    _check(load().ftk_tuning_override(assign_variant, generic_tiles, update_path))


def absmax(X: torch.Tensor) -> torch.Tensor:
    out = torch.empty(1, dtype=torch.float64, device=X.device)
    _check(load().ftk_absmax(_dtype_code(X), X.data_ptr(), X.numel(), out.data_ptr(), _stream()))
    return out


def update_geometry(dtype_code: int, N: int, D: int, K: int, rows_aligned16: bool = True) -> Geometry:
    g = Geometry()
    _check(load().ftk_update_geometry(dtype_code, N, D, K, 1 if rows_aligned16 else 0, ctypes.byref(g)))
    return g


def kmeans_update(X, labels, C, counts=None, x_absmax=None, workspace=None, ft_mode=FT_OFF, faults=None,
                  stats=None):
    """Update step (Eq. 2), in place on C; with ft_mode on, under dual modular redundancy.
    Returns (C, counts int32 [K])."""
    _dev2d(X, "X"), _dev2d(C, "C")
    N, D = X.shape
    K = C.shape[0]
    if labels.dtype != torch.int32 or labels.shape != (N,) or not labels.is_contiguous():
        raise ValueError("labels must be a contiguous int32 vector of length N")
    if counts is None:
        counts = torch.empty(K, dtype=torch.int32, device=X.device)
    if workspace is None:
        workspace = new_workspace(X, K, FT_OFF)
    wp, wn = _ws_args(workspace)
    if ft_mode == FT_OFF and faults is None and stats is None:
        _check(load().ftk_kmeans_update(_dtype_code(X), X.data_ptr(), labels.data_ptr(), N, D, K,
                                        C.data_ptr(), counts.data_ptr(), _ptr(x_absmax), wp, wn, _stream()))
    else:
        nf = 0 if faults is None else int(faults.shape[0])
        _check(load().ftk_kmeans_update_ft(_dtype_code(X), X.data_ptr(), labels.data_ptr(), N, D, K,
                                           C.data_ptr(), counts.data_ptr(), _ptr(x_absmax), ft_mode,
                                           _ptr(faults), nf, _ptr(stats), wp, wn, _stream()))
    return C, counts


def kmeans_step_batched(X, C, batch_rows, labels=None, mindist=None, counts=None, x_absmax=None, workspace=None):
    """One Lloyd iteration in batches of `batch_rows` points (assign a batch, add it to the sums while
    it is cache-resident); C is updated in place.  Returns (labels, mindist, counts)."""
    _dev2d(X, "X"), _dev2d(C, "C")
    N, D = X.shape
    K = C.shape[0]
    if labels is None:
        labels = torch.empty(N, dtype=torch.int32, device=X.device)
    if mindist is None:
        mindist = torch.empty(N, dtype=X.dtype, device=X.device)
    if counts is None:
        counts = torch.empty(K, dtype=torch.int32, device=X.device)
    if x_absmax is None:
        x_absmax = absmax(X)
    if workspace is None:
        workspace = new_workspace(X, K, FT_OFF)
    wp, wn = _ws_args(workspace)
    _check(load().ftk_kmeans_step_batched(_dtype_code(X), X.data_ptr(), N, D, K, C.data_ptr(), labels.data_ptr(),
                                          _ptr(mindist), counts.data_ptr(), x_absmax.data_ptr(), int(batch_rows),
                                          wp, wn, _stream()))
    return labels, mindist, counts


def seeded_indices(seed: int, N: int, K: int):
    import numpy as np
    idx = np.empty(K, dtype=np.int64)
    _check(load().ftk_seeded_indices(seed & (2**64 - 1), N, K, idx.ctypes.data))
    return idx


def profile_enable(on: bool) -> None:
    _check(load().ftk_profile_enable(1 if on else 0))


def profile_read():
    """(total milliseconds, launches) of the main assignment kernel since the last read."""
    ms, n = ctypes.c_double(0.0), ctypes.c_int64(0)
    _check(load().ftk_profile_read(ctypes.byref(ms), ctypes.byref(n)))
    return ms.value, n.value


def kmeans_fit(X, K, iters, seed=0, C_init=None, ft_mode=FT_OFF, stats=None, workspace=None,
               want_inertia=True, fast=False):
    """Lloyd loop.  Returns dict(C, labels, counts, inertia (numpy, host) or None).
    fast=True runs the assignment on the split-bf16 matrix path (fp32, D <= 128)."""
    import numpy as np
    _dev2d(X, "X")
    N, D = X.shape
    if C_init is not None:
        _dev2d(C_init, "C_init")
        if C_init.shape != (K, D) or C_init.dtype != X.dtype:
            raise ValueError("C_init must be [K,D] of X's dtype")
    C = torch.empty(K, D, dtype=X.dtype, device=X.device)
    labels = torch.empty(N, dtype=torch.int32, device=X.device)
    counts = torch.empty(K, dtype=torch.int32, device=X.device)
    inertia = np.zeros(iters, dtype=np.float64) if want_inertia else None
    if workspace is None:
        workspace = _mode_workspace(X, K, ft_mode)
    wp, wn = _ws_args(workspace)
    if fast:
        _check(load().ftk_kmeans_fit_fast(_dtype_code(X), X.data_ptr(), N, D, K, iters, seed & (2**64 - 1),
                                          _ptr(C_init), C.data_ptr(), labels.data_ptr(), counts.data_ptr(),
                                          None if inertia is None else inertia.ctypes.data, ft_mode,
                                          _ptr(stats), wp, wn, _stream()))
        return dict(C=C, labels=labels, counts=counts, inertia=inertia)
    _check(load().ftk_kmeans_fit(_dtype_code(X), X.data_ptr(), N, D, K, iters, seed & (2**64 - 1),
                                 _ptr(C_init), C.data_ptr(), labels.data_ptr(), counts.data_ptr(),
                                 None if inertia is None else inertia.ctypes.data, ft_mode,
                                 _ptr(stats), wp, wn, _stream()))
    return dict(C=C, labels=labels, counts=counts, inertia=inertia)


# ---- rows sorted by label and back -----------------------------------------------------------

_ROW_DTYPES = {torch.float32: F32, torch.float64: F64, torch.bfloat16: BF16, torch.float16: F16}
ROUTE_FEW = 1024  # slots that are sorted without a workspace
_MX_DTYPES = {torch.float32: F32, torch.bfloat16: BF16, torch.float16: F16}


def _row_code(t: torch.Tensor, name: str, dtypes=_ROW_DTYPES) -> int:
    code = dtypes.get(t.dtype)
    if code is None:
        raise TypeError("%s: %s is not one of %s" % (name, t.dtype, ", ".join(str(d)[6:] for d in dtypes)))
    return code


def _row_stride(t: torch.Tensor, name: str) -> int:
    """Row stride of a 2-D device tensor whose rows are contiguous."""
    if not t.is_cuda:
        raise ValueError("%s must live on the GPU" % name)
    strides = t.stride()
    if len(strides) == 2:
        rows, D = t.shape
        ld, unit = strides
        if rows <= 1:
            ld = D
        if unit == 1 or D <= 1 or rows == 0:
            if ld < D:
                raise ValueError("%s: its rows overlap" % name)
            return ld
    raise ValueError("%s must be a 2-D tensor of contiguous rows" % name)


def _workspace(workspace, need, device):
    """(workspace, address, bytes): the caller's workspace, or a new one where any is needed, to be held until the call is enqueued."""
    if workspace is None:
        if not need:
            return None, None, 0
        workspace = torch.empty(need + 256, dtype=torch.uint8, device=device)
    return workspace, *_ws_args(workspace)


def _index(t: torch.Tensor, name: str, *shape) -> torch.Tensor:
    if not t.is_cuda or t.dtype != torch.int32 or tuple(t.shape) != shape or not t.is_contiguous():
        raise ValueError("%s must be a contiguous int32 device tensor of shape %s" % (name, list(shape)))
    return t


def _new_rows(out, rows, D, like, name, dtype=None):
    """(out, its row stride): the caller's, or a new one."""
    dtype = like.dtype if dtype is None else dtype
    if out is None:
        return torch.empty((rows, D), dtype=dtype, device=like.device), D
    if out.shape != (rows, D) or out.dtype != dtype:
        raise ValueError("%s must be [%d, %d] of %s" % (name, rows, D, dtype))
    return out, _row_stride(out, name)


class Route:
    """Where every slot's row goes (device tensors, int32): offsets [E + 1], counts [E], order [rows], pos [N, k]."""

    __slots__ = ("offsets", "counts", "order", "pos", "align")

    def __init__(self, offsets, counts, order, pos, align=1):
        self.offsets, self.counts, self.order, self.pos, self.align = offsets, counts, order, pos, align

    @property
    def experts(self):
        return self.offsets.shape[0] - 1

    @property
    def rows(self):
        return self.order.shape[0]

    def check(self):
        N, k = self.pos.shape
        _index(self.offsets, "offsets", self.experts + 1), _index(self.order, "order", self.rows)
        _index(self.pos, "pos", N, k)
        return N, k


def route_rows(N: int, k: int, E: int, align: int = 1) -> int:
    """Sorted rows that N tokens of k slots may need."""
    n = load().ftk_route_rows(N, k, E, align)
    if n < 0:
        raise FtkError(1, load().ftk_last_error().decode())
    return n


def route_workspace_bytes(N: int, k: int, E: int) -> int:
    n = load().ftk_route_workspace_bytes(N, k, E)
    if n == 0:
        raise FtkError(1, load().ftk_last_error().decode())
    return n


def _route_args(labels, E, align, route, workspace):
    if labels.dim() == 1:
        labels = labels.unsqueeze(1)
    if labels.dim() != 2:
        raise ValueError("labels must be [N] or [N, k]")
    N, k = labels.shape
    _index(labels, "labels", N, k)
    if route is None:
        rows, dev = route_rows(N, k, E, align), labels.device
        whole = torch.empty(2 * E + 1 + rows + N * k, dtype=torch.int32, device=dev)
        offsets, counts, order, pos = whole.split_with_sizes((E + 1, E, rows, N * k))
        route = Route(offsets, counts, order, pos.view(N, k), align)
    else:
        if route.check() != (N, k) or route.experts != E or route.align != align:
            raise ValueError("route is not one of %d x %d slots, %d experts and align %d" % (N, k, E, align))
        _index(route.counts, "counts", E)
    need = route_workspace_bytes(N, k, E) if N * k > ROUTE_FEW else 0
    return labels, N, k, route, *_workspace(workspace, need, labels.device)


def route_plan(labels, E, align=1, route=None, workspace=None):
    """Sorts the slots of labels (int32 [N] or [N, k]; outside [0, E): dropped) by expert.  Returns a Route."""
    labels, N, k, route, workspace, wp, wn = _route_args(labels, E, align, route, workspace)
    _check(load().ftk_route_plan(labels.data_ptr(), N, k, E, align, route.rows, route.offsets.data_ptr(),
                                 route.counts.data_ptr(), route.order.data_ptr(), route.pos.data_ptr(), wp, wn, _stream()))
    return route


def route_dispatch(X, labels, E, align=1, out=None, route=None, workspace=None):
    """route_plan and route_gather in one call.  Returns (sorted rows [rows, D], Route)."""
    labels, N, k, route, workspace, wp, wn = _route_args(labels, E, align, route, workspace)
    ld = _row_stride(X, "X")
    if X.shape[0] != N:
        raise ValueError("X must have a row for each of the %d tokens" % N)
    out, ldo = _new_rows(out, route.rows, X.shape[1], X, "out")
    _check(load().ftk_route_dispatch(_row_code(X, "X"), X.data_ptr(), ld, X.shape[1], labels.data_ptr(), N, k, E, align,
                                     route.rows, route.offsets.data_ptr(), route.counts.data_ptr(),
                                     route.order.data_ptr(), route.pos.data_ptr(), out.data_ptr(),
                                     ldo, wp, wn, _stream()))
    return out, route


def _weights(weights, like, N, k):
    dtype = torch.float64 if like.dtype == torch.float64 else torch.float32
    if weights is not None and (not weights.is_cuda or weights.dtype != dtype or tuple(weights.shape) != (N, k)
                                or not weights.is_contiguous()):
        raise ValueError("weights must be a contiguous device tensor [%d, %d] of %s" % (N, k, dtype))
    return weights


def route_gather(X, route, weights=None, out=None):
    """Tokens' rows X [N, D], times weights [N, k] if given, to their sorted places [rows, D]; rows without a slot are zero."""
    N, k = route.check()
    ld = _row_stride(X, "X")
    if X.shape[0] != N:
        raise ValueError("X must have a row for each of the %d tokens" % N)
    out, ldo = _new_rows(out, route.rows, X.shape[1], X, "out")
    _check(load().ftk_route_gather(_row_code(X, "X"), X.data_ptr(), ld, N, k, X.shape[1], route.order.data_ptr(),
                                   route.pos.data_ptr(), route.rows, _ptr(_weights(weights, X, N, k)), out.data_ptr(),
                                   ldo, _stream()))
    return out


def route_combine(Y, route, weights=None, out=None):
    """Sorted rows Y [rows, D] back to their tokens [N, D]: the sum over a token's slots, times weights [N, k] if given."""
    N, k = route.check()
    ld = _row_stride(Y, "Y")
    if Y.shape[0] != route.rows:
        raise ValueError("Y must have the %d sorted rows" % route.rows)
    out, ldo = _new_rows(out, N, Y.shape[1], Y, "out")
    _check(load().ftk_route_combine(_row_code(Y, "Y"), Y.data_ptr(), ld, route.rows, route.pos.data_ptr(),
                                    _ptr(_weights(weights, Y, N, k)), N, k, Y.shape[1], out.data_ptr(),
                                    ldo, _stream()))
    return out


def route_combine_grad(dOut, Y, route, weights, dY=None, dweights=None):
    """Gradients of route_combine(Y, route, weights) for dOut [N, D].  Returns (dY [rows, D], dweights [N, k]).
    (The gradient of route_gather without weights is route_combine without weights.)"""
    N, k = route.check()
    D = dOut.shape[1]
    ldg, ldy = _row_stride(dOut, "dOut"), _row_stride(Y, "Y")
    if dOut.shape[0] != N or tuple(Y.shape) != (route.rows, D) or Y.dtype != dOut.dtype:
        raise ValueError("dOut [N, D] and Y [rows, D] must share type and D")
    _weights(weights, Y, N, k)
    dY, ldo = _new_rows(dY, route.rows, D, Y, "dY")
    dweights = torch.empty_like(weights) if dweights is None else _weights(dweights, Y, N, k)
    _check(load().ftk_route_combine_grad(_row_code(Y, "Y"), dOut.data_ptr(), ldg, Y.data_ptr(), ldy,
                                         route.order.data_ptr(), route.pos.data_ptr(), route.rows, weights.data_ptr(),
                                         N, k, D, dY.data_ptr(), ldo, dweights.data_ptr(), _stream()))
    return dY, dweights


# ---- rows in microscaled 4-bit floating point ------------------------------------------------


class Mx4:
    """Packed rows (device tensors, uint8): codes [N, Dp / 2], scales [N, Dp / 32]; D elements a row, Dp = D rounded up
    to 128."""

    __slots__ = ("codes", "scales", "D")

    def __init__(self, codes, scales, D):
        self.codes, self.scales, self.D = codes, scales, D

    @property
    def N(self):
        return self.codes.shape[0]

    def check(self, name):
        Dp = -(-self.D // 128) * 128
        for t, width, part in ((self.codes, Dp // 2, "codes"), (self.scales, Dp // 32, "scales")):
            if (not t.is_cuda or t.dtype != torch.uint8 or tuple(t.shape) != (self.codes.shape[0], width)
                    or not t.is_contiguous()):
                raise ValueError("%s.%s must be a contiguous uint8 device tensor [N, %d]" % (name, part, width))
        return self


def mx4_quantize(X, transpose=False, out=None):
    """Packs the rows of X [N, D] (transpose: its columns, as rows of N elements).  Returns an Mx4."""
    ld = _row_stride(X, "X")
    N, D = X.shape
    n, d = (D, N) if transpose else (N, D)
    if out is None:
        Dp = -(-d // 128) * 128
        out = Mx4(torch.empty(n, Dp // 2, dtype=torch.uint8, device=X.device),
                  torch.empty(n, Dp // 32, dtype=torch.uint8, device=X.device), d)
    elif out.N != n or out.D != d:
        raise ValueError("out must hold %d rows of %d elements" % (n, d))
    else:
        out.check("out")
    _check(load().ftk_mx4_quantize(_row_code(X, "X", _MX_DTYPES), X.data_ptr(), ld, N, D, 1 if transpose else 0,
                                   out.codes.data_ptr(), out.scales.data_ptr(), _stream()))
    return out


def mx4_dequantize(q, dtype=torch.float32, out=None):
    """The values of packed rows, [N, D]."""
    q.check("q")
    out, ldo = _new_rows(out, q.N, q.D, q.codes, "out", dtype)
    if q.D == 0:
        return out
    _check(load().ftk_mx4_dequantize(_row_code(out, "out", _MX_DTYPES), q.codes.data_ptr(), q.scales.data_ptr(), q.N, q.D,
                                     out.data_ptr(), ldo, _stream()))
    return out


def _groups(B, route, gather, sources):
    """(E, F, M, offsets, order, k) of a product."""
    B.check("B")
    if route is None:
        return 1, B.N, sources, None, None, 1
    N, k = route.check()
    E = route.experts
    if B.N % E:
        raise ValueError("%d rows of B are not %d matrices of equal height" % (B.N, E))
    if sources != (N if gather else route.rows):
        raise ValueError("%d rows given, the route has %d %s" % (sources, N if gather else route.rows,
                                                                 "tokens" if gather else "sorted rows"))
    return E, B.N // E, route.rows, route.offsets, route.order if gather else None, k


def mx4_matmul(A, B, route=None, gather=False, out=None, out_dtype=torch.bfloat16):
    """Products of packed rows: [A.N, B.N] without a route.  With one, B holds the experts' matrices one after the other and a
    sorted row meets its expert's: A holds sorted rows, or with gather=True the tokens' rows; [rows, F]."""
    A.check("A")
    if A.D != B.D:
        raise ValueError("A and B must share D (got %d and %d)" % (A.D, B.D))
    E, F, M, offsets, order, k = _groups(B, route, gather, A.N)
    out, ldo = _new_rows(out, M, F, A.codes, "out", out_dtype if out is None else out.dtype)
    _check(load().ftk_mx4_matmul(_row_code(out, "out", _MX_DTYPES), A.codes.data_ptr(), A.scales.data_ptr(), A.N,
                                 B.codes.data_ptr(), B.scales.data_ptr(), M, F, A.D, E, _ptr(offsets), _ptr(order), k,
                                 out.data_ptr(), ldo, _stream()))
    return out


def mx4_workspace_bytes(N: int, D: int, M: int, E: int = 1) -> int:
    n = load().ftk_mx4_workspace_bytes(N, D, M, E)
    if n < 0:
        raise FtkError(1, load().ftk_last_error().decode())
    return n


def mx4_linear(X, B, route=None, gather=False, out=None, workspace=None):
    """mx4_matmul of dense rows X, packed on the way; the result has their type."""
    ld = _row_stride(X, "X")
    N, D = X.shape
    if D != B.D:
        raise ValueError("X and B must share D (got %d and %d)" % (D, B.D))
    E, F, M, offsets, order, k = _groups(B, route, gather, N)
    out, ldo = _new_rows(out, M, F, X, "out")
    workspace, wp, wn = _workspace(workspace, mx4_workspace_bytes(N, D, M, E), X.device)
    _check(load().ftk_mx4_linear(_row_code(X, "X", _MX_DTYPES), X.data_ptr(), ld, N, B.codes.data_ptr(),
                                 B.scales.data_ptr(), M, F, D, E, _ptr(offsets), _ptr(order), k, out.data_ptr(),
                                 ldo, wp, wn, _stream()))
    return out


def mx4_outer(A, B, route=None, out=None, out_dtype=torch.float32):
    """Sums over the rows of every expert, [E, F, D]: A holds F and B holds D packed rows across all sorted rows
    (mx4_quantize(..., transpose=True)); the route's align must be a multiple of 128."""
    A.check("A"), B.check("B")
    if A.D != B.D:
        raise ValueError("A and B must have equally many elements a row (got %d and %d)" % (A.D, B.D))
    E = 1
    if route is not None:
        route.check()
        E = route.experts
        if route.align % 128 or A.D != route.rows:
            raise ValueError("mx4_outer takes all sorted rows, and a route whose align is a multiple of 128")
    if out is None:
        out = torch.empty(E, A.N, B.N, dtype=out_dtype, device=A.codes.device)
    elif not out.is_cuda:
        raise ValueError("out must live on the GPU")
    elif tuple(out.shape) != (E, A.N, B.N) or not out.is_contiguous():
        raise ValueError("out must be a contiguous tensor [%d, %d, %d]" % (E, A.N, B.N))
    _check(load().ftk_mx4_outer(_row_code(out, "out", _MX_DTYPES), A.codes.data_ptr(), A.scales.data_ptr(),
                                B.codes.data_ptr(), B.scales.data_ptr(), A.D, A.N, B.N, E,
                                None if route is None else route.offsets.data_ptr(), out.data_ptr(), _stream()))
    return out


# ---- a gate that learns ----------------------------------------------------------------------

GATE_FEW = 16384  # logits that need no workspace (FTK_ROUTE_GATE_FEW)


class Gate:
    """What a gate decided (device tensors): labels int32 and weights float [N, k], lse float [N]; counts int32 [E + 1] (slots of every
    expert, then the rows that took part), probs float [E], loss float [1]."""

    __slots__ = ("labels", "weights", "lse", "counts", "probs", "loss", "normalise")

    def __init__(self, labels, weights, lse, counts, probs, loss, normalise):
        self.labels, self.weights, self.lse = labels, weights, lse
        self.counts, self.probs, self.loss, self.normalise = counts, probs, loss, normalise


def _here(*tensors):
    """All on the current device: calls are enqueued on its current stream."""
    device = torch.cuda.current_device()
    for t in tensors:
        if t is not None and t.get_device() != device:
            raise ValueError("a tensor lives on device %d, the current one is %d" % (t.get_device(), device))


def _floats(t, name, *shape):
    if not t.is_cuda or t.dtype != torch.float32 or tuple(t.shape) != shape or not t.is_contiguous():
        raise ValueError("%s must be a contiguous float32 device tensor of shape %s" % (name, list(shape)))
    return t


def route_gate_workspace_bytes(N: int, E: int) -> int:
    n = load().ftk_route_gate_workspace_bytes(N, E)
    if n == 0:
        raise FtkError(1, load().ftk_last_error().decode())
    return n


def route_gate(logits, k, normalise=True, gate=None, workspace=None):
    """The k experts of every row of logits [N, E], their weights (probabilities; normalise: over the k alone), and how evenly the
    rows use the experts.  Returns a Gate, whose labels route_plan and route_dispatch take."""
    ld = _row_stride(logits, "logits")
    N, E = logits.shape
    code, dev = _row_code(logits, "logits", _MX_DTYPES), logits.device
    if gate is None:
        if not 1 <= k <= E:
            raise ValueError("need 1 <= k <= %d experts, got %d" % (E, k))
        ints = torch.empty(N * k + E + 1, dtype=torch.int32, device=dev)
        labels, counts = ints.split_with_sizes((N * k, E + 1))
        floats = torch.empty(N * k + N + E + 1, dtype=torch.float32, device=dev)
        weights, lse, probs, loss = floats.split_with_sizes((N * k, N, E, 1))
        gate = Gate(labels.view(N, k), weights.view(N, k), lse, counts, probs, loss, normalise)
    else:
        _index(gate.labels, "labels", N, k), _floats(gate.weights, "weights", N, k), _floats(gate.lse, "lse", N)
        _index(gate.counts, "counts", E + 1), _floats(gate.probs, "probs", E), _floats(gate.loss, "loss", 1)
        _here(gate.labels, gate.weights, gate.lse, gate.counts, gate.probs, gate.loss)
        gate.normalise = normalise
    _here(logits, workspace)
    workspace, wp, wn = _workspace(workspace, route_gate_workspace_bytes(N, E) if N * E > GATE_FEW else 0, dev)
    _check(load().ftk_route_gate(code, logits.data_ptr(), ld, N, E, k, 1 if normalise else 0, gate.labels.data_ptr(),
                                 gate.weights.data_ptr(), gate.lse.data_ptr(), gate.counts.data_ptr(), gate.probs.data_ptr(),
                                 gate.loss.data_ptr(), wp, wn, _stream()))
    return gate


def route_gate_grad(logits, gate, dweights=None, dloss=None, out=None):
    """Gradient [N, E] of sum(dweights * gate.weights) + dloss * gate.loss; dweights float [N, k], dloss float [1], either may be None.
    Labels and counts are held fixed.  out may be logits."""
    ld = _row_stride(logits, "logits")
    N, E = logits.shape
    k = gate.labels.shape[1]
    _index(gate.labels, "labels", N, k), _floats(gate.weights, "weights", N, k), _floats(gate.lse, "lse", N)
    _index(gate.counts, "counts", E + 1)
    if dweights is not None:
        _floats(dweights, "dweights", N, k)
    if dloss is not None:
        _floats(dloss, "dloss", 1)
    out, ldo = _new_rows(out, N, E, logits, "out")
    _here(logits, gate.labels, gate.weights, gate.lse, gate.counts, dweights, dloss, out)
    _check(load().ftk_route_gate_grad(_row_code(logits, "logits", _MX_DTYPES), logits.data_ptr(), ld, N, E, k,
                                      1 if gate.normalise else 0, gate.labels.data_ptr(), gate.weights.data_ptr(),
                                      gate.lse.data_ptr(), gate.counts.data_ptr(), _ptr(dweights), _ptr(dloss), out.data_ptr(), ldo,
                                      _stream()))
    return out


# ---- softmax cross entropy over many classes -------------------------------------------------


def xent_workspace_bytes(dtype_code: int, N: int, V: int, D: int, grad: bool) -> int:
    n = load().ftk_xent_workspace_bytes(dtype_code, N, V, D, 1 if grad else 0)
    if n < 0:
        raise FtkError(1, load().ftk_last_error().decode())
    return n


def _xent_args(X, W, labels, bias):
    ldx, ldw = _row_stride(X, "X"), _row_stride(W, "W")
    N, D = X.shape
    V = W.shape[0]
    if W.shape[1] != D or W.dtype != X.dtype:
        raise ValueError("X [N, D] and W [V, D] must share type and D")
    _index(labels, "labels", N)
    if bias is not None:
        _floats(bias, "bias", V)
    _here(X, W, labels, bias)
    return _row_code(X, "X", _MX_DTYPES), ldx, ldw, N, V, D


def xent(X, W, labels, bias=None, scale=1.0, loss=None, lse=None, workspace=None):
    """Softmax cross entropy of rows X [N, D] against the classes' rows W [V, D]: logits scale * X W^T + bias, which are not kept.
    labels int32 [N]; a row whose label lies outside [0, V) is ignored.  Returns (loss, lse), float [N]."""
    code, ldx, ldw, N, V, D = _xent_args(X, W, labels, bias)
    if loss is None or lse is None:
        both = torch.empty(2, N, dtype=torch.float32, device=X.device)
        loss, lse = both[0] if loss is None else loss, both[1] if lse is None else lse
    _floats(loss, "loss", N), _floats(lse, "lse", N)
    _here(loss, lse, workspace)
    if N == 0:
        return loss, lse
    workspace, wp, wn = _workspace(workspace, xent_workspace_bytes(code, N, V, D, False), X.device)
    _check(load().ftk_xent(code, X.data_ptr(), ldx, N, W.data_ptr(), ldw, V, D, _ptr(bias), scale, labels.data_ptr(),
                           loss.data_ptr(), lse.data_ptr(), wp, wn, _stream()))
    return loss, lse


def xent_grad(X, W, labels, lse, dloss, bias=None, scale=1.0, dX=None, dW=None, dbias=None, need=(True, True, None), workspace=None):
    """Gradients of sum(dloss * loss), dloss float [N]; lse as xent returned it.  Returns (dX [N, D], dW [V, D], dbias float [V]); those
    that `need` leaves out are None (dbias by default unless there is a bias)."""
    code, ldx, ldw, N, V, D = _xent_args(X, W, labels, bias)
    _floats(lse, "lse", N), _floats(dloss, "dloss", N)
    lddx = lddw = D
    if need[0] or dX is not None:
        dX, lddx = _new_rows(dX, N, D, X, "dX")
    if need[1] or dW is not None:
        dW, lddw = _new_rows(dW, V, D, W, "dW")
    if dbias is not None:
        _floats(dbias, "dbias", V)
    elif need[2] or (need[2] is None and bias is not None):
        dbias = torch.empty(V, dtype=torch.float32, device=X.device)
    _here(lse, dloss, dX, dW, dbias, workspace)
    workspace, wp, wn = _workspace(workspace, xent_workspace_bytes(code, N, V, D, True), X.device)
    # (an empty tensor has no address, and no rows that would need one)
    _check(load().ftk_xent_grad(code, X.data_ptr(), ldx, N, W.data_ptr(), ldw, V, D, _ptr(bias), scale, labels.data_ptr(),
                                lse.data_ptr(), dloss.data_ptr(), _ptr(dX) if N else None, lddx, _ptr(dW), lddw, _ptr(dbias), wp, wn,
                                _stream()))
    return dX, dW, dbias


# ---- many weights updated at once ------------------------------------------------------------


class _AdamwTensor(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("param", "grad", "m", "v", "m_scales", "v_scales", "master")] + [("count", ctypes.c_int64)]


class _AdamwOptions(ctypes.Structure):
    _fields_ = ([(n, ctypes.c_double) for n in ("lr", "beta1", "beta2", "eps", "weight_decay")]
                + [(n, ctypes.c_void_p) for n in ("lr_scale", "grad_scale", "step")] + [("seed", ctypes.c_uint64)])


class AdamW:
    """Weights and their states for adamw_step: contiguous device tensors of one type (float32, bfloat16 or float16), not overlapping,
    which stay where they are in memory, as their states do: new values are copied into them.

    bits: 32 (m, v float32) or 8 (m, v uint8 codes and a scale byte for every 32 elements).  States that are not given start at
    zero.  master: float32 copies of 16-bit weights; True makes them from the weights."""

    def __init__(self, params, bits=32, m=None, v=None, m_scales=None, v_scales=None, master=None):
        if bits not in (8, 32):
            raise ValueError("states have 8 or 32 bits, got %r" % (bits,))
        self.params, self.bits = list(params), bits
        if not self.params:
            raise ValueError("no weights given")
        self.dtype = self.params[0].dtype
        self.code = _row_code(self.params[0], "params", _MX_DTYPES)
        if master and self.dtype == torch.float32:
            raise ValueError("weights in 32 bits are their own masters")
        state, zeros = torch.uint8 if bits == 8 else torch.float32, torch.zeros_like
        self.m = [zeros(p, dtype=state) for p in self.params] if m is None else list(m)
        self.v = [zeros(p, dtype=state) for p in self.params] if v is None else list(v)
        scales = lambda given: [torch.zeros(-(-p.numel() // 32), dtype=torch.uint8, device=p.device)  # noqa: E731
                                for p in self.params] if given is None else list(given)
        self.m_scales, self.v_scales = (scales(m_scales), scales(v_scales)) if bits == 8 else (None, None)
        self.master = [p.float() for p in self.params] if master is True else list(master) if master else None
        self._table = (_AdamwTensor * len(self.params))()
        lists = [("params", self.params, self.dtype), ("m", self.m, state), ("v", self.v, state), ("m_scales", self.m_scales, torch.uint8),
                 ("v_scales", self.v_scales, torch.uint8), ("master", self.master, torch.float32)]
        spans = []
        for name, tensors, dtype in lists:
            if tensors is None:
                continue
            if len(tensors) != len(self.params):
                raise ValueError("%s: %d tensors for %d weights" % (name, len(tensors), len(self.params)))
            for t, p, row in zip(tensors, self.params, self._table):
                need = -(-p.numel() // 32) if name.endswith("scales") else p.numel()
                if not t.is_cuda or t.device != self.params[0].device or t.dtype != dtype or t.numel() != need or not t.is_contiguous():
                    raise ValueError("%s must be contiguous tensors of %s with the weights' elements, on their device" % (name, dtype))
                if need:
                    setattr(row, "param" if name == "params" else name, t.data_ptr())
                    spans.append((t.data_ptr(), t.data_ptr() + need * t.element_size()))
        # (the memory that the table names, held whatever becomes of the states' tensors)
        self._states = list(self._all_states())
        self._memory = [t.detach() for t in self._states]
        self._counts = [p.numel() for p in self.params]
        self._places = [p.data_ptr() for p in self.params]
        for n, row in zip(self._counts, self._table):
            row.count = n
        self._grads = (ctypes.c_uint64 * (8 * len(self.params))).from_buffer(self._table)  # the table by words, the gradient's is the second
        spans.sort()
        if any(a[1] > b[0] for a, b in zip(spans, spans[1:])):
            raise ValueError("weights or states overlap")

    def _all_states(self):
        return itertools.chain(self.m, self.v, self.m_scales or (), self.v_scales or (), self.master or ())

    def _check_states(self):
        if not all(map(operator.is_, self._all_states(), self._states)):
            raise ValueError("states have been replaced since they were given: new values are copied into them")


def _alike(tensors, counts, dtype, device):
    """Contiguous tensors of so many elements, one type and one device (a list of hundreds is gone through at every step)."""
    T = torch.Tensor
    return (list(map(T.numel, tensors)) == counts and set(map(T.get_device, tensors)) == {device} and all(map(T.is_contiguous, tensors))
            and {t.dtype for t in tensors} == {dtype})


def adamw_step(state, grads, step, lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.01, seed=0, lr_scale=None, grad_scale=None):
    """One AdamW step over all of state's weights, in place.  grads: a contiguous tensor for each weight, of one type (float32 or the
    weights'; float32 weights: any), or None: that weight stays.  step: int64 device tensor of one element, 1 at the first
    step.  lr_scale, grad_scale: float32 device tensors of one element that multiply the rate and the gradients.  seed: of the
    rounding of 8-bit states."""
    given = [g for g in grads if g is not None]
    counts = state._counts
    if len(grads) != len(counts):
        raise ValueError("%d gradients for %d weights" % (len(grads), len(counts)))
    if not given:
        return
    if len(given) < len(counts):
        counts = [n for n, g in zip(counts, grads) if g is not None]
    dtype, device = given[0].dtype, state.params[0].get_device()
    if not _alike(given, counts, dtype, device):
        raise ValueError("gradients must be contiguous tensors of one type with the weights' elements, on their device")
    if list(map(torch.Tensor.data_ptr, state.params)) != state._places:
        raise ValueError("weights have moved since their state was made")
    state._check_states()
    state._grads[1::8] = [0 if g is None else g.data_ptr() for g in grads]
    code = _MX_DTYPES.get(dtype)
    if code is None:
        raise TypeError("gradients: %s is not one of float32, bfloat16, float16" % dtype)
    if not step.is_cuda or step.dtype != torch.int64 or step.numel() != 1:
        raise ValueError("step must be an int64 device tensor of one element")
    for t, name in ((lr_scale, "lr_scale"), (grad_scale, "grad_scale")):
        if t is not None and (not t.is_cuda or t.dtype != torch.float32 or t.numel() != 1):
            raise ValueError("%s must be a float32 device tensor of one element" % name)
    _here(state.params[0], step, lr_scale, grad_scale)
    options = _AdamwOptions(lr, beta1, beta2, eps, weight_decay, _ptr(lr_scale), _ptr(grad_scale), step.data_ptr(), seed & (2**64 - 1))
    _check(load().ftk_adamw_step(state.code, code, state.bits, state._table, len(grads), ctypes.byref(options), _stream()))


def adamw_moments(state, out=None, dtype=torch.float32):
    """What 8-bit states stand for: lists (m, v) of tensors of the weights' sizes; out: such a pair of lists to write to."""
    if state.bits != 8:
        raise ValueError("states in 32 bits are their own values")
    if out is None:
        out = [[torch.empty_like(p, dtype=dtype) for p in state.params] for _ in range(2)]
    state._check_states()
    dtype, device, lists = out[0][0].dtype, state.params[0].get_device(), []
    for ts in out:
        if not _alike(ts, state._counts, dtype, device):
            raise ValueError("out must be two lists of contiguous tensors of one type with the weights' elements, on their device")
        pointers = (ctypes.c_void_p * len(ts))()
        pointers[:] = list(map(torch.Tensor.data_ptr, ts))
        lists.append(pointers)
    _here(state.params[0])
    _check(load().ftk_adamw_moments(_row_code(out[0][0], "out", _MX_DTYPES), state._table, len(state.params), lists[0], lists[1], _stream()))
    return out
