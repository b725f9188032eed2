"""Binding of libsgap.so: argument marshalling only.

sgap_spmm_csr_ex, sgap_spmm_csr_cfg, sgap_sddmm_csr, sgap_sddmm_csr_windows, sgap_ttm_csf, sgap_mttkrp_csf_ex and the
calls of a mixture of experts (sgap_route_*, sgap_grouped_*, sgap_embed*, sgap_f8_*) go through a small native module
(csrc/sgap_python.cpp), which reads the tensors and calls the library in a few hundred nanoseconds; what it does not take (another type, a wrong length, a number that is no int) goes through ctypes and the
checks below, which say what is wrong.  The other calls, and all of them where that module has not been built, go
through ctypes: about 8 us of host time each.

Function names mirror the C ABI in include/sgap.h.  Tensors are torch CUDA
tensors (used purely as device memory); every computation happens in the HIP
kernels of the library.  There is no fallback: if the shared library is not
built, or a tensor is not on the GPU, the call raises.
"""
from __future__ import annotations

import ctypes
import os

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libsgap.so")

SGAP_OK = 0
SGAP_ERR_INVALID_ARG = 1
SGAP_ERR_UNSUPPORTED = 2
SGAP_ERR_HIP = 3

SGAP_REDUCE_PARALLEL = 0
SGAP_REDUCE_SERIAL = 1
SGAP_SCHED_ROW_SPLIT = 0
SGAP_SCHED_NNZ_BALANCED = 1

STRATEGIES = {"parallel": SGAP_REDUCE_PARALLEL, "serial": SGAP_REDUCE_SERIAL}
SCHEDULES = {"row_split": SGAP_SCHED_ROW_SPLIT, "nnz_balanced": SGAP_SCHED_NNZ_BALANCED}
STRATEGY_NAMES = {v: k for k, v in STRATEGIES.items()}
SCHEDULE_NAMES = {v: k for k, v in SCHEDULES.items()}
GROUP_SIZES = (1, 2, 4, 8, 16, 32, 64)

# every symbol include/sgap.h and include/sgap_debug.h declare: name -> (restype, argtypes)
_i64, _int, _p = ctypes.c_int64, ctypes.c_int, ctypes.c_void_p
EXPORTS = {
    "sgap_set_schedule": (_int, [_int]),
    "sgap_get_schedule": (_int, []),
    "sgap_spmm_csr": (_int, [_i64, _i64, _i64, _p, _p, _p, _p, _p, _int, _int, _p]),
    "sgap_spmm_csr_ex": (_int, [_i64, _i64, _i64, _p, _p, _p, _p, _p, _int, _int, _int, _i64, _p]),
    "sgap_spmm_csr_gr": (_int, [_i64, _i64, _i64, _p, _p, _p, _p, _p, _int, _int, _i64, _p]),
    "sgap_config_init": (_int, [_p]),
    "sgap_spmm_csr_workspace_size": (_i64, [_i64, _i64, _i64, _p]),
    "sgap_spmm_csr_cfg": (_int, [_i64, _i64, _i64, _p, _p, _p, _p, _p, _p, _i64, _p, _i64, _p]),
    "sgap_spmm_csr_cfg_static": (_int, [_i64, _i64, _i64, _p, _p, _p, _p, _p, _p, _i64, _p]),
    "sgap_autotune_csr": (_int, [_i64, _i64, _i64, _p, _p, _p, _p, _p, _i64, _int, _p, _p, _p]),
    "sgap_autotune_csr_cfg": (_int, [_i64, _i64, _i64, _p, _p, _p, _p, _p, _i64, _int, _p, _i64, _p, _int, _p, _p, _p]),
    "sgap_sddmm_csr": (_int, [_i64, _i64, _i64, _p, _p, _p, _p, _p, _p, _int, _int, _i64, _p]),
    "sgap_sddmm_csr_windows": (_int, [_i64, _i64, _i64, _p, _p, _p, _p, _p, _p, _int, _int, _i64, _int, _int, _int, _p,
                                      _i64, _p]),
    "sgap_sddmm_csr_workspace_size": (_i64, [_i64, _i64, _int, _int]),
    "sgap_validate_csr": (_int, [_i64, _i64, _p, _p, _i64, _p, _p]),
    "sgap_reorder_rows_workspace_size": (_i64, [_i64]),
    "sgap_reorder_rows_csr": (_int, [_i64, _i64, _p, _p, _p, _int, _p, _p, _p, _p, _p, _i64, _p]),
    "sgap_ttm_csf": (_int, [_i64, _i64, _i64, _p, _p, _p, _p, _p, _int, _int, _int, _i64, _p]),
    "sgap_mttkrp_csf": (_int, [_i64, _i64, _i64, _i64, _p, _p, _p, _p, _p, _p, _p, _p, _int, _int, _p]),
    "sgap_mttkrp_csf_ex": (_int, [_i64, _i64, _i64, _i64, _p, _p, _p, _p, _p, _p, _p, _p, _int, _int, _int, _i64, _p]),
    "sgap_route_topk_workspace_size": (_i64, [_i64, _i64, _i64]),
    "sgap_route_topk": (_int, [_i64, _i64, _i64, _int, _p, _i64, _int, _p, _p, _p, _p, _p, _p, _i64, _p]),
    "sgap_route_topk_grad": (_int, [_i64, _i64, _i64, _int, _p, _i64, _int, _p, _p, _p, _p, _i64, _p]),
    "sgap_route_combine": (_int, [_i64, _i64, _i64, _int, _p, _p, _p, _p, _p]),
    "sgap_route_combine_grad": (_int, [_i64, _i64, _i64, _int, _p, _p, _p, _p, _p, _p, _p, _p]),
    "sgap_grouped_mm": (_int, [_i64, _i64, _i64, _i64, _int, _p, _p, _i64, _i64, _p, _i64, _p, _int, _p, _i64, _p]),
    "sgap_grouped_mm_wgrad": (_int, [_i64, _i64, _i64, _i64, _int, _p, _p, _i64, _i64, _p, _i64, _p, _i64, _p, _int, _p]),
    "sgap_w4_layout_size": (_i64, [_i64, _i64, _i64, _i64, _int]),
    "sgap_w4_layout": (_int, [_i64, _i64, _i64, _i64, _p, _p, _p, _p, _i64, _p]),
    "sgap_grouped_mm_w4": (_int, [_i64, _i64, _i64, _i64, _int, _i64, _int, _p, _p, _i64, _i64, _p, _i64, _p, _i64, _p, _i64, _p]),
    "sgap_route_balance_workspace_size": (_i64, [_i64, _i64, _i64, _i64]),
    "sgap_route_balance": (_int, [_i64, _i64, _i64, _i64, _int, _p, _i64, _p, _p, _p, _p, _p, _p, _i64, _p]),
    "sgap_route_balance_grad": (_int, [_i64, _i64, _i64, _i64, _int, _p, _i64, _p, _p, _p, _p, _p, _int, _p, _i64, _p]),
    "sgap_embed": (_int, [_i64, _i64, _i64, _int, _p, _p, _i64, ctypes.c_float, _p, _i64, _p]),
    "sgap_embed_grad_workspace_size": (_i64, [_i64, _i64, _i64]),
    "sgap_embed_grad": (_int, [_i64, _i64, _i64, _int, _p, _p, _i64, ctypes.c_float, _int, _int, _p, _i64, _p, _i64, _p]),
    "sgap_f8_rows": (_int, [_i64, _i64, _int, _p, _i64, _p, _p, _p]),
    "sgap_f8_weights": (_int, [_i64, _i64, _i64, _int, _p, _p, _p, _p, _p, _p]),
    "sgap_grouped_mm_f8": (_int, [_i64, _i64, _i64, _i64, _int, _p, _p, _p, _i64, _p, _i64, _p, _p, _p, _i64, _p]),
    "sgap_status_string": (ctypes.c_char_p, [_int]),
    "sgap_last_error": (ctypes.c_char_p, []),
    "sgap_version": (_int, []),
    "sgap_set_tuning": (_int, [_int, _int]),
    "sgap_profile_enable": (_int, [_int]),
    "sgap_profile_collect": (_int, [ctypes.POINTER(ctypes.c_double), ctypes.POINTER(_int)]),
    "sgap_debug_group_reduce": (_int, [_p, _p, _int, _int, _p]),
    "sgap_debug_group_partial_reduce": (_int, [_p, _p, _int, _int, _int, _p]),
    "sgap_debug_group_seg_reduce": (_int, [_p, _p, _p, _int, _int, _p]),
    "sgap_debug_tile_deal": (_i64, [_i64, _int, _int, _p, _i64]),
    "sgap_debug_plan_nnz_serial": (_int, [_int, _int, _int, _i64, _int, _int, _p, _p, _p]),
    "sgap_debug_finder_rows": (_i64, [_i64, _int, _int, _p, _i64]),
    "sgap_debug_plan_row_split": (_int, [_int, _int, _i64, _i64, _int, _int, _i64, _int, _p, _p, _p, _p, _p]),
    "sgap_debug_plan_windows": (_int, [_int] + [_i64] * 8 + [_int] * 3 + [_p] * 6),
    "sgap_debug_row_quads": (_int, [_i64, _i64, _i64, _p, _int]),
    "sgap_debug_spmm_teams": (_int, [_i64, _i64, _i64, _i64, _p, _int]),
    "sgap_debug_mttkrp_teams": (_int, [_i64, _i64, _int, _int, _int, _i64]),
    "sgap_debug_sddmm_quads": (_int, [_i64, _i64, _i64, _int, _i64, _p, _p]),
    "sgap_debug_grouped_plan": (_int, [_i64, _i64, _i64, _i64, _int, _int, _i64, _i64, _i64, _int, _int, _int, _int, _p]),
    "sgap_debug_f8_plan": (_int, [_i64, _i64, _i64, _i64, _int, _int, _int, _i64, _int, _p]),
    "sgap_copy_f32": (_int, [_p, _p, _i64, _p]),
    "sgap_stream_f32": (_int, [_p, _p, _i64, _int, _p]),
}

_lib = None
_native = None


class SgapError(RuntimeError):
    def __init__(self, status: int, what: str):
        super().__init__(f"sgap status {status} ({what})")
        self.status = status


def load():
    """Load libsgap.so (once).  Raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(
                f"{LIB_PATH} is missing: build it with `python -m paper_2209_02882_amd.build` "
                "(there is no CPU fallback)")
        lib = ctypes.CDLL(LIB_PATH)
        for name, (res, args) in EXPORTS.items():
            fn = getattr(lib, name)
            fn.restype = res
            fn.argtypes = args
        _lib = lib
    return _lib


class _TakesNothing:
    """In the native module's place where that is missing: every call is left to ctypes."""

    def __getattr__(self, name):
        return lambda *args: -1


def _load_native():
    """The native module (once); without it the calls work all the same, and a warning says that they are slow."""
    global _native
    if _native is None:
        import torch  # noqa: F401  (its libraries have to be there first)

        load()
        try:
            from . import _native as module
        except ImportError as e:
            import warnings

            warnings.warn(f"calls go through ctypes, about 8 us each: the native module cannot be loaded ({e}); build it "
                          "with `python -m paper_2209_02882_amd.build`", RuntimeWarning, stacklevel=3)
            module = _TakesNothing()
        _native = module
    return _native


def _check(status: int):
    if status != SGAP_OK:
        lib = load()
        what = lib.sgap_status_string(status).decode()
        detail = lib.sgap_last_error().decode()
        raise SgapError(status, f"{what}: {detail}" if detail else what)


def _dev_ptr(t, dtype, name):
    import torch

    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a CUDA tensor (device memory)")
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t.data_ptr() if t.numel() else None


def _stream_ptr(stream):
    import torch

    if stream is None:
        stream = torch.cuda.current_stream()
    return ctypes.c_void_p(stream.cuda_stream)


def sgap_version() -> int:
    return load().sgap_version()


def sgap_set_schedule(schedule: int) -> None:
    _check(load().sgap_set_schedule(int(schedule)))


def sgap_get_schedule() -> int:
    return load().sgap_get_schedule()


def _spmm_args(M, K, N, rowptr, colidx, vals, B, C):
    import torch

    if rowptr.numel() != M + 1:
        raise ValueError("rowptr must have M+1 entries")
    if colidx.numel() != vals.numel():
        raise ValueError("colidx and vals must have the same length")
    if B.numel() != K * N or C.numel() != M * N:
        raise ValueError("B must hold K*N and C must hold M*N elements")
    return (
        _dev_ptr(rowptr, torch.int32, "rowptr"), _dev_ptr(colidx, torch.int32, "colidx"),
        _dev_ptr(vals, torch.float32, "vals"), _dev_ptr(B, torch.float32, "B"),
        _dev_ptr(C, torch.float32, "C"))


def sgap_spmm_csr(M, K, N, rowptr, colidx, vals, B, C, group_size, strategy, stream=None) -> None:
    """C = A_csr * B with the process-wide schedule (see include/sgap.h)."""
    ptrs = _spmm_args(M, K, N, rowptr, colidx, vals, B, C)
    _check(load().sgap_spmm_csr(M, K, N, *ptrs, int(group_size), int(strategy), _stream_ptr(stream)))


def sgap_spmm_csr_ex(M, K, N, rowptr, colidx, vals, B, C, group_size, strategy, schedule,
                     nnz_hint=None, stream=None) -> None:
    """C = A_csr * B with an explicit schedule.  nnz_hint defaults to the
    length of colidx, which the host knows without touching the device."""
    st = (_native or _load_native()).spmm_csr_ex(M, K, N, rowptr, colidx, vals, B, C, group_size, strategy, schedule, nnz_hint, stream)
    if st == 0:
        return
    if st > 0:
        _check(st)
    ptrs = _spmm_args(M, K, N, rowptr, colidx, vals, B, C)
    if nnz_hint is None:
        nnz_hint = colidx.numel()
    _check(load().sgap_spmm_csr_ex(M, K, N, *ptrs, int(group_size), int(strategy), int(schedule),
                                   int(nnz_hint), _stream_ptr(stream)))


SGAP_TUNE_TILE_COLS = 0
SGAP_TUNE_XCD_REMAP = 1
SGAP_TUNE_ROWS_PER_GROUP = 2
SGAP_TUNE_PERSISTENT = 3
SGAP_TUNE_NNZ_TILE = 4
SGAP_TUNE_SDDMM_ROW_CACHE = 5


class Config(ctypes.Structure):
    """Mirror of sgap_config: the point of the design space and the tiling knobs of one call."""
    _fields_ = [(name, ctypes.c_int) for name in (
        "schedule", "strategy", "group_size", "reduce_size", "block_size", "tile_cols", "rows_per_group",
        "xcd_remap", "persistent", "nnz_tile", "wave_rows", "long_row_min", "window_kb", "max_long_rows")]

    def as_dict(self):
        return {name: getattr(self, name) for name, _ in self._fields_}


def make_config(group_size, strategy, schedule, **knobs) -> Config:
    """sgap_config with the library's defaults (sgap_config_init) and the named fields set; strategy and
    schedule by name or number."""
    c = Config()
    _check(load().sgap_config_init(ctypes.byref(c)))
    c.group_size = int(group_size)
    c.strategy = STRATEGIES.get(strategy, strategy)
    c.schedule = SCHEDULES.get(schedule, schedule)
    for k, v in knobs.items():
        if k not in dict(Config._fields_):
            raise KeyError(k)
        setattr(c, k, int(v))
    return c


def sgap_spmm_csr_workspace_size(M, K, N, config: Config) -> int:
    size = load().sgap_spmm_csr_workspace_size(M, K, N, ctypes.byref(config))
    if size < 0:
        raise SgapError(SGAP_ERR_INVALID_ARG, load().sgap_last_error().decode())
    return size


def _workspace_args(workspace):
    import torch

    if workspace is None:
        return None, 0
    if not isinstance(workspace, torch.Tensor) or not workspace.is_cuda or workspace.dtype != torch.uint8:
        raise TypeError("workspace must be a CUDA uint8 tensor")
    return (workspace.data_ptr() if workspace.numel() else None), workspace.numel()


def sgap_spmm_csr_cfg(M, K, N, rowptr, colidx, vals, B, C, config: Config, nnz_hint=None, workspace=None,
                      stream=None) -> None:
    """C = A_csr * B at the point and with the tiling `config` names; `workspace` is a CUDA uint8 tensor of
    at least sgap_spmm_csr_workspace_size bytes when the configuration sets long rows apart."""
    st = (_native or _load_native()).spmm_csr_cfg(M, K, N, rowptr, colidx, vals, B, C, config, nnz_hint, workspace, stream)
    if st == 0:
        return
    if st > 0:
        _check(st)
    ptrs = _spmm_args(M, K, N, rowptr, colidx, vals, B, C)
    if nnz_hint is None:
        nnz_hint = colidx.numel()
    ws, ws_bytes = _workspace_args(workspace)
    _check(load().sgap_spmm_csr_cfg(M, K, N, *ptrs, ctypes.byref(config), int(nnz_hint), ws, ws_bytes,
                                    _stream_ptr(stream)))


def sgap_set_tuning(knob: int, value: int) -> None:
    _check(load().sgap_set_tuning(int(knob), int(value)))


def sgap_profile_enable(on: bool) -> None:
    _check(load().sgap_profile_enable(1 if on else 0))


def sgap_profile_collect():
    """(total milliseconds, number of timed main-kernel launches) since the last collect."""
    total = ctypes.c_double(0.0)
    count = ctypes.c_int(0)
    _check(load().sgap_profile_collect(ctypes.byref(total), ctypes.byref(count)))
    return total.value, count.value


def sgap_spmm_csr_gr(M, K, N, rowptr, colidx, vals, B, C, group_size, reduce_size, nnz_hint=None,
                     stream=None) -> None:
    """Row-split C = A_csr * B with group_size lanes per row reducing in
    sub-groups of reduce_size lanes (see include/sgap.h)."""
    ptrs = _spmm_args(M, K, N, rowptr, colidx, vals, B, C)
    if nnz_hint is None:
        nnz_hint = colidx.numel()
    _check(load().sgap_spmm_csr_gr(M, K, N, *ptrs, int(group_size), int(reduce_size), int(nnz_hint),
                                   _stream_ptr(stream)))


def sgap_sddmm_csr(M, K, J, rowptr, colidx, vals, X1, X2T, out_vals, group_size, strategy, nnz_hint=None,
                   stream=None) -> None:
    """out_vals[p] = vals[p] * <X1[row(p), :], X2T[colidx[p], :]> (see include/sgap.h)."""
    st = (_native or _load_native()).sddmm_csr(M, K, J, rowptr, colidx, vals, X1, X2T, out_vals, group_size, strategy, nnz_hint, stream)
    if st == 0:
        return
    if st > 0:
        _check(st)
    import torch

    if rowptr.numel() != M + 1:
        raise ValueError("rowptr must have M+1 entries")
    if colidx.numel() != vals.numel() or out_vals.numel() != vals.numel():
        raise ValueError("colidx, vals and out_vals must have the same length")
    if X1.numel() != M * J or X2T.numel() != K * J:
        raise ValueError("X1 must hold M*J and X2T must hold K*J elements")
    if nnz_hint is None:
        nnz_hint = colidx.numel()
    _check(load().sgap_sddmm_csr(
        M, K, J, _dev_ptr(rowptr, torch.int32, "rowptr"), _dev_ptr(colidx, torch.int32, "colidx"),
        _dev_ptr(vals, torch.float32, "vals"), _dev_ptr(X1, torch.float32, "X1"),
        _dev_ptr(X2T, torch.float32, "X2T"), _dev_ptr(out_vals, torch.float32, "out_vals"),
        int(group_size), int(strategy), int(nnz_hint), _stream_ptr(stream)))


def sgap_sddmm_csr_workspace_size(K, J, window_kb=0, max_long_rows=0) -> int:
    size = load().sgap_sddmm_csr_workspace_size(K, J, int(window_kb), int(max_long_rows))
    if size < 0:
        raise SgapError(SGAP_ERR_INVALID_ARG, load().sgap_last_error().decode())
    return size


def sgap_sddmm_csr_windows(M, K, J, rowptr, colidx, vals, X1, X2T, out_vals, group_size, strategy, long_row_min,
                           window_kb=0, max_long_rows=0, workspace=None, nnz_hint=None, stream=None) -> None:
    """sgap_sddmm_csr with the stored entries of rows of at least long_row_min entries taken by column
    windows of X2T (see include/sgap.h)."""
    st = (_native or _load_native()).sddmm_csr_windows(M, K, J, rowptr, colidx, vals, X1, X2T, out_vals, group_size, strategy, nnz_hint,
                                                        long_row_min, window_kb, max_long_rows, workspace, stream)
    if st == 0:
        return
    if st > 0:
        _check(st)
    import torch

    if rowptr.numel() != M + 1:
        raise ValueError("rowptr must have M+1 entries")
    if colidx.numel() != vals.numel() or out_vals.numel() != vals.numel():
        raise ValueError("colidx, vals and out_vals must have the same length")
    if X1.numel() != M * J or X2T.numel() != K * J:
        raise ValueError("X1 must hold M*J and X2T must hold K*J elements")
    if nnz_hint is None:
        nnz_hint = colidx.numel()
    ws, ws_bytes = _workspace_args(workspace)
    _check(load().sgap_sddmm_csr_windows(
        M, K, J, _dev_ptr(rowptr, torch.int32, "rowptr"), _dev_ptr(colidx, torch.int32, "colidx"),
        _dev_ptr(vals, torch.float32, "vals"), _dev_ptr(X1, torch.float32, "X1"),
        _dev_ptr(X2T, torch.float32, "X2T"), _dev_ptr(out_vals, torch.float32, "out_vals"),
        int(group_size), int(strategy), int(nnz_hint), int(long_row_min), int(window_kb), int(max_long_rows),
        ws, ws_bytes, _stream_ptr(stream)))


def sgap_ttm_csf(F, K, L, eptr, eidx, vals, X1, Yf, group_size, strategy, schedule, nnz_hint=None,
                 stream=None) -> None:
    """Yf[f, :] = sum over the entries p of fiber f of vals[p] * X1[eidx[p], :] (see include/sgap.h)."""
    st = (_native or _load_native()).spmm_csr_ex(F, K, L, eptr, eidx, vals, X1, Yf, group_size, strategy, schedule, nnz_hint, stream)
    if st == 0:
        return
    if st > 0:
        _check(st)
    ptrs = _spmm_args(F, K, L, eptr, eidx, vals, X1, Yf)
    if nnz_hint is None:
        nnz_hint = eidx.numel()
    _check(load().sgap_ttm_csf(F, K, L, *ptrs, int(group_size), int(strategy), int(schedule), int(nnz_hint),
                               _stream_ptr(stream)))


def sgap_mttkrp_csf(I, K, L, J, fptr, fidx, eptr, eidx, vals, X1, X2, Y, group_size, strategy, stream=None) -> None:
    """Y[i, j] = sum over the stored (i, k, l) of A[i,k,l] * X1[k, j] * X2[l, j] (see include/sgap.h)."""
    import torch

    if fptr.numel() != I + 1:
        raise ValueError("fptr must have I+1 entries")
    if eptr.numel() != fidx.numel() + 1:
        raise ValueError("eptr must have one entry more than fidx")
    if eidx.numel() != vals.numel():
        raise ValueError("eidx and vals must have the same length")
    if X1.numel() != K * J or X2.numel() != L * J or Y.numel() != I * J:
        raise ValueError("X1 must hold K*J, X2 L*J and Y I*J elements")
    _check(load().sgap_mttkrp_csf(
        I, K, L, J, _dev_ptr(fptr, torch.int32, "fptr"), _dev_ptr(fidx, torch.int32, "fidx"),
        _dev_ptr(eptr, torch.int32, "eptr"), _dev_ptr(eidx, torch.int32, "eidx"),
        _dev_ptr(vals, torch.float32, "vals"), _dev_ptr(X1, torch.float32, "X1"), _dev_ptr(X2, torch.float32, "X2"),
        _dev_ptr(Y, torch.float32, "Y"), int(group_size), int(strategy), _stream_ptr(stream)))


def sgap_mttkrp_csf_ex(I, K, L, J, fptr, fidx, eptr, eidx, vals, X1, X2, Y, group_size, strategy, schedule,
                       nnz_hint=None, stream=None) -> None:
    """sgap_mttkrp_csf with a choice of schedule: slices (row-split) or stored entries (nnz-balanced) as the
    unit of work.  nnz_hint defaults to the length of vals."""
    st = (_native or _load_native()).mttkrp_csf_ex(I, K, L, J, fptr, fidx, eptr, eidx, vals, X1, X2, Y, group_size, strategy, schedule,
                                                    nnz_hint, stream)
    if st == 0:
        return
    if st > 0:
        _check(st)
    import torch

    if fptr.numel() != I + 1:
        raise ValueError("fptr must have I+1 entries")
    if eptr.numel() != fidx.numel() + 1:
        raise ValueError("eptr must have one entry more than fidx")
    if eidx.numel() != vals.numel():
        raise ValueError("eidx and vals must have the same length")
    if X1.numel() != K * J or X2.numel() != L * J or Y.numel() != I * J:
        raise ValueError("X1 must hold K*J, X2 L*J and Y I*J elements")
    if nnz_hint is None:
        nnz_hint = vals.numel()
    _check(load().sgap_mttkrp_csf_ex(
        I, K, L, J, _dev_ptr(fptr, torch.int32, "fptr"), _dev_ptr(fidx, torch.int32, "fidx"),
        _dev_ptr(eptr, torch.int32, "eptr"), _dev_ptr(eidx, torch.int32, "eidx"),
        _dev_ptr(vals, torch.float32, "vals"), _dev_ptr(X1, torch.float32, "X1"), _dev_ptr(X2, torch.float32, "X2"),
        _dev_ptr(Y, torch.float32, "Y"), int(group_size), int(strategy), int(schedule), int(nnz_hint),
        _stream_ptr(stream)))


def sgap_validate_csr(M, K, rowptr, colidx, stream=None):
    """Counts of (rowptr defects, columns out of range, unsorted or repeated
    columns, empty rows) of a CSR matrix in device memory; the last two are -1
    when rowptr is damaged.  Waits for the stream (see include/sgap.h)."""
    import torch

    if rowptr.numel() != M + 1:
        raise ValueError("rowptr must have M+1 entries")
    report = (ctypes.c_int64 * 4)()
    _check(load().sgap_validate_csr(M, K, _dev_ptr(rowptr, torch.int32, "rowptr"),
                                    _dev_ptr(colidx, torch.int32, "colidx"), colidx.numel(), report,
                                    _stream_ptr(stream)))
    return tuple(report)


ROW_ORDERS = {"first_column": 0, "length": 1}


def sgap_reorder_rows_workspace_size(M):
    size = load().sgap_reorder_rows_workspace_size(M)
    if size < 0:
        raise SgapError(SGAP_ERR_INVALID_ARG, load().sgap_last_error().decode())
    return size


def sgap_reorder_rows_csr(M, K, rowptr, colidx, vals, order, perm, rowptr_out, colidx_out, vals_out, workspace,
                          stream=None):
    """Enqueue the row reordering of a CSR matrix in device memory (see include/sgap.h); `order` is a name of
    ROW_ORDERS or its number.  All arrays are the caller's tensors; nothing is allocated here."""
    import torch

    if rowptr.numel() != M + 1 or rowptr_out.numel() != M + 1:
        raise ValueError("rowptr and rowptr_out must have M+1 entries")
    if perm.numel() != M:
        raise ValueError("perm must have M entries")
    if colidx_out.numel() != colidx.numel() or vals_out.numel() != vals.numel() or vals.numel() != colidx.numel():
        raise ValueError("colidx, vals and their outputs must have nnz entries each")
    ws_ptr, ws_bytes = _workspace_args(workspace)
    _check(load().sgap_reorder_rows_csr(M, K, _dev_ptr(rowptr, torch.int32, "rowptr"),
                                        _dev_ptr(colidx, torch.int32, "colidx"), _dev_ptr(vals, torch.float32, "vals"),
                                        ROW_ORDERS.get(order, order), _dev_ptr(perm, torch.int32, "perm"),
                                        _dev_ptr(rowptr_out, torch.int32, "rowptr_out"),
                                        _dev_ptr(colidx_out, torch.int32, "colidx_out"),
                                        _dev_ptr(vals_out, torch.float32, "vals_out"), ws_ptr, ws_bytes,
                                        _stream_ptr(stream)))


class PointTime(ctypes.Structure):
    """Mirror of sgap_point_time."""
    _fields_ = [("group_size", ctypes.c_int), ("strategy", ctypes.c_int), ("schedule", ctypes.c_int),
                ("ms", ctypes.c_float)]


SGAP_NUM_POINTS = 28


def sgap_autotune_csr(M, K, N, rowptr, colidx, vals, B, C, nnz_hint=None, reps=3, stream=None):
    """Time every design-space point on these operands (blocking).  Returns
    (best, table): PointTime of the fastest point and the list of all 28."""
    ptrs = _spmm_args(M, K, N, rowptr, colidx, vals, B, C)
    if nnz_hint is None:
        nnz_hint = colidx.numel()
    table = (PointTime * SGAP_NUM_POINTS)()
    best = PointTime()
    _check(load().sgap_autotune_csr(M, K, N, *ptrs, int(nnz_hint), int(reps),
                                    ctypes.cast(table, ctypes.c_void_p), ctypes.cast(ctypes.pointer(best), ctypes.c_void_p),
                                    _stream_ptr(stream)))
    return best, list(table)


def sgap_spmm_csr_cfg_static(M, K, N, rowptr, colidx, vals, B, C, config: Config, nnz_hint=None, stream=None) -> None:
    """sgap_spmm_csr_cfg with the working memory in the library's built-in array (no allocation anywhere)."""
    ptrs = _spmm_args(M, K, N, rowptr, colidx, vals, B, C)
    if nnz_hint is None:
        nnz_hint = colidx.numel()
    _check(load().sgap_spmm_csr_cfg_static(M, K, N, *ptrs, ctypes.byref(config), int(nnz_hint), _stream_ptr(stream)))


class TunedPoint(ctypes.Structure):
    """Mirror of sgap_tuned_point."""
    _fields_ = [("config", Config), ("ms", ctypes.c_float)]


SGAP_MAX_TUNED_POINTS = 96


def sgap_autotune_csr_cfg(M, K, N, rowptr, colidx, vals, B, C, nnz_hint=None, reps=3, workspace=None, stream=None):
    """Rate the whole configuration space on these operands (blocking).  Returns (best, table): the
    fastest TunedPoint and the list of all rated ones."""
    ptrs = _spmm_args(M, K, N, rowptr, colidx, vals, B, C)
    if nnz_hint is None:
        nnz_hint = colidx.numel()
    ws, ws_bytes = _workspace_args(workspace)
    table = (TunedPoint * SGAP_MAX_TUNED_POINTS)()
    best = TunedPoint()
    count = ctypes.c_int(0)
    _check(load().sgap_autotune_csr_cfg(M, K, N, *ptrs, int(nnz_hint), int(reps), ws, ws_bytes,
                                        ctypes.cast(table, ctypes.c_void_p), SGAP_MAX_TUNED_POINTS,
                                        ctypes.cast(ctypes.pointer(count), ctypes.c_void_p),
                                        ctypes.cast(ctypes.pointer(best), ctypes.c_void_p), _stream_ptr(stream)))
    return best, list(table)[:min(count.value, SGAP_MAX_TUNED_POINTS)]


def sgap_debug_group_partial_reduce(inp, out, group_size, reduce_size, lanes_per_row, stream=None) -> None:
    import torch

    _check(load().sgap_debug_group_partial_reduce(
        _dev_ptr(inp, torch.float32, "in"), _dev_ptr(out, torch.float32, "out"),
        int(group_size), int(reduce_size), int(lanes_per_row), _stream_ptr(stream)))


def sgap_debug_group_reduce(inp, out, group_size, lanes_per_row, stream=None) -> None:
    import torch

    _check(load().sgap_debug_group_reduce(
        _dev_ptr(inp, torch.float32, "in"), _dev_ptr(out, torch.float32, "out"),
        int(group_size), int(lanes_per_row), _stream_ptr(stream)))


def sgap_debug_group_seg_reduce(inp, span, out, group_size, lanes_per_row, stream=None) -> None:
    import torch

    _check(load().sgap_debug_group_seg_reduce(
        _dev_ptr(inp, torch.float32, "in"), _dev_ptr(span, torch.int32, "span"),
        _dev_ptr(out, torch.float32, "out"), int(group_size), int(lanes_per_row), _stream_ptr(stream)))


def sgap_copy_f32(src, dst, n=None, stream=None) -> None:
    import torch

    if n is None:
        n = src.numel()
    if n > src.numel() or n > dst.numel():
        raise ValueError("copy length exceeds a buffer")
    _check(load().sgap_copy_f32(_dev_ptr(src, torch.float32, "src"), _dev_ptr(dst, torch.float32, "dst"),
                                int(n), _stream_ptr(stream)))


def sgap_stream_f32(src, dst, n, mode, stream=None) -> None:
    """mode 0: copy src -> dst; 1: read src only (dst: a one-float sink); 2: write dst only (see include/sgap_debug.h)."""
    import torch

    _check(load().sgap_stream_f32(_dev_ptr(src, torch.float32, "src") if src is not None else None,
                                  _dev_ptr(dst, torch.float32, "dst"), int(n), int(mode), _stream_ptr(stream)))


# --------------------------------------------------------------------------
# mixtures of experts
# --------------------------------------------------------------------------

SGAP_F32, SGAP_F16, SGAP_BF16 = 0, 1, 2
SGAP_MAX_EXPERTS, SGAP_MAX_CHOSEN = 1024, 16
WEIGHT_LAYOUTS = {"nk": 0, "kn": 1}


def _element_type(t, name):
    import torch

    types = {torch.float32: SGAP_F32, torch.float16: SGAP_F16, torch.bfloat16: SGAP_BF16}
    if not isinstance(t, torch.Tensor) or t.dtype not in types:
        raise TypeError(f"{name} must be a float32, float16 or bfloat16 tensor")
    return types[t.dtype]


def _flat(t, dtype, count, name):
    """Device pointer of a contiguous tensor of `count` elements."""
    ptr = _dev_ptr(t, dtype, name)
    if t.numel() != count:
        raise ValueError(f"{name} must have {count} elements, got {t.numel()}")
    return ptr


def _rows(t, dtype, rows, columns, name):
    """(device pointer, elements from row to row) of a matrix whose rows are contiguous."""
    import torch

    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a CUDA tensor (device memory)")
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if t.dim() != 2 or (rows is not None and t.shape[0] != rows) or t.shape[1] != columns:
        raise ValueError(f"{name} must be {'any number of' if rows is None else rows} rows of {columns}, got {tuple(t.shape)}")
    if (columns > 1 and t.stride(1) != 1) or (t.shape[0] > 1 and t.stride(0) < columns):
        raise ValueError(f"the rows of {name} must be contiguous and must not overlap")
    return (t.data_ptr() if t.numel() else None), (t.stride(0) if t.shape[0] > 1 else columns)


def _bytes(t, name):
    """(device pointer, bytes) of a contiguous uint8 tensor, or of None."""
    import torch

    return (None, 0) if t is None else (_dev_ptr(t, torch.uint8, name), t.numel())


def sgap_route_topk_workspace_size(T, E, k) -> int:
    size = load().sgap_route_topk_workspace_size(int(T), int(E), int(k))
    if size < 0:
        raise SgapError(SGAP_ERR_INVALID_ARG, load().sgap_last_error().decode())
    return size


def sgap_route_topk(T, E, k, logits, gates, experts, slot, order, offsets, renormalise=True, workspace=None, stream=None) -> None:
    """The k largest of E logits for each of T tokens, their gates, and the pairs (token, expert) grouped by expert (see
    include/sgap.h).  `workspace`: a CUDA uint8 tensor of sgap_route_topk_workspace_size bytes, None where that is 0."""
    renormalise = int(bool(renormalise))
    st = (_native or _load_native()).route_topk(T, E, k, logits, gates, experts, slot, order, offsets, renormalise, workspace, stream)
    if st == 0:
        return
    if st > 0:
        _check(st)
    import torch

    dtype = _element_type(logits, "logits")
    ptr, ld = _rows(logits, logits.dtype, T, E, "logits")
    ws, ws_bytes = _bytes(workspace, "workspace")
    _check(load().sgap_route_topk(
        T, E, k, dtype, ptr, ld, renormalise, _flat(gates, torch.float32, T * k, "gates"),
        _flat(experts, torch.int32, T * k, "experts"), _flat(slot, torch.int32, T * k, "slot"),
        _flat(order, torch.int32, T * k, "order"), _flat(offsets, torch.int32, E + 1, "offsets"), ws, ws_bytes, _stream_ptr(stream)))


def sgap_route_topk_grad(T, E, k, logits, gates, experts, dgates, dlogits, renormalise=True, stream=None) -> None:
    """dlogits from the gradient of the gates that sgap_route_topk gave (see include/sgap.h)."""
    renormalise = int(bool(renormalise))
    st = (_native or _load_native()).route_topk_grad(T, E, k, logits, gates, experts, dgates, dlogits, renormalise, stream)
    if st == 0:
        return
    if st > 0:
        _check(st)
    import torch

    dtype = _element_type(logits, "logits")
    ptr, ld = _rows(logits, logits.dtype, T, E, "logits")
    dptr, ldd = _rows(dlogits, logits.dtype, T, E, "dlogits")
    _check(load().sgap_route_topk_grad(
        T, E, k, dtype, ptr, ld, renormalise, _flat(gates, torch.float32, T * k, "gates"),
        _flat(experts, torch.int32, T * k, "experts"), _flat(dgates, torch.float32, T * k, "dgates"), dptr, ldd,
        _stream_ptr(stream)))


def sgap_route_combine(T, k, D, Z, slot, gates, out, stream=None) -> None:
    """out[t] = sum over j of gates[t, j] * Z[slot[t, j]]; gates None: all 1 (see include/sgap.h)."""
    st = (_native or _load_native()).route_combine(T, k, D, Z, slot, gates, out, stream)
    if st == 0:
        return
    if st > 0:
        _check(st)
    import torch

    dtype = _element_type(Z, "Z")
    _check(load().sgap_route_combine(
        T, k, D, dtype, _flat(Z, Z.dtype, T * k * D, "Z"), _flat(slot, torch.int32, T * k, "slot"),
        None if gates is None else _flat(gates, torch.float32, T * k, "gates"), _flat(out, Z.dtype, T * D, "out"),
        _stream_ptr(stream)))


def sgap_route_combine_grad(T, k, D, Z, slot, order, gates, dout, dZ, dgates, stream=None) -> None:
    """The gradients of sgap_route_combine (see include/sgap.h)."""
    st = (_native or _load_native()).route_combine_grad(T, k, D, Z, slot, order, gates, dout, dZ, dgates, stream)
    if st == 0:
        return
    if st > 0:
        _check(st)
    import torch

    dtype = _element_type(Z, "Z")
    _check(load().sgap_route_combine_grad(
        T, k, D, dtype, _flat(Z, Z.dtype, T * k * D, "Z"), _flat(slot, torch.int32, T * k, "slot"),
        _flat(order, torch.int32, T * k, "order"), _flat(gates, torch.float32, T * k, "gates"), _flat(dout, Z.dtype, T * D, "dout"),
        _flat(dZ, Z.dtype, T * k * D, "dZ"), _flat(dgates, torch.float32, T * k, "dgates"), _stream_ptr(stream)))


def _grouped_args(G, R, K, offsets, X, src, src_div):
    """(offsets, X, ldx, rows of X, src, src_div) of a product over groups."""
    import torch

    off = None if offsets is None else _flat(offsets, torch.int32, G + 1, "offsets")
    ptr, ld = _rows(X, X.dtype, None, K, "X")
    return off, ptr, ld, X.shape[0], None if src is None else _flat(src, torch.int32, R, "src"), int(src_div)


def sgap_grouped_mm(G, R, K, N, offsets, X, W, Y, layout="nk", src=None, src_div=1, stream=None) -> None:
    """Y[r] = X[src[r] // src_div] * op(W[g]) for the rows r of each group g; `layout` "nk" (W[g] is N x K) or "kn" (see
    include/sgap.h).  offsets None: one group of all rows; src None: row r takes row r."""
    layout = WEIGHT_LAYOUTS.get(layout, layout)
    st = (_native or _load_native()).grouped_mm(G, R, K, N, offsets, X, W, Y, layout, src, src_div, stream)
    if st == 0:
        return
    if st > 0:
        _check(st)
    dtype = _element_type(X, "X")
    args = _grouped_args(G, R, K, offsets, X, src, src_div)
    w = _flat(W, X.dtype, G * K * N, "W")
    y, ldy = _rows(Y, X.dtype, R, N, "Y")
    _check(load().sgap_grouped_mm(G, R, K, N, dtype, *args, w, int(layout), y, ldy, _stream_ptr(stream)))


def sgap_grouped_mm_wgrad(G, R, K, N, offsets, X, dY, dW, layout="nk", src=None, src_div=1, stream=None) -> None:
    """The gradient of sgap_grouped_mm's weights (see include/sgap.h)."""
    layout = WEIGHT_LAYOUTS.get(layout, layout)
    st = (_native or _load_native()).grouped_mm_wgrad(G, R, K, N, offsets, X, dY, dW, layout, src, src_div, stream)
    if st == 0:
        return
    if st > 0:
        _check(st)
    dtype = _element_type(X, "X")
    args = _grouped_args(G, R, K, offsets, X, src, src_div)
    d, ldd = _rows(dY, X.dtype, R, N, "dY")
    w = _flat(dW, X.dtype, G * K * N, "dW")
    _check(load().sgap_grouped_mm_wgrad(G, R, K, N, dtype, *args, d, ldd, w, int(layout), _stream_ptr(stream)))


def sgap_w4_layout_size(G, K, N, group_k, zeros=False) -> int:
    size = load().sgap_w4_layout_size(int(G), int(K), int(N), int(group_k), int(bool(zeros)))
    if size < 0:
        raise SgapError(SGAP_ERR_INVALID_ARG, load().sgap_last_error().decode())
    return size


def sgap_w4_layout(G, K, N, group_k, codes, scales, zeros, weights, stream=None) -> None:
    """4-bit weights as sgap_grouped_mm_w4 reads them, into the CUDA uint8 tensor `weights` of sgap_w4_layout_size bytes: codes
    G x N x K/2 (uint8), scales G x N x K/group_k (float16 or bfloat16), zeros the same in uint8 or None for 8."""
    import torch

    if _element_type(scales, "scales") == SGAP_F32:
        raise TypeError("scales must be float16 or bfloat16")
    blocks = K // max(int(group_k), 1)
    ws, ws_bytes = _bytes(weights, "weights")
    _check(load().sgap_w4_layout(
        G, K, N, int(group_k), _flat(codes, torch.uint8, G * N * (K // 2), "codes"), _flat(scales, scales.dtype, G * N * blocks, "scales"),
        None if zeros is None else _flat(zeros, torch.uint8, G * N * blocks, "zeros"), ws, ws_bytes, _stream_ptr(stream)))


def sgap_grouped_mm_w4(G, R, K, N, group_k, offsets, X, weights, Y, zeros=False, src=None, src_div=1, stream=None) -> None:
    """sgap_grouped_mm with the weights that sgap_w4_layout left in `weights`; `zeros`: whether there were zero points.  X and Y
    have the scales' type (see include/sgap.h)."""
    zeros = int(bool(zeros))
    st = (_native or _load_native()).grouped_mm_w4(G, R, K, N, group_k, offsets, X, weights, Y, zeros, src, src_div, stream)
    if st == 0:
        return
    if st > 0:
        _check(st)
    dtype = _element_type(X, "X")
    args = _grouped_args(G, R, K, offsets, X, src, src_div)
    ws, ws_bytes = _bytes(weights, "weights")
    y, ldy = _rows(Y, X.dtype, R, N, "Y")
    _check(load().sgap_grouped_mm_w4(G, R, K, N, dtype, int(group_k), zeros, *args, ws, ws_bytes, y, ldy, _stream_ptr(stream)))


def sgap_route_balance_workspace_size(T, E, k, S) -> int:
    size = load().sgap_route_balance_workspace_size(int(T), int(E), int(k), int(S))
    if size < 0:
        raise SgapError(SGAP_ERR_INVALID_ARG, load().sgap_last_error().decode())
    return size


def sgap_route_balance(T, E, k, S, logits, experts, segments, loss, counts, rows, workspace=None, stream=None) -> None:
    """The balance loss over S sequences of tokens (segments None: one of all), each expert's pairs and the tokens that chose, from
    a router's logits and choice (see include/sgap.h).  `workspace`: a CUDA uint8 tensor of sgap_route_balance_workspace_size bytes."""
    st = (_native or _load_native()).route_balance(T, E, k, S, logits, experts, segments, loss, counts, rows, workspace, stream)
    if st == 0:
        return
    if st > 0:
        _check(st)
    import torch

    dtype = _element_type(logits, "logits")
    ptr, ld = _rows(logits, logits.dtype, T, E, "logits")
    ws, ws_bytes = _bytes(workspace, "workspace")
    _check(load().sgap_route_balance(
        T, E, k, S, dtype, ptr, ld, _flat(experts, torch.int32, T * k, "experts"),
        None if segments is None else _flat(segments, torch.int32, S + 1, "segments"), _flat(loss, torch.float32, 1, "loss"),
        _flat(counts, torch.int32, S * E, "counts"), _flat(rows, torch.int32, S, "rows"), ws, ws_bytes, _stream_ptr(stream)))


def sgap_route_balance_grad(T, E, k, S, logits, experts, segments, counts, rows, dloss, dlogits, accumulate=False, stream=None) -> None:
    """dlogits from the gradient of the balance loss, or added to what is there (see include/sgap.h)."""
    accumulate = int(bool(accumulate))
    st = (_native or _load_native()).route_balance_grad(T, E, k, S, logits, experts, segments, counts, rows, dloss, dlogits, accumulate,
                                                        stream)
    if st == 0:
        return
    if st > 0:
        _check(st)
    import torch

    dtype = _element_type(logits, "logits")
    ptr, ld = _rows(logits, logits.dtype, T, E, "logits")
    dptr, ldd = _rows(dlogits, logits.dtype, T, E, "dlogits")
    _check(load().sgap_route_balance_grad(
        T, E, k, S, dtype, ptr, ld, _flat(experts, torch.int32, T * k, "experts"),
        None if segments is None else _flat(segments, torch.int32, S + 1, "segments"), _flat(counts, torch.int32, S * E, "counts"),
        _flat(rows, torch.int32, S, "rows"), _flat(dloss, torch.float32, 1, "dloss"), accumulate, dptr, ldd, _stream_ptr(stream)))


def sgap_embed(T, V, D, ids, weights, out, scale=1.0, stream=None) -> None:
    """out[t] = scale * weights[ids[t]]; an id outside 0 .. V gives zeros (see include/sgap.h)."""
    scale = float(scale)
    st = (_native or _load_native()).embed(T, V, D, ids, weights, out, scale, stream)
    if st == 0:
        return
    if st > 0:
        _check(st)
    import torch

    dtype = _element_type(weights, "weights")
    w, ldw = _rows(weights, weights.dtype, V, D, "weights")
    o, ldo = _rows(out, weights.dtype, T, D, "out")
    _check(load().sgap_embed(T, V, D, dtype, _flat(ids, torch.int32, T, "ids"), w, ldw, scale, o, ldo, _stream_ptr(stream)))


def sgap_embed_grad_workspace_size(T, V, D) -> int:
    size = load().sgap_embed_grad_workspace_size(int(T), int(V), int(D))
    if size < 0:
        raise SgapError(SGAP_ERR_INVALID_ARG, load().sgap_last_error().decode())
    return size


def sgap_embed_grad(T, V, D, ids, dout, dweights, scale=1.0, accumulate=False, workspace=None, stream=None) -> None:
    """dweights[v] = scale * the sum of dout[t] over the tokens with ids[t] = v, or that added to what is there; dweights has
    dout's type or float32 (see include/sgap.h).  `workspace`: a CUDA uint8 tensor of sgap_embed_grad_workspace_size bytes."""
    scale, accumulate = float(scale), int(bool(accumulate))
    st = (_native or _load_native()).embed_grad(T, V, D, ids, dout, dweights, scale, accumulate, workspace, stream)
    if st == 0:
        return
    if st > 0:
        _check(st)
    import torch

    dtype, grad_dtype = _element_type(dout, "dout"), _element_type(dweights, "dweights")
    d, ldd = _rows(dout, dout.dtype, T, D, "dout")
    w, ldw = _rows(dweights, dweights.dtype, V, D, "dweights")
    ws, ws_bytes = _bytes(workspace, "workspace")
    _check(load().sgap_embed_grad(T, V, D, dtype, _flat(ids, torch.int32, T, "ids"), d, ldd, scale, accumulate, grad_dtype, w, ldw, ws,
                                  ws_bytes, _stream_ptr(stream)))


SGAP_F8_BLOCK = 128
SGAP_MAX_SEQUENCES = 65536


def _f8_blocks(n):
    return (n + SGAP_F8_BLOCK - 1) // SGAP_F8_BLOCK


def sgap_f8_rows(R, K, X, codes, scales, stream=None) -> None:
    """The rows of X in 8 bits: codes (torch.float8_e4m3fn, R rows of 128 * ceil(K / 128)) and scales (float32, R x ceil(K / 128))
    (see include/sgap.h)."""
    st = (_native or _load_native()).f8_rows(R, K, X, codes, scales, stream)
    if st == 0:
        return
    if st > 0:
        _check(st)
    import torch

    dtype = _element_type(X, "X")
    ptr, ld = _rows(X, X.dtype, R, K, "X")
    blocks = _f8_blocks(K)
    _check(load().sgap_f8_rows(R, K, dtype, ptr, ld, _flat(codes, torch.float8_e4m3fn, R * blocks * SGAP_F8_BLOCK, "codes"),
                               _flat(scales, torch.float32, R * blocks, "scales"), _stream_ptr(stream)))


def sgap_f8_weights(G, K, N, W, codes, scales, codes_t=None, scales_t=None, stream=None) -> None:
    """Weights G x N x K in 8 bits: codes (torch.float8_e4m3fn, G x N rows of 128 * ceil(K / 128)), scales (float32, G x ceil(N /
    128) x ceil(K / 128)), and, if they are given, the same of the transposed matrices (see include/sgap.h)."""
    st = (_native or _load_native()).f8_weights(G, K, N, W, codes, scales, codes_t, scales_t, stream)
    if st == 0:
        return
    if st > 0:
        _check(st)
    import torch

    dtype = _element_type(W, "W")
    nb, kb = _f8_blocks(N), _f8_blocks(K)
    _check(load().sgap_f8_weights(
        G, K, N, dtype, _flat(W, W.dtype, G * N * K, "W"), _flat(codes, torch.float8_e4m3fn, G * N * kb * SGAP_F8_BLOCK, "codes"),
        _flat(scales, torch.float32, G * nb * kb, "scales"),
        None if codes_t is None else _flat(codes_t, torch.float8_e4m3fn, G * K * nb * SGAP_F8_BLOCK, "codes_t"),
        None if scales_t is None else _flat(scales_t, torch.float32, G * nb * kb, "scales_t"), _stream_ptr(stream)))


def sgap_grouped_mm_f8(G, R, K, N, offsets, X, x_scales, W, w_scales, Y, src=None, src_div=1, stream=None) -> None:
    """sgap_grouped_mm with rows and weights (G x N x K) in 8 bits, as sgap_f8_rows and sgap_f8_weights put them; Y is float32,
    float16 or bfloat16 (see include/sgap.h)."""
    st = (_native or _load_native()).grouped_mm_f8(G, R, K, N, offsets, X, x_scales, W, w_scales, Y, src, src_div, stream)
    if st == 0:
        return
    if st > 0:
        _check(st)
    import torch

    dtype = _element_type(Y, "Y")
    nb, kb = _f8_blocks(N), _f8_blocks(K)
    if not isinstance(X, torch.Tensor) or X.dim() != 2:
        raise ValueError("X must be a matrix of codes")
    x_rows = X.shape[0]
    y, ldy = _rows(Y, Y.dtype, R, N, "Y")
    _check(load().sgap_grouped_mm_f8(
        G, R, K, N, dtype, None if offsets is None else _flat(offsets, torch.int32, G + 1, "offsets"),
        _flat(X, torch.float8_e4m3fn, x_rows * kb * SGAP_F8_BLOCK, "X"), _flat(x_scales, torch.float32, x_rows * kb, "x_scales"), x_rows,
        None if src is None else _flat(src, torch.int32, R, "src"), int(src_div),
        _flat(W, torch.float8_e4m3fn, G * N * kb * SGAP_F8_BLOCK, "W"), _flat(w_scales, torch.float32, G * nb * kb, "w_scales"), y, ldy,
        _stream_ptr(stream)))
