"""ctypes binding of libtilefusion.so: same entry points as include/tilefusion.h.

Argument marshalling only.  Device operands are passed as objects with a `data_ptr()` method
(torch tensors) or as integer device addresses.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional

import numpy as np

TF_F32, TF_F64, TF_BF16, TF_F16 = 0, 1, 2, 3
TF_FLAG_NO_SPLIT = 1
TF_FLAG_SCHEDULE_ONLY = 2
TF_FLAG_REORDER = 4
TF_FLAG_C_TRANSPOSED = 8
TF_FLAG_SKIP_UNREAD = 16
TF_FLAG_NO_BASELINE = 32
TF_EXECUTE_WAVEFRONTS, TF_EXECUTE_ONE_PASS, TF_EXECUTE_GATHER_FIRST, TF_EXECUTE_PLAIN_PAIR = 0, 1, 2, 3

TF_Q4_INT, TF_Q4_E2M1 = 0, 1
TF_ROUTE_SOFTMAX, TF_ROUTE_SOFTMAX_TOP, TF_ROUTE_SIGMOID, TF_ROUTE_SIGMOID_TOP = 0, 1, 2, 3
TF_ACT_IDENTITY, TF_ACT_RELU, TF_ACT_SILU, TF_ACT_GELU = 0, 1, 2, 3

_STATUS = {0: "TF_OK", 1: "TF_EINVAL", 2: "TF_EBADCSR", 3: "TF_ENOMEM", 4: "TF_EHIP",
           5: "TF_EUNSUPPORTED", 6: "TF_EMISMATCH"}

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "libtilefusion.so")
_lib = None


class TfError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"{_STATUS.get(status, status)}: {message}")
        self.status = status
        self.status_name = _STATUS.get(status, str(status))


class tf_csr(ctypes.Structure):
    _fields_ = [("n_rows", ctypes.c_int64), ("n_cols", ctypes.c_int64), ("nnz", ctypes.c_int64),
                ("rowptr", ctypes.c_void_p), ("colidx", ctypes.c_void_p),
                ("vals", ctypes.c_void_p), ("dtype", ctypes.c_int32),
                ("on_device", ctypes.c_int32)]


class tf_tile_params(ctypes.Structure):
    _fields_ = [("ct_size", ctypes.c_int32), ("p", ctypes.c_int32),
                ("fast_mem_bytes", ctypes.c_int64), ("col_slice", ctypes.c_int32),
                ("flags", ctypes.c_uint32), ("gather_slices", ctypes.c_int32),
                ("reserved0", ctypes.c_int32)]


class tf_schedule_view(ctypes.Structure):
    _fields_ = [("n", ctypes.c_int64), ("nnz", ctypes.c_int64), ("t", ctypes.c_int32),
                ("col_slice", ctypes.c_int32), ("n_slices", ctypes.c_int32),
                ("dtype", ctypes.c_int32), ("b_is_sparse", ctypes.c_int32),
                ("execution", ctypes.c_int32),
                ("n_coarse_tiles", ctypes.c_int64), ("n_tiles", ctypes.c_int64),
                ("tile_first_ptr", ctypes.POINTER(ctypes.c_int32)),
                ("first_rows", ctypes.POINTER(ctypes.c_int32)),
                ("tile_second_ptr", ctypes.POINTER(ctypes.c_int32)),
                ("second_rows", ctypes.POINTER(ctypes.c_int32)),
                ("n_wf1_units", ctypes.c_int64),
                ("wf1_unit_ptr", ctypes.POINTER(ctypes.c_int32)),
                ("wf1_rows", ctypes.POINTER(ctypes.c_int32)),
                ("spill", ctypes.POINTER(ctypes.c_uint8)),
                ("n_fused_rows", ctypes.c_int64), ("n_wf1_rows", ctypes.c_int64),
                ("n_spill_rows", ctypes.c_int64), ("fused_nnz", ctypes.c_int64),
                ("fused_ratio_eq3", ctypes.c_double), ("fused_ratio_rows", ctypes.c_double),
                ("fused_ratio_nnz", ctypes.c_double),
                ("fast_mem_bytes", ctypes.c_int64), ("lds_fixed_bytes", ctypes.c_int64),
                ("lds_bytes_per_row", ctypes.c_int64), ("lds_row_granule", ctypes.c_int32),
                ("second_block_in_lds", ctypes.c_int32),
                ("eq2_cost_max", ctypes.c_double), ("plan_seconds", ctypes.c_double),
                ("alg_bytes", ctypes.c_int64), ("alg_bytes_unfused", ctypes.c_int64),
                ("second_block_bytes", ctypes.c_int64), ("lds_launch_bytes", ctypes.c_int64),
                ("n_first_rows", ctypes.c_int64),
                ("spill_slot", ctypes.POINTER(ctypes.c_int32)), ("n_direct_rows", ctypes.c_int64),
                ("d1_slices", ctypes.c_int32), ("d1_slice_cols", ctypes.c_int32),
                ("d1_rows", ctypes.c_int64), ("first_wavefront_streams", ctypes.c_int32),
                ("grown_tiles", ctypes.c_int32), ("n_demoted_rows", ctypes.c_int64),
                ("far_rows", ctypes.c_int32), ("automatic", ctypes.c_int32)]


class tf_q4(ctypes.Structure):
    _fields_ = [("n_mats", ctypes.c_int64), ("n_rows", ctypes.c_int64), ("n_cols", ctypes.c_int64),
                ("codes", ctypes.c_void_p), ("scales", ctypes.c_void_p),
                ("kind", ctypes.c_int32), ("group", ctypes.c_int32)]


class tf_moe_desc(ctypes.Structure):
    _fields_ = [("n_experts", ctypes.c_int64), ("n_in", ctypes.c_int64), ("n_hidden", ctypes.c_int64),
                ("n_out", ctypes.c_int64), ("max_tokens", ctypes.c_int64),
                ("max_entries", ctypes.c_int64), ("dtype", ctypes.c_int32),
                ("activation", ctypes.c_int32), ("gated", ctypes.c_int32),
                ("reserved0", ctypes.c_int32)]


class tf_xent_desc(ctypes.Structure):
    _fields_ = [("n_classes", ctypes.c_int64), ("n_in", ctypes.c_int64), ("max_rows", ctypes.c_int64),
                ("dtype", ctypes.c_int32), ("gradients", ctypes.c_int32)]


EXPORTS = ["tf_plan_create", "tf_plan_destroy", "tf_plan_schedule", "tf_plan_workspace",
           "tf_gemm_spmm", "tf_gemm_spmm_static", "tf_spmm_spmm", "tf_unfused_gemm_spmm",
           "tf_unfused_spmm_spmm", "tf_run_wavefront", "tf_plan_prepare_unfused", "tf_plan_workspace_unfused",
           "tf_csr_validate", "tf_q4_sizes", "tf_q4_pack", "tf_q4_quantize", "tf_q4_unpack", "tf_q4_matvec",
           "tf_moe_route", "tf_moe_create", "tf_moe_destroy", "tf_moe_layer", "tf_moe_layer_q4",
           "tf_moe_balance_size", "tf_moe_balance", "tf_moe_route_grad", "tf_xent_size", "tf_xent_create", "tf_xent_destroy",
           "tf_xent_device", "tf_xent_loss", "tf_xent_grad", "tf_xent_grad_by_loss",
           "tf_last_error", "tf_version"]
_INT_RETURNS = [e for e in EXPORTS if e not in ("tf_last_error", "tf_version")]


def library_path() -> str:
    return _LIB_PATH


def load_library():
    """Loads libtilefusion.so.  There is no fallback: a missing library is an error."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(_LIB_PATH):
        raise ImportError(f"{_LIB_PATH} is not built; run `python -m paper_2407_00243_amd.build` "
                          f"(or __graft_entry__.build())")
    lib = ctypes.CDLL(_LIB_PATH)
    vp, i32, i64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64
    lib.tf_plan_create.argtypes = [ctypes.POINTER(tf_csr), i64, i64, i32,
                                   ctypes.POINTER(tf_tile_params), ctypes.POINTER(vp)]
    lib.tf_plan_destroy.argtypes = [vp]
    lib.tf_plan_schedule.argtypes = [vp, ctypes.POINTER(tf_schedule_view)]
    lib.tf_plan_workspace.argtypes = [vp, ctypes.POINTER(vp)]
    lib.tf_gemm_spmm.argtypes = [vp, vp, vp, vp, vp]
    lib.tf_unfused_gemm_spmm.argtypes = [vp, vp, vp, vp, vp]
    lib.tf_gemm_spmm_static.argtypes = [vp, vp, vp, vp, vp]
    lib.tf_spmm_spmm.argtypes = [vp, ctypes.POINTER(tf_csr), vp, vp, vp]
    lib.tf_unfused_spmm_spmm.argtypes = [vp, ctypes.POINTER(tf_csr), vp, vp, vp]
    lib.tf_run_wavefront.argtypes = [vp, i32, vp, ctypes.POINTER(tf_csr), vp, vp, vp]
    lib.tf_plan_prepare_unfused.argtypes = [vp]
    lib.tf_plan_workspace_unfused.argtypes = [vp, ctypes.POINTER(vp)]
    lib.tf_csr_validate.argtypes = [ctypes.POINTER(tf_csr)]
    q4 = ctypes.POINTER(tf_q4)
    csr = ctypes.POINTER(tf_csr)
    lib.tf_q4_sizes.argtypes = [q4, ctypes.POINTER(i64), ctypes.POINTER(i64)]
    lib.tf_q4_pack.argtypes = [q4, vp, vp, vp]
    lib.tf_q4_quantize.argtypes = [q4, vp, i32, vp]
    lib.tf_q4_unpack.argtypes = [q4, i32, vp, vp]
    lib.tf_q4_matvec.argtypes = [q4, vp, i64, vp, i64, i64, i32, vp]
    lib.tf_moe_route.argtypes = [vp, i64, i32, vp, i32, ctypes.c_float, csr, vp]
    lib.tf_moe_create.argtypes = [ctypes.POINTER(tf_moe_desc), ctypes.POINTER(vp)]
    lib.tf_moe_destroy.argtypes = [vp]
    lib.tf_moe_layer.argtypes = [vp, csr, vp, i64, vp, vp, vp, i64, vp]
    lib.tf_moe_layer_q4.argtypes = [vp, csr, vp, i64, q4, q4, vp, i64, vp]
    lib.tf_moe_balance_size.argtypes = [i64, i64, ctypes.POINTER(i64)]
    lib.tf_moe_balance.argtypes = [vp, i64, i32, i32, csr, vp, vp, vp, vp, vp]
    lib.tf_moe_route_grad.argtypes = [vp, i64, i32, i32, ctypes.c_float, csr, vp, vp, vp, vp, i64, vp]
    lib.tf_xent_size.argtypes = [ctypes.POINTER(tf_xent_desc), ctypes.POINTER(i64)]
    lib.tf_xent_create.argtypes = [ctypes.POINTER(tf_xent_desc), ctypes.POINTER(vp)]
    lib.tf_xent_destroy.argtypes = [vp]
    lib.tf_xent_device.argtypes = [vp, ctypes.POINTER(i32)]
    lib.tf_xent_loss.argtypes = [vp, vp, i64, vp, i64, vp, i64, vp, vp, vp]
    lib.tf_xent_grad.argtypes = [vp, vp, i64, vp, i64, vp, vp, vp, i64, vp, i64, vp, i64, vp]
    lib.tf_xent_grad_by_loss.argtypes = [vp, vp, i64, vp, i64, vp, vp, vp, vp, i64, vp, i64, vp, i64, vp]
    for name in _INT_RETURNS:
        getattr(lib, name).restype = ctypes.c_int
    lib.tf_last_error.restype = ctypes.c_char_p
    lib.tf_version.restype = ctypes.c_char_p
    _lib = lib
    return lib


def tf_last_error() -> str:
    return load_library().tf_last_error().decode()


def tf_version() -> str:
    return load_library().tf_version().decode()


def _check(status: int):
    if status != 0:
        raise TfError(status, tf_last_error())


def _addr(x) -> Optional[int]:
    if x is None:
        return None
    if isinstance(x, int):
        return x
    if isinstance(x, np.ndarray):
        return x.ctypes.data
    return int(x.data_ptr())


def _dtype_code(dt) -> int:
    s = str(dt)
    if s.endswith("float32"):
        return TF_F32
    if s.endswith("float64"):
        return TF_F64
    raise TypeError(f"unsupported element type {dt}")


class DeviceCsr:
    """A CSR matrix whose three arrays are device tensors (kept alive by this object)."""

    def __init__(self, n_rows: int, n_cols: int, rowptr, colidx, vals):
        self.n_rows, self.n_cols = int(n_rows), int(n_cols)
        self.rowptr, self.colidx, self.vals = rowptr, colidx, vals
        self.nnz = int(colidx.numel())

    def as_struct(self) -> tf_csr:
        return tf_csr(self.n_rows, self.n_cols, self.nnz, _addr(self.rowptr), _addr(self.colidx),
                      _addr(self.vals), _dtype_code(self.vals.dtype), 1)


def _host_csr_struct(A, keep: list) -> tf_csr:
    rowptr = np.ascontiguousarray(A.rowptr, dtype=np.int32)
    colidx = np.ascontiguousarray(A.colidx, dtype=np.int32)
    vals = np.ascontiguousarray(A.vals)
    keep.extend([rowptr, colidx, vals])
    return tf_csr(int(A.n_rows), int(A.n_cols), int(colidx.size), rowptr.ctypes.data,
                  colidx.ctypes.data if colidx.size else None,
                  vals.ctypes.data if vals.size else None, _dtype_code(vals.dtype), 0)


def tf_plan_create(A, bcol: int, ccol: int, b_is_sparse: bool, ct_size: int = 0, p: int = 0,
                   fast_mem_bytes: int = 0, col_slice: int = 0, flags: int = 0,
                   gather_slices: int = 0) -> int:
    """A: host CSR (anything with n_rows, n_cols, rowptr, colidx, vals as numpy arrays), a
    DeviceCsr, or a ready tf_csr struct.  Returns the opaque plan handle."""
    lib = load_library()
    keep: list = []
    if isinstance(A, tf_csr):
        a = A
    elif isinstance(A, DeviceCsr):
        a = A.as_struct()
    else:
        a = _host_csr_struct(A, keep)
    tp = tf_tile_params(ct_size, p, fast_mem_bytes, col_slice, flags, gather_slices, 0)
    out = ctypes.c_void_p()
    _check(lib.tf_plan_create(ctypes.byref(a), bcol, ccol, 1 if b_is_sparse else 0,
                              ctypes.byref(tp), ctypes.byref(out)))
    return out.value


def tf_plan_destroy(plan: Optional[int]) -> None:
    _check(load_library().tf_plan_destroy(plan))


def _np_copy(ptr, count: int, dtype) -> np.ndarray:
    if count == 0:
        return np.zeros(0, dtype=dtype)
    return np.ctypeslib.as_array(ptr, shape=(count,)).astype(dtype, copy=True)


def tf_plan_schedule(plan: int) -> dict:
    """Host copy of the plan's schedule: arrays as numpy, counters as Python numbers."""
    v = tf_schedule_view()
    _check(load_library().tf_plan_schedule(plan, ctypes.byref(v)))
    out = {name: getattr(v, name) for name, _ in tf_schedule_view._fields_
           if not name.startswith("reserved")}
    nt, nu = v.n_tiles, v.n_wf1_units
    out["tile_first_ptr"] = _np_copy(v.tile_first_ptr, nt + 1, np.int32)
    out["first_rows"] = _np_copy(v.first_rows, v.n_first_rows, np.int32)
    out["tile_second_ptr"] = _np_copy(v.tile_second_ptr, nt + 1, np.int32)
    out["second_rows"] = _np_copy(v.second_rows, v.n_fused_rows, np.int32)
    out["wf1_unit_ptr"] = _np_copy(v.wf1_unit_ptr, nu + 1, np.int32)
    out["wf1_rows"] = _np_copy(v.wf1_rows, v.n_wf1_rows, np.int32)
    out["spill"] = _np_copy(v.spill, v.n, np.uint8)
    out["spill_slot"] = _np_copy(v.spill_slot, v.n, np.int32)
    return out


def tf_plan_workspace(plan: int) -> int:
    out = ctypes.c_void_p()
    _check(load_library().tf_plan_workspace(plan, ctypes.byref(out)))
    return out.value or 0


def tf_plan_workspace_unfused(plan: int) -> int:
    out = ctypes.c_void_p()
    _check(load_library().tf_plan_workspace_unfused(plan, ctypes.byref(out)))
    return out.value or 0


def tf_plan_prepare_unfused(plan: int) -> None:
    _check(load_library().tf_plan_prepare_unfused(plan))


def tf_csr_validate(M) -> None:
    """M: host CSR (numpy arrays), a DeviceCsr or a tf_csr struct; raises TfError if malformed."""
    keep: list = []
    m = M if isinstance(M, tf_csr) else (M.as_struct() if isinstance(M, DeviceCsr)
                                         else _host_csr_struct(M, keep))
    _check(load_library().tf_csr_validate(ctypes.byref(m)))


def tf_gemm_spmm(plan: int, B, C, D, stream=None) -> None:
    _check(load_library().tf_gemm_spmm(plan, _addr(B), _addr(C), _addr(D), _addr(stream)))


def tf_gemm_spmm_static(plan: int, B, C, D, stream=None) -> None:
    _check(load_library().tf_gemm_spmm_static(plan, _addr(B), _addr(C), _addr(D), _addr(stream)))


def tf_unfused_gemm_spmm(plan: int, B, C, D, stream=None) -> None:
    _check(load_library().tf_unfused_gemm_spmm(plan, _addr(B), _addr(C), _addr(D),
                                               _addr(stream)))


def _csr_arg(B) -> tf_csr:
    return B if isinstance(B, tf_csr) else B.as_struct()


def tf_spmm_spmm(plan: int, B, C, D, stream=None) -> None:
    b = _csr_arg(B)
    _check(load_library().tf_spmm_spmm(plan, ctypes.byref(b), _addr(C), _addr(D), _addr(stream)))


def tf_unfused_spmm_spmm(plan: int, B, C, D, stream=None) -> None:
    b = _csr_arg(B)
    _check(load_library().tf_unfused_spmm_spmm(plan, ctypes.byref(b), _addr(C), _addr(D),
                                               _addr(stream)))


def tf_run_wavefront(plan: int, wavefront: int, B, C, D, stream=None) -> None:
    """B: dense device operand, DeviceCsr / tf_csr, or None (wavefront 1 only)."""
    lib = load_library()
    if B is None or hasattr(B, "data_ptr") or isinstance(B, int):
        _check(lib.tf_run_wavefront(plan, wavefront, _addr(B), None, _addr(C), _addr(D),
                                    _addr(stream)))
    else:
        b = _csr_arg(B)
        _check(lib.tf_run_wavefront(plan, wavefront, None, ctypes.byref(b), _addr(C), _addr(D),
                                    _addr(stream)))


# ------------------------------------------------------------------------------- routed operators

_ROUTED = {"torch.float32": TF_F32, "float32": TF_F32, "torch.bfloat16": TF_BF16,
           "torch.float16": TF_F16, "float16": TF_F16}
_codes: dict = {}          # of element types that have been seen, by the type itself
_csr_types: set = set()     # the types of a routing matrix's arrays that have been seen and are right, by the types themselves


def _routed_code(dt) -> int:
    code = _codes.get(dt)
    if code is None:
        code = dt if isinstance(dt, int) else _ROUTED.get(str(dt))
        if code is None:
            raise TypeError(f"unsupported element type {dt}")
        _codes[dt] = code
    return code


def _matrix(x, what: str, cols: Optional[int] = None):
    """Rows, columns and distance of the rows (in elements) of a matrix whose rows are contiguous."""
    shape = x.shape
    if len(shape) != 2:
        raise ValueError(f"{what} must be a matrix")
    rows, n = shape
    if cols is not None and n != cols:
        raise ValueError(f"{what} must have {cols} columns, not {n}")
    ld, step = x.stride()
    if step != 1 and n > 1:
        raise ValueError(f"the rows of {what} must be contiguous")
    return rows, n, ld if rows > 1 else max(ld, n)


def _routing(A, device: int) -> tf_csr:
    """A routing matrix as the library takes it: indices of 32 bits, values in fp32, arrays on `device` that hold all of them.
    (A tf_csr is the caller's affair.)"""
    if isinstance(A, tf_csr):
        return A
    rowptr, colidx, vals, n_rows, nnz = A.rowptr, A.colidx, A.vals, A.n_rows, A.nnz
    types = rowptr.dtype, colidx.dtype, vals.dtype
    if types not in _csr_types:
        if [str(t) for t in types[:2]] != ["torch.int32"] * 2:
            raise TypeError("rowptr and colidx of A must be int32")
        if _routed_code(types[2]) != TF_F32:
            raise TypeError("the values of A must be fp32")
        _csr_types.add(types)
    if rowptr.numel() <= n_rows or colidx.numel() < nnz or vals.numel() < nnz:
        raise ValueError(f"the arrays of A must hold {n_rows + 1} row pointers and {nnz} columns and values")
    if not (rowptr.is_contiguous() and colidx.is_contiguous() and vals.is_contiguous()):
        raise ValueError("the arrays of A must be contiguous")
    if device < 0 or rowptr.get_device() != device or colidx.get_device() != device or vals.get_device() != device:
        _refuse_devices()
    return tf_csr(n_rows, A.n_cols, nnz, rowptr.data_ptr(), colidx.data_ptr(), vals.data_ptr(), TF_F32, 1)


def _refuse_devices():
    raise ValueError("all operands must be on one device, and not on the host")


def _device_of(W, device):
    """Number of the device of a Q4Matrix or an array, -1 for the host; for addresses, which are the caller's affair, `device`."""
    if isinstance(W, Q4Matrix):
        return device if W.device is None else W.device
    if isinstance(W, np.ndarray):
        return -1
    return W.get_device() if hasattr(W, "get_device") else device


def _contiguous(x, what: str, shape, dtype: Optional[int] = None):
    if tuple(x.shape) != tuple(shape):
        raise ValueError(f"{what} must have the shape {tuple(shape)}, not {tuple(x.shape)}")
    if not x.is_contiguous():
        raise ValueError(f"{what} must be contiguous")
    if dtype is not None and _routed_code(x.dtype) != dtype:
        raise TypeError(f"{what} has another element type than the call")


class Q4Matrix:
    """Stacked matrices with weights of 4 bits in device arrays of the caller's (kept alive by this object), of
    the sizes that tf_q4_sizes tells."""

    def __init__(self, n_rows: int, n_cols: int, kind: int, group: int, codes, scales, n_mats: int = 1):
        self.n_mats, self.n_rows, self.n_cols = int(n_mats), int(n_rows), int(n_cols)
        self.kind, self.group = int(kind), int(group)
        self.codes, self.scales = codes, scales
        need = tf_q4_sizes(n_rows, n_cols, kind, group, n_mats)
        for what, x, n in (("codes", codes, need[0]), ("scales", scales, need[1])):
            if hasattr(x, "numel") and (x.numel() * x.element_size() < n or not x.is_contiguous()):
                raise ValueError(f"{what} must hold {n} contiguous bytes")
        # number of their device, -1 for the host; None where both are addresses
        devices = {_device_of(x, None) for x in (codes, scales)} - {None}
        if len(devices) > 1:
            raise ValueError("codes and scales must be on one device")
        self.device = devices.pop() if devices else None
        self.struct = tf_q4(self.n_mats, self.n_rows, self.n_cols, _addr(codes), _addr(scales), self.kind,
                            self.group)
        self.ref = ctypes.byref(self.struct)


def tf_q4_sizes(n_rows: int, n_cols: int, kind: int, group: int, n_mats: int = 1):
    """Bytes of the codes and of the scales of n_mats matrices."""
    w = tf_q4(n_mats, n_rows, n_cols, None, None, kind, group)
    codes, scales = ctypes.c_int64(), ctypes.c_int64()
    _check(load_library().tf_q4_sizes(ctypes.byref(w), ctypes.byref(codes), ctypes.byref(scales)))
    return codes.value, scales.value


def tf_q4_pack(W: Q4Matrix, codes, scales, stream=None) -> None:
    """codes: int8, n_mats x n_rows x n_cols; scales: bf16, n_mats x n_rows x groups."""
    for what, x, n, t in (("codes", codes, W.n_cols, "torch.int8"),
                          ("scales", scales, -(-W.n_cols // W.group), "torch.bfloat16")):
        if hasattr(x, "is_contiguous"):
            _contiguous(x, what, (W.n_mats, W.n_rows, n))
            if str(x.dtype) != t:
                raise TypeError(f"{what} must be {t}")
    device = _device_of(W, 0)
    if device < 0 or _device_of(codes, device) != device or _device_of(scales, device) != device:
        _refuse_devices()
    _check(load_library().tf_q4_pack(ctypes.byref(W.struct), _addr(codes), _addr(scales), _addr(stream)))


def tf_q4_quantize(W: Q4Matrix, weights, stream=None) -> None:
    _contiguous(weights, "weights", (W.n_mats, W.n_rows, W.n_cols))
    device = weights.get_device()
    if device < 0 or _device_of(W, device) != device:
        _refuse_devices()
    _check(load_library().tf_q4_quantize(ctypes.byref(W.struct), _addr(weights), _routed_code(weights.dtype),
                                         _addr(stream)))


def tf_q4_unpack(W: Q4Matrix, weights, stream=None) -> None:
    _contiguous(weights, "weights", (W.n_mats, W.n_rows, W.n_cols))
    device = weights.get_device()
    if device < 0 or _device_of(W, device) != device:
        _refuse_devices()
    _check(load_library().tf_q4_unpack(ctypes.byref(W.struct), _routed_code(weights.dtype), _addr(weights),
                                       _addr(stream)))


def tf_q4_matvec(W: Q4Matrix, X, Y, stream=None) -> None:
    """Y = X W^T; X and Y are matrices of one element type, their rows may be further apart than they are wide."""
    m, _, ldx = _matrix(X, "X", W.n_cols)
    my, _, ldy = _matrix(Y, "Y", W.n_rows)
    if m != my:
        raise ValueError("X and Y must have the same number of rows")
    if X.dtype != Y.dtype:
        raise TypeError("X and Y must have the same element type")
    device = X.get_device()
    if device < 0 or Y.get_device() != device or (W.device != device and W.device is not None):
        _refuse_devices()
    status = load_library().tf_q4_matvec(W.ref, X.data_ptr(), ldx, Y.data_ptr(), ldy, m, _routed_code(X.dtype), stream)
    if status:
        _check(status)


def tf_moe_route(scores, A: DeviceCsr, scoring: int = TF_ROUTE_SOFTMAX_TOP, bias=None, scale: float = 1.0,
                 stream=None) -> None:
    """Writes the arrays of A (rowptr, colidx, vals): the nnz / n_rows best experts of each token."""
    rows, _, ld = _matrix(scores, "scores", A.n_cols)
    if rows != A.n_rows:
        raise ValueError("A must have a row for each row of the scores")
    if bias is not None and hasattr(bias, "shape"):
        _contiguous(bias, "bias", (A.n_cols,), TF_F32)
    device = scores.get_device()
    a = _routing(A, device)
    if bias is not None and _device_of(bias, device) != device:
        _refuse_devices()
    status = load_library().tf_moe_route(scores.data_ptr(), ld, _routed_code(scores.dtype), _addr(bias), scoring, scale,
                                         ctypes.byref(a), stream)
    if status:
        _check(status)


def tf_moe_create(n_experts: int, n_in: int, n_hidden: int, n_out: int, dtype, max_tokens: int,
                  max_entries: int, activation: int = TF_ACT_SILU, gated: bool = True) -> int:
    """Returns the opaque handle of a plan for mixture-of-experts layers of these sizes."""
    d = tf_moe_desc(n_experts, n_in, n_hidden, n_out, max_tokens, max_entries, _routed_code(dtype), activation,
                    1 if gated else 0, 0)
    out = ctypes.c_void_p()
    _check(load_library().tf_moe_create(ctypes.byref(d), ctypes.byref(out)))
    return out.value


def tf_moe_destroy(plan: Optional[int]) -> None:
    _check(load_library().tf_moe_destroy(plan))


def _layer_operands(A, X, D, *weights):
    """The routing matrix and the distances of the rows of X and D."""
    rows, _, ldx = _matrix(X, "X")
    rows_d, _, ldd = _matrix(D, "D")
    if rows != A.n_rows or rows_d != rows:
        raise ValueError("X and D must have a row for each row of A")
    if X.dtype != D.dtype:
        raise TypeError("X and D must have the same element type")
    device = X.get_device()
    a = _routing(A, device)
    if device < 0 or D.get_device() != device or any(_device_of(w, device) != device for w in weights):
        _refuse_devices()
    return a, ldx, ldd


def tf_moe_layer(plan: int, A: DeviceCsr, X, W1, W2, D, stream=None) -> None:
    """The caller answers for what a handle does not tell: columns, element type and weights are to be the plan's (MoePlan looks)."""
    a, ldx, ldd = _layer_operands(A, X, D, W1, W2)
    _check(load_library().tf_moe_layer(plan, ctypes.byref(a), X.data_ptr(), ldx, W1.data_ptr(), W2.data_ptr(), D.data_ptr(), ldd, stream))


def tf_moe_layer_q4(plan: int, A: DeviceCsr, X, W1: Q4Matrix, W2: Q4Matrix, D, stream=None) -> None:
    a, ldx, ldd = _layer_operands(A, X, D, W1, W2)
    _check(load_library().tf_moe_layer_q4(plan, ctypes.byref(a), X.data_ptr(), ldx, W1.ref, W2.ref, D.data_ptr(), ldd, stream))


class MoePlan:
    """Owns a plan for mixture-of-experts layers; checks the operands that it is given."""

    def __init__(self, n_experts: int, n_in: int, n_hidden: int, dtype, max_tokens: int, max_entries: int,
                 n_out: int = 0, activation: int = TF_ACT_SILU, gated: bool = True):
        self.handle = None
        self.n_experts, self.n_in, self.n_hidden, self.n_out = n_experts, n_in, n_hidden, n_out or n_in
        self.dtype, self.gated = _routed_code(dtype), bool(gated)
        self.handle = tf_moe_create(n_experts, n_in, n_hidden, self.n_out, self.dtype, max_tokens, max_entries,
                                    activation, gated)

    def run(self, A: DeviceCsr, X, W1, W2, D, stream=None) -> None:
        """W1 and W2: both dense (n_experts x (2) n_hidden x n_in, n_experts x n_out x n_hidden) or both Q4Matrix."""
        rows, _, ldx = _matrix(X, "X", self.n_in)
        rows_d, _, ldd = _matrix(D, "D", self.n_out)
        if rows != A.n_rows or rows_d != rows:
            raise ValueError("X and D must have a row for each row of A")
        if _routed_code(X.dtype) != self.dtype or _routed_code(D.dtype) != self.dtype:
            raise TypeError("X and D must have the element type of the plan")
        lib, device = load_library(), X.get_device()
        a = ctypes.byref(_routing(A, device))
        if device < 0 or D.get_device() != device or _device_of(W1, device) != device or _device_of(W2, device) != device:
            _refuse_devices()
        if isinstance(W1, Q4Matrix) and isinstance(W2, Q4Matrix):
            status = lib.tf_moe_layer_q4(self.handle, a, X.data_ptr(), ldx, W1.ref, W2.ref, D.data_ptr(), ldd, stream)
        elif isinstance(W1, Q4Matrix) or isinstance(W2, Q4Matrix):
            raise TypeError("W1 and W2 must both be dense or both have 4 bits")
        else:
            _contiguous(W1, "W1", (self.n_experts, self.n_hidden * (2 if self.gated else 1), self.n_in), self.dtype)
            _contiguous(W2, "W2", (self.n_experts, self.n_out, self.n_hidden), self.dtype)
            status = lib.tf_moe_layer(self.handle, a, X.data_ptr(), ldx, W1.data_ptr(), W2.data_ptr(), D.data_ptr(), ldd, stream)
        if status:
            _check(status)

    def close(self) -> None:
        if self.handle:
            tf_moe_destroy(self.handle)
            self.handle = None

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


# -------------------------------------------------------------------------- losses and their gradients

def _vector(x, what: str, n: int, dtype: str, device: int):
    """Address of a contiguous vector of n elements on `device`."""
    if str(x.dtype) != dtype:
        raise TypeError(f"{what} must be {dtype}")
    if tuple(x.shape) != (n,) or not x.is_contiguous():
        raise ValueError(f"{what} must be contiguous and have {n} elements")
    if x.get_device() != device:
        _refuse_devices()
    return x.data_ptr()


def _router_operands(scores, A):
    """Address, distance of the rows, device and routing matrix of a call on a router's scores."""
    rows, _, ld = _matrix(scores, "scores", A.n_cols)
    if rows != A.n_rows:
        raise ValueError("A must have a row for each row of the scores")
    device = scores.get_device()
    if device < 0:
        _refuse_devices()
    return scores.data_ptr(), ld, device, ctypes.byref(_routing(A, device))


def tf_moe_balance_size(n_tokens: int, n_experts: int) -> int:
    """Bytes of the workspace of tf_moe_balance."""
    out = ctypes.c_int64()
    _check(load_library().tf_moe_balance_size(n_tokens, n_experts, ctypes.byref(out)))
    return out.value


def tf_moe_balance(scores, A: DeviceCsr, counts, mass, loss, workspace, scoring: int = TF_ROUTE_SOFTMAX_TOP,
                   stream=None) -> None:
    """Writes counts (int32, experts + 1), mass (float32, experts) and loss (float32, 1).  workspace: bytes."""
    p, ld, device, a = _router_operands(scores, A)
    e = A.n_cols
    if str(workspace.dtype) != "torch.uint8" or not workspace.is_contiguous() or workspace.get_device() != device:
        raise ValueError("the workspace must be contiguous bytes on the device of the scores")
    if workspace.numel() < tf_moe_balance_size(A.n_rows, e):
        raise ValueError("the workspace is too small")
    status = load_library().tf_moe_balance(
        p, ld, _routed_code(scores.dtype), scoring, a, _vector(counts, "counts", e + 1, "torch.int32", device),
        _vector(mass, "mass", e, "torch.float32", device), _vector(loss, "loss", 1, "torch.float32", device),
        workspace.data_ptr(), stream)
    if status:
        _check(status)


def tf_moe_route_grad(scores, A: DeviceCsr, dscores, scoring: int = TF_ROUTE_SOFTMAX_TOP, scale: float = 1.0, dvals=None,
                      counts=None, dloss=None, stream=None) -> None:
    """Writes dscores: dvals (float32, one for each entry of A) and dloss (float32, 1, with the counts of
    tf_moe_balance) are the gradients of A's values and of the balance loss."""
    p, ld, device, a = _router_operands(scores, A)
    rows, _, ldd = _matrix(dscores, "dscores", A.n_cols)
    if rows != A.n_rows:
        raise ValueError("dscores must have a row for each row of the scores")
    if dscores.dtype != scores.dtype:
        raise TypeError("scores and dscores must have the same element type")
    if dscores.get_device() != device:
        _refuse_devices()
    status = load_library().tf_moe_route_grad(
        p, ld, _routed_code(scores.dtype), scoring, scale, a,
        None if dvals is None else _vector(dvals, "dvals", A.nnz, "torch.float32", device),
        None if counts is None else _vector(counts, "counts", A.n_cols + 1, "torch.int32", device),
        None if dloss is None else _vector(dloss, "dloss", 1, "torch.float32", device), dscores.data_ptr(), ldd, stream)
    if status:
        _check(status)


def tf_xent_size(n_classes: int, n_in: int, dtype, max_rows: int, gradients: bool = True) -> int:
    """Bytes of device memory that a plan for these sizes holds."""
    d, out = tf_xent_desc(n_classes, n_in, max_rows, _routed_code(dtype), 1 if gradients else 0), ctypes.c_int64()
    _check(load_library().tf_xent_size(ctypes.byref(d), ctypes.byref(out)))
    return out.value


def tf_xent_create(n_classes: int, n_in: int, dtype, max_rows: int, gradients: bool = True) -> int:
    """Returns the opaque handle of a plan for the cross entropy of products of these sizes."""
    d = tf_xent_desc(n_classes, n_in, max_rows, _routed_code(dtype), 1 if gradients else 0)
    out = ctypes.c_void_p()
    _check(load_library().tf_xent_create(ctypes.byref(d), ctypes.byref(out)))
    return out.value


def tf_xent_destroy(plan: Optional[int]) -> None:
    _check(load_library().tf_xent_destroy(plan))


def tf_xent_device(plan: int) -> int:
    out = ctypes.c_int32()
    _check(load_library().tf_xent_device(plan, ctypes.byref(out)))
    return out.value


def tf_xent_loss(plan: int, X, W, labels, loss, lse, stream=None) -> None:
    """The caller answers for what a handle does not tell: columns, classes and element type are to be the plan's (XentPlan looks)."""
    rows, n, ldx = _matrix(X, "X")
    _, _, ldw = _matrix(W, "W", n)
    _xent_types(X, W)
    device = X.get_device()
    status = load_library().tf_xent_loss(
        plan, X.data_ptr(), ldx, W.data_ptr(), ldw, _vector(labels, "labels", rows, "torch.int32", device), rows,
        _vector(loss, "loss", rows, "torch.float32", device), _vector(lse, "lse", rows, "torch.float32", device), stream)
    if status:
        _check(status)


def tf_xent_grad(plan: int, X, W, labels, lse, dloss, dX=None, dW=None, stream=None) -> None:
    tf_xent_grad_by_loss(plan, X, W, labels, None, lse, dloss, dX, dW, stream)


def tf_xent_grad_by_loss(plan: int, X, W, labels, loss, lse, dloss, dX=None, dW=None, stream=None) -> None:
    """loss: that of tf_xent_loss, with which the gradients of rows that are nearly certain of their label keep their precision, or None."""
    rows, n, ldx = _matrix(X, "X")
    classes, _, ldw = _matrix(W, "W", n)
    _xent_types(X, W, dX, dW)
    device = X.get_device()
    lddx = lddw = n
    for what, d, want in (("dX", dX, rows), ("dW", dW, classes)):
        if d is not None:
            have, _, step = _matrix(d, what, n)
            if have != want:
                raise ValueError(f"{what} must have {want} rows, not {have}")
            lddx, lddw = (step, lddw) if what == "dX" else (lddx, step)
    status = load_library().tf_xent_grad_by_loss(
        plan, X.data_ptr(), ldx, W.data_ptr(), ldw, _vector(labels, "labels", rows, "torch.int32", device),
        None if loss is None else _vector(loss, "loss", rows, "torch.float32", device), _vector(lse, "lse", rows, "torch.float32", device), _vector(dloss, "dloss", rows, "torch.float32", device), rows,
        _addr(dX), lddx, _addr(dW), lddw, stream)
    if status:
        _check(status)


def _xent_types(X, *others):
    """All operands (or None) have X's element type and lie on its device, which is not the host."""
    device = X.get_device()
    for x in others:
        if x is not None:
            if x.dtype != X.dtype:
                raise TypeError("X, W and their gradients must have the same element type")
            if x.get_device() != device:
                _refuse_devices()
    if device < 0:
        _refuse_devices()


class XentPlan:
    """Owns a plan for the softmax cross entropy of X W^T; checks the operands that it is given."""

    def __init__(self, n_classes: int, n_in: int, dtype, max_rows: int, gradients: bool = True):
        self.handle = None
        self.n_classes, self.n_in, self.dtype = n_classes, n_in, _routed_code(dtype)
        self.handle = tf_xent_create(n_classes, n_in, self.dtype, max_rows, gradients)
        self.device = tf_xent_device(self.handle)

    def _look(self, X, W):
        if tuple(W.shape) != (self.n_classes, self.n_in) or X.shape[-1] != self.n_in:
            raise ValueError(f"W must have the shape {(self.n_classes, self.n_in)} and X {self.n_in} columns")
        if _routed_code(X.dtype) != self.dtype:
            raise TypeError("X must have the element type of the plan")
        if X.get_device() != self.device:
            _refuse_devices()

    def loss(self, X, W, labels, loss, lse, stream=None) -> None:
        """Writes loss and lse (float32, one for each row of X).  labels: int32, others than 0 .. n_classes - 1 for rows without one."""
        self._look(X, W)
        tf_xent_loss(self.handle, X, W, labels, loss, lse, stream)

    def grad(self, X, W, labels, lse, dloss, dX=None, dW=None, stream=None, loss=None) -> None:
        """Writes dX and dW (like X and W; None: not wanted) from lse and the gradient of each row's loss (float32).  loss: what the call of that
        name wrote; with it the gradients of rows that are nearly certain of their label keep their precision."""
        self._look(X, W)
        tf_xent_grad_by_loss(self.handle, X, W, labels, loss, lse, dloss, dX, dW, stream)

    def close(self) -> None:
        if self.handle:
            tf_xent_destroy(self.handle)
            self.handle = None

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class Plan:
    """Owns a plan handle; a convenience over the tf_* functions."""

    def __init__(self, A, bcol: int, ccol: int, b_is_sparse: bool, **params):
        self.handle = tf_plan_create(A, bcol, ccol, b_is_sparse, **params)
        self.b_is_sparse = bool(b_is_sparse)

    def schedule(self) -> dict:
        return tf_plan_schedule(self.handle)

    def run(self, B, C, D, stream=None) -> None:
        (tf_spmm_spmm if self.b_is_sparse else tf_gemm_spmm)(self.handle, B, C, D, stream)

    def run_unfused(self, B, C, D, stream=None) -> None:
        (tf_unfused_spmm_spmm if self.b_is_sparse else tf_unfused_gemm_spmm)(
            self.handle, B, C, D, stream)

    def run_wavefront(self, wavefront: int, B, C, D, stream=None) -> None:
        tf_run_wavefront(self.handle, wavefront, B, C, D, stream)

    def workspace(self) -> int:
        return tf_plan_workspace(self.handle)

    def workspace_unfused(self) -> int:
        return tf_plan_workspace_unfused(self.handle)

    def prepare_unfused(self) -> None:
        tf_plan_prepare_unfused(self.handle)

    def close(self) -> None:
        if self.handle:
            tf_plan_destroy(self.handle)
            self.handle = None

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
