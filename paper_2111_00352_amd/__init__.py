"""GNN-aggregation SpMM with per-layer sparse-format selection on MI355X.

A thin ctypes binding over ``libgnnspmm.so`` (HIP kernels for gfx950 behind
the C ABI of ``include/gnnspmm.h``).  This module only marshals arguments:
validation, conversion, feature extraction, selection and every SpMM run in
the library.  PyTorch supplies device memory (its caching allocator is
installed as the library's allocator) and streams (the current stream).

Paper: Qiu, You, Wang, "Optimizing Sparse Matrix Multiplications for Graph
Neural Networks", arXiv 2111.00352 -- storage formats Sec. 2.2, SpMM Sec. 2.1,
features Sec. 4.4 / Table 2, the per-layer ``SpMMPredict`` runtime Sec. 4.6.

There is no fallback: if the library is missing or no GPU is present, calls
raise.
"""
from __future__ import annotations

import ctypes
import functools
import os

import torch

__all__ = [
    "FORMATS", "FORMAT_NAMES", "GnnSpmmError", "Matrix", "SelectContext", "build_format",
    "extract_features", "lib", "library_path", "FEATURE_NAMES", "set_allocator",
    "SavedActivation", "save_activation", "relu_grad", "saved_weight_grad", "SAVED_GRAD_WIDTH",
    "Mxfp4", "mxfp4_quantize", "mxfp4_matmul",
]

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "libgnnspmm.so")

FORMATS = {"coo": 0, "csr": 1, "ell": 2, "dia": 3, "bsr": 4, "csc": 5}
FORMAT_NAMES = {v: k for k, v in FORMATS.items()}
FEATURE_NAMES = [
    "numRow", "numCol", "NNZ", "N_diags", "aver_RD", "max_RD", "min_RD", "dev_RD",
    "aver_CD", "max_CD", "min_CD", "dev_CD", "ER_DIA", "ER_CD", "row_bounce",
    "col_bounce", "density", "cv", "max_mu",
]
SEL_MODES = {"model": 0, "profile": 1, "fixed": 2}

_i64, _u64, _i32, _p = ctypes.c_int64, ctypes.c_uint64, ctypes.c_int32, ctypes.c_void_p


class _Coo(ctypes.Structure):
    _fields_ = [("n_rows", _i64), ("n_cols", _i64), ("nnz", _i64),
                ("row", _p), ("col", _p), ("val", _p)]


class _BuildOpts(ctypes.Structure):
    _fields_ = [("bsr_block", _i32), ("assume_canonical", _i32), ("max_bytes", _u64)]


class _Info(ctypes.Structure):
    _fields_ = [("format", _i32), ("bsr_block", _i32), ("n_rows", _i64), ("n_cols", _i64),
                ("nnz", _i64), ("param", _i64), ("device_bytes", _u64)]


class _Features(ctypes.Structure):
    _fields_ = [("n_rows", _i64), ("n_cols", _i64), ("nnz", _i64), ("n_diags", _i64),
                ("max_rd", _i64), ("min_rd", _i64), ("max_cd", _i64), ("min_cd", _i64),
                ("sum_rd2", _u64), ("sum_cd2", _u64), ("bounce_r", _u64), ("bounce_c", _u64),
                ("n_blocks16", _i64), ("f", ctypes.c_double * 19)]


class _SelOpts(ctypes.Structure):
    _fields_ = [("mode", _i32), ("fixed", _i32), ("model_path", ctypes.c_char_p),
                ("max_bytes", _u64), ("bsr_block", _i32), ("profile_reps", _i32),
                ("formats", ctypes.c_uint32), ("mem_weight", ctypes.c_double)]


class _SelStats(ctypes.Structure):
    _fields_ = [("t_features", ctypes.c_double), ("t_predict", ctypes.c_double),
                ("t_convert", ctypes.c_double), ("chosen", _i32), ("feasible_mask", _i32),
                ("scores", ctypes.c_double * len(FORMATS))]


class _Saved(ctypes.Structure):
    _fields_ = [("rows", _i64), ("cols", _i64), ("act", _i32), ("codes", _p), ("scales", _p)]


class _Mxfp4(ctypes.Structure):
    _fields_ = [("rows", _i64), ("cols", _i64), ("codes", _p), ("scales", _p)]


_ALLOC_FN = ctypes.CFUNCTYPE(_p, ctypes.c_size_t, _p, _p)
_FREE_FN = ctypes.CFUNCTYPE(None, _p, _p, _p)


class _Allocator(ctypes.Structure):
    _fields_ = [("alloc", _ALLOC_FN), ("free", _FREE_FN), ("ctx", _p)]


class GnnSpmmError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"gnnspmm error {code}: {msg}")
        self.code = code


ERR_INVALID_ARG, ERR_INDEX, ERR_DUPLICATE, ERR_EXPLICIT_ZERO = -1, -2, -3, -4
ERR_INFEASIBLE, ERR_OOM, ERR_HIP, ERR_MODEL, ERR_UNSUPPORTED = -5, -6, -7, -8, -9

_lib = None
_alloc_keep = None
# Every hook set ever installed through set_allocator, kept for the life of
# the process: the library frees each buffer through the hooks that
# allocated it, so a collected callback would be called after it is gone.
_hooks_alive: list = []


def library_path() -> str:
    return _LIB_PATH


def lib() -> ctypes.CDLL:
    """Loads libgnnspmm.so (raises if it has not been built)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(_LIB_PATH):
        raise RuntimeError(
            f"{_LIB_PATH} is missing: build it with `python -m paper_2111_00352_amd.build`"
        )
    L = ctypes.CDLL(_LIB_PATH)
    c_int = ctypes.c_int
    P = ctypes.POINTER
    sigs = {
        "gs_set_allocator": (c_int, [P(_Allocator)]),
        "gs_build_format": (c_int, [P(_Coo), c_int, P(_BuildOpts), _p, P(_p), P(_u64)]),
        "gs_convert": (c_int, [_p, c_int, P(_BuildOpts), _p, P(_p), P(_u64)]),
        "gs_spmm": (c_int, [_p, _p, _i64, _p, _i64, _i64, _p]),
        "gs_spmm_noalloc": (c_int, [_p, _p, _i64, _p, _i64, _i64, _p]),
        "gs_to_coo": (c_int, [_p, _p, _p, _p, _p]),
        "gs_get_info": (c_int, [_p, P(_Info)]),
        "gs_get_array": (c_int, [_p, c_int, P(_p), P(_u64)]),
        "gs_copy_array": (c_int, [_p, c_int, _p, _u64, _p]),
        "gs_destroy": (None, [_p]),
        "gs_extract_features": (c_int, [P(_Coo), P(_BuildOpts), _p, P(_Features)]),
        "gs_matrix_features": (c_int, [_p, _p, P(_Features)]),
        "gs_ctx_create": (c_int, [P(_SelOpts), P(_p)]),
        "gs_ctx_destroy": (None, [_p]),
        "gs_select": (c_int, [_p, _u64, P(_Coo), _i64, _p, P(_i32)]),
        "gs_select_and_run": (c_int, [_p, _u64, P(_Coo), _p, _i64, _p, _i64, _i64, _p, P(_i32)]),
        "gs_ctx_stats": (c_int, [_p, P(_SelStats)]),
        "gs_weight_grad_workspace": (c_int, [_i64, _i64, _i64, P(_u64)]),
        "gs_weight_grad": (c_int, [_p, _i64, _p, _i64, _i64, _i64, _i64, _p, _p, _u64, _p]),
        "gs_saved_layout": (c_int, [_i64, P(_i64), P(_i64)]),
        "gs_save_activation": (c_int, [_p, _i64, c_int, P(_Saved), _p, _i64, _p]),
        "gs_saved_dequantize": (c_int, [P(_Saved), _p, _i64, c_int, _p]),
        "gs_relu_grad": (c_int, [P(_Saved), _p, _i64, c_int, _p, _i64, _p]),
        "gs_saved_weight_grad_workspace": (c_int, [_i64, _i64, _i64, P(_u64)]),
        "gs_saved_weight_grad": (c_int, [P(_Saved), _p, _i64, c_int, _i64, _p, _p, _u64, _p]),
        "gs_mxfp4_layout": (c_int, [_i64, P(_i64), P(_i64)]),
        "gs_mxfp4_quantize": (c_int, [_p, _i64, c_int, _i64, _i64, c_int, P(_Mxfp4), _p]),
        "gs_mxfp4_dequantize": (c_int, [P(_Mxfp4), _p, _i64, c_int, _p]),
        "gs_mxfp4_matmul": (c_int, [P(_Mxfp4), P(_Mxfp4), P(_Saved), _p, _i64, c_int, _p, _u64, _p]),
        "gs_mxfp4_matmul_dense": (c_int, [_p, _i64, c_int, _i64, P(_Mxfp4), P(_Saved), _p, _i64, c_int, _p, _u64, _p]),
        "gs_mxfp4_matmul_workspace": (c_int, [_i64, _i64, _i64, c_int, P(_u64)]),
        "gs_last_error": (ctypes.c_char_p, []),
        "gs_abi_version": (c_int, []),
    }
    for name, (res, args) in sigs.items():
        fn = getattr(L, name)
        fn.restype = res
        fn.argtypes = args
    _lib = L
    return L


def _check(rc: int):
    if rc != 0:
        raise GnnSpmmError(rc, lib().gs_last_error().decode(errors="replace"))


def _require_gpu():
    if not torch.cuda.is_available():
        raise RuntimeError("gnnspmm needs a ROCm GPU (torch.cuda.is_available() is False)")
    _install_torch_allocator()


def _install_torch_allocator(reinstall: bool = False):
    """Routes the library's device allocations through PyTorch's caching allocator."""
    global _alloc_keep
    if _alloc_keep is not None:
        if reinstall:
            _check(lib().gs_set_allocator(ctypes.byref(_alloc_keep[0])))
        return

    # (what torch.cuda.caching_allocator_alloc / _delete call for the current
    # device, without their device switch: a first call makes some fifty of these)
    raw_alloc = torch._C._cuda_cudaCachingAllocator_raw_alloc
    raw_delete = torch._C._cuda_cudaCachingAllocator_raw_delete

    def _alloc(nbytes, stream, _ctx):
        try:
            return raw_alloc(nbytes, stream or 0)
        except Exception:  # out of memory -> the library reports GS_ERR_OOM
            return None

    def _free(ptr, _stream, _ctx):
        raw_delete(ptr)

    a = _Allocator(_ALLOC_FN(_alloc), _FREE_FN(_free), None)
    _check(lib().gs_set_allocator(ctypes.byref(a)))
    _alloc_keep = (a, _alloc, _free)


def set_allocator(alloc=None, free=None):
    """Installs device allocation hooks for all later library allocations
    (gs_set_allocator).  alloc(nbytes, stream) returns a device pointer
    (int) aligned to 256 bytes, or 0 / None when it cannot allocate;
    free(ptr, stream) releases one; both must be stream-ordered (see
    gs_allocator).  No arguments reinstall PyTorch's caching allocator.

    Buffers always go back through the hooks that allocated them, so the
    hooks must outlive every handle built with them: this binding keeps each
    hook set (the callables and their ctypes wrappers) referenced until the
    process ends, whatever the caller does with its own references."""
    if (alloc is None) != (free is None):
        raise ValueError("alloc and free must both be given or both be None")
    if alloc is None:
        _install_torch_allocator(reinstall=True)
        return

    def _a(nbytes, stream, _ctx):
        try:
            p = alloc(int(nbytes), int(stream or 0))
        except Exception:  # reported by the library as GS_ERR_OOM
            return None
        return int(p) if p else None

    def _f(ptr, stream, _ctx):
        free(int(ptr), int(stream or 0))

    hooks = _Allocator(_ALLOC_FN(_a), _FREE_FN(_f), None)
    _hooks_alive.append((hooks, _a, _f, alloc, free))
    _check(lib().gs_set_allocator(ctypes.byref(hooks)))


def _stream(stream=None) -> int:
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())
    return int(stream.cuda_stream if hasattr(stream, "cuda_stream") else stream)


def _ptr(t: torch.Tensor | None) -> int | None:
    return None if t is None or t.numel() == 0 else t.data_ptr()


def _coo_struct(row, col, val, shape, into=None):
    """The gs_coo of the triplets (written to `into` if given)."""
    if not (row.is_cuda and col.is_cuda and val.is_cuda and row.dtype == torch.int32 and col.dtype == torch.int32
            and val.dtype == torch.float32 and row.dim() == 1 and col.dim() == 1 and val.dim() == 1
            and row.is_contiguous() and col.is_contiguous() and val.is_contiguous()):
        raise ValueError("row/col must be contiguous CUDA int32, val contiguous CUDA float32")
    n = row.numel()
    if not (n == col.numel() == val.numel()):
        raise ValueError("row, col and val must have the same length")
    A = _Coo() if into is None else into
    A.n_rows, A.n_cols, A.nnz = int(shape[0]), int(shape[1]), n
    A.row, A.col, A.val = (row.data_ptr(), col.data_ptr(), val.data_ptr()) if n else (None, None, None)
    return A


def _opts(bsr_block=16, assume_canonical=False, max_bytes=None):
    return _BuildOpts(int(bsr_block), 1 if assume_canonical else 0, int(max_bytes or 0))


def _check_dense(X: torch.Tensor, name: str):
    if not X.is_cuda or X.dtype != torch.float32 or X.dim() != 2 or X.stride(1) != 1:
        raise ValueError(f"{name} must be a 2-D CUDA float32 tensor with unit column stride")


class Matrix:
    """A sparse matrix held on the device in one storage format."""

    def __init__(self, handle: int):
        self._h = ctypes.c_void_p(handle)
        info = _Info()
        _check(lib().gs_get_info(self._h, ctypes.byref(info)))
        self.format = FORMAT_NAMES[info.format]
        self.shape = (info.n_rows, info.n_cols)
        self.nnz = info.nnz
        self.param = info.param
        self.bsr_block = info.bsr_block
        self.device_bytes = info.device_bytes

    @property
    def handle(self) -> ctypes.c_void_p:
        return self._h

    def close(self):
        if self._h:
            lib().gs_destroy(self._h)
            self._h = ctypes.c_void_p(None)

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def spmm(self, X: torch.Tensor, out: torch.Tensor | None = None, stream=None) -> torch.Tensor:
        """Y = A.X (Sec. 2.1), asynchronous on the current stream."""
        _check_dense(X, "X")
        R, C = self.shape
        if X.shape[0] != C:
            raise ValueError(f"X has {X.shape[0]} rows, A has {C} columns")
        F = X.shape[1]
        if out is None:
            out = X.new_empty((R, F))
        else:
            _check_dense(out, "out")
            if out.shape[0] != R or out.shape[1] != F:
                raise ValueError("out has the wrong shape")
        rc = lib().gs_spmm(self._h, _ptr(X), X.stride(0), _ptr(out), out.stride(0), F, _stream(stream))
        if rc:
            _check(rc)
        return out

    def spmm_noalloc(self, X: torch.Tensor, out: torch.Tensor, stream=None) -> torch.Tensor:
        """Y = A.X into the preallocated `out` without any device allocation
        (gs_spmm_noalloc: the workspace is the library's fixed per-device
        scratch array, shared by every such call on the device)."""
        _check_dense(X, "X")
        _check_dense(out, "out")
        R, C = self.shape
        if X.shape[0] != C or out.shape[0] != R or out.shape[1] != X.shape[1]:
            raise ValueError("X / out shapes do not match A")
        _check(lib().gs_spmm_noalloc(self._h, _ptr(X), X.stride(0), _ptr(out), out.stride(0), X.shape[1],
                                     _stream(stream)))
        return out

    def to_coo(self, stream=None):
        dev = torch.device("cuda", torch.cuda.current_device())
        row = torch.empty(self.nnz, dtype=torch.int32, device=dev)
        col = torch.empty(self.nnz, dtype=torch.int32, device=dev)
        val = torch.empty(self.nnz, dtype=torch.float32, device=dev)
        _check(lib().gs_to_coo(self._h, _ptr(row), _ptr(col), _ptr(val), _stream(stream)))
        return row, col, val

    def array(self, which: int, dtype=None, stream=None) -> torch.Tensor:
        """Copy of raw array `which` (see gs_get_array) as a 1-D tensor."""
        p, nbytes = ctypes.c_void_p(), _u64()
        _check(lib().gs_get_array(self._h, which, ctypes.byref(p), ctypes.byref(nbytes)))
        if dtype is None:
            dtype = torch.float32 if self._is_value_array(which) else torch.int32
        item = torch.empty((), dtype=dtype).element_size()
        out = torch.empty(nbytes.value // item, dtype=dtype,
                          device=torch.device("cuda", torch.cuda.current_device()))
        _check(lib().gs_copy_array(self._h, which, _ptr(out), nbytes.value, _stream(stream)))
        return out

    def _is_value_array(self, which: int) -> bool:
        f = self.format
        return (which == 2) or (which == 1 and f in ("ell", "dia"))

    def features(self, stream=None) -> dict:
        out = _Features()
        _check(lib().gs_matrix_features(self._h, _stream(stream), ctypes.byref(out)))
        return _features_dict(out)

    def convert(self, fmt: str, bsr_block=16, max_bytes=None, stream=None) -> "Matrix":
        h, need = ctypes.c_void_p(), _u64()
        o = _opts(bsr_block, False, max_bytes)
        rc = lib().gs_convert(self._h, FORMATS[fmt], ctypes.byref(o), _stream(stream),
                              ctypes.byref(h), ctypes.byref(need))
        if rc != 0:
            e = GnnSpmmError(rc, lib().gs_last_error().decode(errors="replace"))
            e.bytes_required = need.value
            raise e
        return Matrix(h.value)


def build_format(row, col, val, shape, fmt: str = "csr", bsr_block: int = 16,
                 max_bytes: int | None = None, assume_canonical: bool = False,
                 stream=None) -> Matrix:
    """Builds A (COO on the device, any order) in format fmt (Sec. 2.2)."""
    _require_gpu()
    A = _coo_struct(row, col, val, shape)
    o = _opts(bsr_block, assume_canonical, max_bytes)
    h, need = ctypes.c_void_p(), _u64()
    rc = lib().gs_build_format(ctypes.byref(A), FORMATS[fmt], ctypes.byref(o), _stream(stream),
                               ctypes.byref(h), ctypes.byref(need))
    if rc != 0:
        e = GnnSpmmError(rc, lib().gs_last_error().decode(errors="replace"))
        e.bytes_required = need.value
        raise e
    return Matrix(h.value)


def weight_grad(H: torch.Tensor, G: torch.Tensor, stream=None) -> torch.Tensor:
    """H^T G for tall H (n x a) and G (n x b) on the matrix cores (gs_weight_grad).
    The result and the workspace, which is given back on return, belong to `stream`."""
    _check_dense(H, "H")
    _check_dense(G, "G")
    if H.shape[0] != G.shape[0]:
        raise ValueError("H and G must have the same number of rows")
    if H.device != G.device:
        raise ValueError("H and G must be on the same device")
    if stream is not None and _stream(stream) != _stream():
        if not isinstance(stream, torch.cuda.Stream):
            raw = _stream(stream)
            stream = torch.cuda.ExternalStream(raw) if raw else torch.cuda.default_stream()
        with torch.cuda.stream(stream):
            return weight_grad(H, G)
    n, a, b = H.shape[0], H.shape[1], G.shape[1]
    need = _u64()
    _check(lib().gs_weight_grad_workspace(n, a, b, ctypes.byref(need)))
    out = torch.empty((a, b), dtype=torch.float32, device=H.device)
    work = torch.empty(need.value // 4, dtype=torch.float32, device=H.device)
    _check(lib().gs_weight_grad(H.data_ptr(), H.stride(0), G.data_ptr(), G.stride(0), n, a, b, out.data_ptr(),
                                work.data_ptr(), need.value, _stream()))
    return out


# ------------------------------------------------- low-bit forms of dense operands
#
# Calls on small operands are bound by what happens here, so arguments are looked at
# once each and nothing is made that the call does not need.
#
# The calls have no derivatives (the layers in gcn define theirs), and codes carry none:
# a backward pass that reaches a result computed from a tensor that requires a gradient
# fails there, rather than going on without that part.

ACTIVATIONS = {"none": 0, "relu": 1}
SAVED_GRAD_WIDTH = 4096  # columns of either operand of saved_weight_grad at most
_DTYPES = {torch.float32: 0, torch.bfloat16: 1}
_STRIDED = torch.strided
_tracing, _forward_ad = torch._C._get_tracing_state, torch.autograd.forward_ad


def _dense(X: torch.Tensor, name: str, index: int | None = -1) -> tuple:
    """(tensor, leading dimension, dtype code, shape, current stream) of a 2-D fp32 or bf16
    operand on the current device, and on the GPU `index` of another operand (None: it is
    on none)."""
    code = _DTYPES.get(X.dtype) if isinstance(X, torch.Tensor) else None
    if code is None or X.layout != _STRIDED or len(shape := X.shape) != 2 or (at := X.get_device()) < 0:
        raise ValueError(f"{name} must be a 2-D CUDA float32 or bfloat16 tensor")
    if _tracing() is not None:
        raise RuntimeError("the low-bit operators cannot be traced: a trace would keep their results as constants")
    if _forward_ad._current_level >= 0 and _forward_ad.unpack_dual(X).tangent is not None:
        raise RuntimeError("the low-bit operators have no forward-mode derivative")
    if at != torch._C._cuda_getDevice() or (index != -1 and at != index):
        raise ValueError(f"{name} is not on the current device, or not on the other operand's")
    if X.is_neg():
        X = X.resolve_neg()
    rows, cols = shape
    ld, step = X.stride()
    if step != 1 and cols > 1 and rows > 0:
        raise ValueError(f"{name} must have unit column stride")
    if ld < cols or rows <= 1:
        if rows > 1:
            raise ValueError(f"{name} must have a row stride of at least its width")
        ld = cols
    return X, ld, code, shape, torch._C._cuda_getCurrentRawStream(at)


class _NoGradient(torch.autograd.Function):
    """The result of a call, in the place of its operands' derivatives."""

    @staticmethod
    def forward(ctx, result, *operands):
        return result

    @staticmethod
    def backward(ctx, *_):
        raise RuntimeError("the low-bit operators have no gradient: detach their operands, or use the layers of gcn")


def _result(t: torch.Tensor, X: torch.Tensor) -> torch.Tensor:
    """t, a new tensor computed from X that requires a gradient, as autograd is to see it."""
    return _NoGradient.apply(t, X) if torch.is_grad_enabled() else t


def _written(out: torch.Tensor) -> torch.Tensor:
    """`out`, whose change a graph that keeps it for a backward pass is to find."""
    if not out.is_inference():
        torch.autograd.graph.increment_version(out)
    return out


def _dtype_code(dtype) -> int:
    if dtype not in _DTYPES:
        raise ValueError("dtype must be torch.float32 or torch.bfloat16")
    return _DTYPES[dtype]


def _on(stream, call, *args):
    """call(*args) with `stream` as the current stream, so that what it allocates belongs
    to it; memory of the arguments is not given out again before it has read them."""
    if _stream(stream) == _stream():
        return call(*args)
    if not isinstance(stream, torch.cuda.Stream):
        raw = _stream(stream)
        stream = torch.cuda.ExternalStream(raw) if raw else torch.cuda.default_stream()
    with torch.cuda.stream(stream):
        out = call(*args)
    for t in args:
        if isinstance(t, (SavedActivation, Mxfp4)):
            t._buf.record_stream(stream)
        elif isinstance(t, torch.Tensor):
            t.record_stream(stream)
    return out


def _out(out, shape, dtype, device, operand=None):
    """`out`, or a new tensor, and its leading dimension; `operand`: what is computed from."""
    if out is None:
        return torch.empty(shape, dtype=dtype, device=device), shape[1]
    if tuple(out.shape) != tuple(shape) or out.dtype != dtype or out.is_neg():
        raise ValueError("out has the wrong shape or dtype")
    if torch.is_grad_enabled() and (out.requires_grad or (operand is not None and operand.requires_grad)):
        raise ValueError("out cannot be given where an argument requires a gradient")
    return out, _dense(out, "out", device.index)[1]


class _Blocks:
    """Codes and scale bytes of a matrix in blocks of 32 columns, in one buffer."""

    def __init__(self, shape, code_pitch, scale_pitch, device, buffer=None):
        rows = shape[0]
        self.shape = (rows, shape[1])
        self._pitches = code_pitch, scale_pitch
        self._at = at = -(-rows * code_pitch // 256) * 256  # (the scales start 256-byte aligned)
        size = at + rows * scale_pitch
        if buffer is None:
            buffer = torch.empty(size, dtype=torch.uint8, device=device)
        elif buffer.shape != (size,) or buffer.dtype != torch.uint8 or not buffer.is_contiguous():
            raise ValueError("the buffer is not that of a matrix of this shape")
        else:
            device = None
        self._buf = buffer
        self.device = device if type(device) is torch.device and device.index is not None else buffer.device
        self._ptr = buffer.data_ptr()

    @property
    def buffer(self) -> torch.Tensor:
        """Codes and scale bytes as one tensor: what a save_for_backward is given."""
        return self._buf

    @property
    def codes(self) -> torch.Tensor:
        rows, pitch = self.shape[0], self._pitches[0]
        return self._buf[:rows * pitch].view(rows, pitch)

    @property
    def scales(self) -> torch.Tensor:
        return self._buf[self._at:].view(self.shape[0], self._pitches[1])

    @property
    def device_bytes(self) -> int:
        return self.shape[0] * sum(self._pitches)

    def dequantize(self, dtype=torch.float32, stream=None) -> torch.Tensor:
        """The values the codes stand for, exact in either type."""
        if stream is not None:
            return _on(stream, type(self).dequantize, self, dtype)
        code = _dtype_code(dtype)
        at = torch._C._cuda_getDevice()
        if self.device.index != at:
            raise ValueError("the codes are not on the current device")
        out = torch.empty(self.shape, dtype=dtype, device=self.device)
        rc = self._values(lib())(self._ref, out.data_ptr(), self.shape[1], code, torch._C._cuda_getCurrentRawStream(at))
        if rc:
            _check(rc)
        return out


class SavedActivation(_Blocks):
    """Activations kept in 8 bits (gs_saved): codes, one power-of-two step per 32 columns of a row.
    buffer: that of other saved activations of this shape, or a copy of it."""

    def __init__(self, shape, act: str, device, buffer: torch.Tensor | None = None):
        blocks = -(-shape[1] // 32)
        super().__init__(shape, 32 * blocks, blocks, device, buffer)
        self.act = act
        self._c = _Saved(shape[0], shape[1], ACTIVATIONS[act], self._ptr, self._ptr + self._at)
        self._ref = ctypes.byref(self._c)

    @staticmethod
    def _values(L):
        return L.gs_saved_dequantize


class Mxfp4(_Blocks):
    """A matrix in MXFP4 (gs_mxfp4): e2m1 codes, one power-of-two scale per 32 columns of a row."""

    def __init__(self, shape, device):
        step = 64 if shape[1] <= 64 else 128
        padded = -(-shape[1] // step) * step
        super().__init__(shape, padded // 2, padded // 32, device)
        self._c = _Mxfp4(shape[0], shape[1], self._ptr, self._ptr + self._at)
        self._ref = ctypes.byref(self._c)

    @staticmethod
    def _values(L):
        return L.gs_mxfp4_dequantize


def save_activation(P: torch.Tensor, act: str = "relu", stream=None) -> tuple:
    """(H, saved): H = relu(P) (act "relu") or P itself (act "none"), and H in 8 bits
    for the backward pass (gs_save_activation)."""
    if stream is not None:
        return _on(stream, save_activation, P, act)
    if act not in ACTIVATIONS:
        raise ValueError("act must be 'relu' or 'none'")
    P, ld, code, shape, s = _dense(P, "P")
    saved = SavedActivation(shape, act, P.device)
    if act == "relu":
        H = torch.empty_like(P) if ld == shape[1] else torch.empty(shape, dtype=P.dtype, device=P.device)
        rc = lib().gs_save_activation(P.data_ptr(), ld, code, saved._ref, H.data_ptr(), shape[1], s)
    else:
        rc = lib().gs_save_activation(P.data_ptr(), ld, code, saved._ref, None, 0, s)
    if rc:
        _check(rc)
    if act != "relu":
        H = P
    elif P.requires_grad:
        H = _result(H, P)
    return H, saved


def relu_grad(saved: SavedActivation, dH: torch.Tensor, out: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """dH where the saved ReLU was active, else 0 (gs_relu_grad); out may be dH."""
    if stream is not None:
        return _on(stream, relu_grad, saved, dH, out)
    dH, ld, code, shape, s = _dense(dH, "dH", saved.device.index)
    if shape != saved.shape:
        raise ValueError("dH and the saved activations have different shapes")
    if out is None and ld == shape[1]:
        dP, ldp = torch.empty_like(dH), ld  # (the quickest way to a tensor of this shape)
    else:
        dP, ldp = _out(out, shape, dH.dtype, dH.device, dH)
    rc = lib().gs_relu_grad(saved._ref, dH.data_ptr(), ld, code, dP.data_ptr(), ldp, s)
    if rc:
        _check(rc)
    if out is not None:
        return _written(dP)
    return _result(dP, dH) if dH.requires_grad else dP


@functools.lru_cache(maxsize=1024)
def _grad_work(n: int, a: int, b: int) -> int:
    need = _u64()
    _check(lib().gs_saved_weight_grad_workspace(n, a, b, ctypes.byref(need)))
    return need.value


def saved_weight_grad(saved: SavedActivation, G: torch.Tensor, stream=None) -> torch.Tensor:
    """H^T G in fp32 from saved activations H (n x a) and G (n x b), a and b at most
    SAVED_GRAD_WIDTH (gs_saved_weight_grad)."""
    if stream is not None:
        return _on(stream, saved_weight_grad, saved, G)
    G, ld, code, shape, s = _dense(G, "G", saved.device.index)
    (n, a), b = saved.shape, shape[1]
    if shape[0] != n:
        raise ValueError("G and the saved activations must have the same number of rows")
    out = torch.empty((a, b), dtype=torch.float32, device=G.device)
    if not a or not b:
        return out
    need = _grad_work(n, a, b)
    work = torch.empty(need, dtype=torch.uint8, device=G.device) if need else None
    rc = lib().gs_saved_weight_grad(saved._ref, G.data_ptr(), ld, code, b, out.data_ptr(),
                                    None if work is None else work.data_ptr(), need, s)
    if rc:
        _check(rc)
    return _result(out, G) if G.requires_grad else out


def mxfp4_quantize(X: torch.Tensor, axis: int = 1, stream=None) -> Mxfp4:
    """X in MXFP4, with blocks of 32 along its rows (axis 1), or X^T with blocks along
    X's columns (axis 0): the operands of mxfp4_matmul for X W are X and W with axis 0
    (gs_mxfp4_quantize)."""
    if stream is not None:
        return _on(stream, mxfp4_quantize, X, axis)
    if axis not in (0, 1):
        raise ValueError("axis must be 0 or 1")
    X, ld, code, (rows, cols), s = _dense(X, "X")
    q = Mxfp4((rows, cols) if axis == 1 else (cols, rows), X.device)
    rc = lib().gs_mxfp4_quantize(X.data_ptr(), ld, code, rows, cols, axis, q._ref, s)
    if rc:
        _check(rc)
    return q


@functools.lru_cache(maxsize=1024)
def _matmul_work(m: int, n: int, k: int, a_code: int) -> int:
    need = _u64()
    _check(lib().gs_mxfp4_matmul_workspace(m, n, k, a_code, ctypes.byref(need)))
    return need.value


def mxfp4_matmul(A, B: Mxfp4, mask: SavedActivation | None = None, dtype=torch.float32,
                 out: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """A B^T for A (m x k: an Mxfp4, or a dense tensor that is quantised along its rows
    within the call) and B (n x k, an Mxfp4), as fp32 or bf16 (gs_mxfp4_matmul).  mask:
    activations saved by a ReLU (m x n); the product is 0 where they are."""
    if stream is not None:
        return _on(stream, mxfp4_matmul, A, B, mask, dtype, out)
    code = _dtype_code(dtype)
    if not isinstance(B, Mxfp4):
        raise ValueError("B must be an Mxfp4")
    device = B.device
    quantised = isinstance(A, Mxfp4)
    if quantised:
        if A.device != device or device.index != torch._C._cuda_getDevice():
            raise ValueError("A and B must be on the current device")
        a_code, (m, k), s = -1, A.shape, _stream()
    else:
        A, lda, a_code, (m, k), s = _dense(A, "A", device.index)
    n, kb = B.shape
    if k != kb:
        raise ValueError(f"A has {k} columns, B has {kb}")
    if mask is not None and (mask.shape != (m, n) or mask.device != device):
        raise ValueError("the mask's shape or device is not the product's")
    C, ldc = _out(out, (m, n), dtype, device, None if quantised else A)
    need = _matmul_work(m, n, k, a_code)
    work = torch.empty(need, dtype=torch.uint8, device=device) if need else None
    mask_ref, at = None if mask is None else mask._ref, None if work is None else work.data_ptr()
    if quantised:
        rc = lib().gs_mxfp4_matmul(A._ref, B._ref, mask_ref, C.data_ptr(), ldc, code, at, need, s)
    else:
        rc = lib().gs_mxfp4_matmul_dense(A.data_ptr(), lda, a_code, m, B._ref, mask_ref, C.data_ptr(), ldc, code, at, need,
                                         s)
    if rc:
        _check(rc)
    if out is not None:
        return _written(C)
    return C if quantised or not A.requires_grad else _result(C, A)


def _features_dict(out: _Features) -> dict:
    d = {k: int(getattr(out, k)) for k, _ in _Features._fields_ if k != "f"}
    d["f"] = [float(x) for x in out.f]
    return d


def extract_features(row, col, val, shape, stream=None) -> dict:
    """Features F1..F19 of Table 2 (Sec. 4.4) plus the integer aggregates."""
    _require_gpu()
    A = _coo_struct(row, col, val, shape)
    out = _Features()
    _check(lib().gs_extract_features(ctypes.byref(A), None, _stream(stream), ctypes.byref(out)))
    return _features_dict(out)


class SelectContext:
    """Per-layer format selection and dispatch (the paper's SpMMPredict, Sec. 4.6)."""

    def __init__(self, mode: str = "model", fixed: str = "csr", model_path: str | None = None,
                 max_bytes: int | None = None, bsr_block: int = 16, profile_reps: int = 3,
                 formats=None, mem_weight: float = 0.0):
        """model_path None: the trained ensemble shipped in selector/model.gsm
        (the library's hand-set trees if that file is absent); "builtin": the
        hand-set trees.  formats: names of the candidate formats of "model"
        and "profile" (None: all).  mem_weight: 1 - w of Eq. 1, the weight of
        the memory footprint against the running time (0: time only); "model"
        needs a model trained for that w."""
        _require_gpu()
        if model_path is None:
            from paper_2111_00352_amd.selector import MODEL_PATH

            model_path = MODEL_PATH if os.path.exists(MODEL_PATH) else None
        elif model_path == "builtin":
            model_path = None
        self._model_path = model_path.encode() if model_path else None
        mask = 0 if formats is None else sum(1 << FORMATS[f] for f in formats)
        o = _SelOpts(SEL_MODES[mode], FORMATS[fixed], self._model_path, int(max_bytes or 0),
                     int(bsr_block), int(profile_reps), mask, float(mem_weight))
        h = ctypes.c_void_p()
        _check(lib().gs_ctx_create(ctypes.byref(o), ctypes.byref(h)))
        self._h = h
        self._keep = {}
        # the arguments of run(), written anew by every call (a context is not
        # thread-safe): making them costs more than filling them in
        self._coo, self._chosen = _Coo(), _i32()
        self._coo_ref, self._chosen_ref = ctypes.byref(self._coo), ctypes.byref(self._chosen)
        self._run = lib().gs_select_and_run

    def close(self):
        if self._h:
            lib().gs_ctx_destroy(self._h)
            self._h = ctypes.c_void_p(None)

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def run(self, key: int, row, col, val, shape, X: torch.Tensor,
            out: torch.Tensor | None = None, stream=None):
        """Y = A.X in the selected format; returns (Y, format name)."""
        _check_dense(X, "X")
        _coo_struct(row, col, val, shape, self._coo)
        F = X.shape[1]
        if out is None:
            out = X.new_empty((int(shape[0]), F))
        else:
            _check_dense(out, "out")
        rc = self._run(self._h, int(key), self._coo_ref, _ptr(X), X.stride(0), _ptr(out), out.stride(0), F,
                       _stream(stream), self._chosen_ref)
        if rc:
            _check(rc)
        return out, FORMAT_NAMES[self._chosen.value]

    def select(self, key: int, row, col, val, shape, F: int, stream=None) -> str:
        A = _coo_struct(row, col, val, shape)
        chosen = _i32()
        _check(lib().gs_select(self._h, int(key), ctypes.byref(A), int(F), _stream(stream),
                               ctypes.byref(chosen)))
        return FORMAT_NAMES[chosen.value]

    def stats(self) -> dict:
        st = _SelStats()
        _check(lib().gs_ctx_stats(self._h, ctypes.byref(st)))
        return dict(t_features=st.t_features, t_predict=st.t_predict, t_convert=st.t_convert,
                    chosen=FORMAT_NAMES.get(st.chosen, "?"), feasible_mask=st.feasible_mask,
                    scores={FORMAT_NAMES[i]: st.scores[i] for i in range(len(FORMATS))})
