"""Operators of a deep layer whose weights depend on a row's type, and of the head that
answers and is trained: norm, products by group, scores, distillation.

Reached as ``paper_2111_00352_amd.rms_norm`` and so on.  As with the low-bit forms, these are
single library calls without derivatives, bound on small operands by what happens here; the
gradients are calls of their own, and ``paper_2111_00352_amd.layers`` joins both for autograd.
"""
from __future__ import annotations

import ctypes
import functools
from typing import NamedTuple

import torch

from paper_2111_00352_amd import (
    _DTYPES, SavedActivation, _check, _dense, _dtype_code, _NoGradient, _on, _out, _seen, _u64, _written, lib)

TOP_MAX = 128  # alternatives of a row at most (log_probs, distill_loss)
_INTS = {torch.int32: 4, torch.int64: 8}
_F32 = {torch.float32: 0}


def _array(t, name: str, shape: tuple, dtypes: dict, index: int) -> int:
    """The code in `dtypes` of a contiguous CUDA tensor of this shape on GPU `index`."""
    code = dtypes.get(t.dtype) if isinstance(t, torch.Tensor) else None
    if code is None or t.get_device() != index or t.layout != torch.strided or tuple(t.shape) != shape or not t.is_contiguous():
        kinds = " or ".join(str(d)[6:] for d in dtypes)
        raise ValueError(f"{name} must be a contiguous CUDA {kinds} tensor of shape {shape} on the other operands' device")
    _seen(t)
    if t.is_neg():
        raise ValueError(f"{name} must not be a negated view")
    return code


def _results(outs, *operands):
    """outs, computed from operands any of which may require a gradient, as autograd is to see them."""
    if not torch.is_grad_enabled() or not any(t is not None and t.requires_grad for t in operands):
        return outs
    operands = [t for t in operands if t is not None]
    return tuple(_NoGradient.apply(t, *operands) if isinstance(t, torch.Tensor) and t.is_floating_point() else t for t in outs)


def _raise(rc: int):
    if rc:
        _check(rc)


def _at(t):
    return None if t is None else t.data_ptr()


# ------------------------------------------------------------------------ norm


def rms_norm(X: torch.Tensor, weight: torch.Tensor | None = None, residual: torch.Tensor | None = None, eps: float = 1e-6,
             save: bool = False, stream=None) -> tuple:
    """(Y, H, rstd): H = X + residual in X's type (X itself without one), rstd the inverse
    root of the mean of a row's H^2 + eps (fp32), Y = H rstd weight, in X's type or with
    save=True in 8 bits (a SavedActivation, act "none") (gs_rms_norm).  weight: one number
    a column, fp32 or bf16."""
    if stream is not None:
        return _on(stream, rms_norm, X, weight, residual, eps, save)
    of = (X, weight, residual)
    X, ld, code, shape, s = _dense(X, "X")
    rows, cols = shape
    at = X.get_device()
    w_code = 0 if weight is None else _array(weight, "weight", (cols,), _DTYPES, at)
    H, ldr, ldh = X, 0, ld
    if residual is not None:
        residual, ldr, r_code, r_shape, _ = _dense(residual, "residual", at)
        if r_code != code or r_shape != shape:
            raise ValueError("X and the residual must have the same shape and type")
        H, ldh = torch.empty(shape, dtype=X.dtype, device=X.device), cols
    rstd = torch.empty(rows, dtype=torch.float32, device=X.device)
    Y = SavedActivation(shape, "none", X.device) if save else torch.empty(shape, dtype=X.dtype, device=X.device)
    _raise(lib().gs_rms_norm(X.data_ptr(), ld, _at(residual), ldr, code, rows, cols, _at(weight), w_code, float(eps), H.data_ptr(), ldh,
                             None if save else Y.data_ptr(), cols, Y._ref if save else None, rstd.data_ptr(), s))
    if residual is None:
        Y, rstd = _results((Y, rstd), *of)
        return Y, of[0], rstd
    return _results((Y, H, rstd), *of)


@functools.lru_cache(maxsize=1024)
def _norm_work(rows: int, cols: int, code: int) -> int:
    need = _u64()
    _check(lib().gs_rms_norm_grad_workspace(rows, cols, code, ctypes.byref(need)))
    return need.value


def rms_norm_grad(H: torch.Tensor, rstd: torch.Tensor, dY: torch.Tensor, weight: torch.Tensor | None = None,
                  dH: torch.Tensor | None = None, stream=None) -> tuple:
    """(dX, dweight) for rms_norm's H and rstd and the gradient dY of its Y (gs_rms_norm_grad):
    dX is the gradient of X and of the residual; dH, what reaches H by another way, is added to
    it.  dweight is fp32, None without a weight."""
    if stream is not None:
        return _on(stream, rms_norm_grad, H, rstd, dY, weight, dH)
    of = (H, rstd, dY, weight, dH)
    H, ldh, code, shape, s = _dense(H, "H")
    rows, cols = shape
    at = H.get_device()
    _array(rstd, "rstd", (rows,), _F32, at)
    dY, ldy, y_code, y_shape, _ = _dense(dY, "dY", at)
    ldd, d_code, d_shape = 0, code, shape
    if dH is not None:
        dH, ldd, d_code, d_shape, _ = _dense(dH, "dH", at)
    if y_code != code or y_shape != shape or d_code != code or d_shape != shape:
        raise ValueError("H and the gradients must have the same shape and type")
    w_code = 0 if weight is None else _array(weight, "weight", (cols,), _DTYPES, at)
    dX = torch.empty(shape, dtype=H.dtype, device=H.device)
    dw = None if weight is None else torch.empty(cols, dtype=torch.float32, device=H.device)
    need = _norm_work(rows, cols, code)
    work = torch.empty(need, dtype=torch.uint8, device=H.device)
    _raise(lib().gs_rms_norm_grad(H.data_ptr(), ldh, rstd.data_ptr(), dY.data_ptr(), ldy, code, rows, cols, _at(weight), w_code,
                                  _at(dH), ldd, dX.data_ptr(), cols, _at(dw), work.data_ptr(), need, s))
    return _results((dX, dw), *of)


# ----------------------------------------------------------- products by group


def _offsets(offsets, groups: int, at: int) -> int:
    return _array(offsets, "offsets", (groups + 1,), _INTS, at)


def grouped_matmul(A, W: torch.Tensor, offsets: torch.Tensor, transpose: bool = False, dtype=None,
                   out: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """Rows offsets[g] .. offsets[g+1] - 1 of A times W[g] (groups x k x n), or with transpose=True
    times W[g]^T, the gradient of A (gs_grouped_matmul).  A: dense in W's type, or a
    SavedActivation.  offsets: int32 or int64 on the device, not descending.  The result has W's
    type or `dtype`; its rows without a group are 0, those of a given `out` left as they are."""
    if stream is not None:
        return _on(stream, grouped_matmul, A, W, offsets, transpose, dtype, out)
    if not isinstance(W, torch.Tensor) or W.dtype not in _DTYPES or W.dim() != 3 or W.layout != torch.strided:
        raise ValueError("W must be a 3-D CUDA float32 or bfloat16 tensor")
    _seen(W)
    saved = isinstance(A, SavedActivation)
    if saved:
        at, shape, of = A.device.index, A.shape, None
        if at != torch._C._cuda_getDevice():
            raise ValueError("A is not on the current device")
        s = torch._C._cuda_getCurrentRawStream(at)
    else:
        of = A
        A, lda, a_code, shape, s = _dense(A, "A")
        at = A.get_device()
        if A.dtype != W.dtype:
            raise ValueError("A and W must have the same type")
    keep = W
    W = W.resolve_neg()
    if W.get_device() != at:
        raise ValueError("W is not on the current device, or not on the other operand's")
    groups, k, n = W.shape
    step, ldw, one = W.stride()
    if (one != 1 and n > 1) or (k > 1 and ldw < n):
        raise ValueError("W's matrices must have unit column stride and a row stride of at least their width")
    ldw = max(ldw, n)
    if shape[1] != (n if transpose else k):
        raise ValueError(f"A has {shape[1]} columns, W's matrices take {n if transpose else k}")
    bytes_ = _offsets(offsets, groups, at)
    if dtype is None:
        dtype = W.dtype if out is None else out.dtype
    c_code = _dtype_code(dtype)
    C, ldc = _out(out, (shape[0], k if transpose else n), dtype, W.device, keep if saved or keep.requires_grad else of)
    rest = (groups, k, n, int(transpose), offsets.data_ptr(), bytes_, int(out is None), C.data_ptr(), ldc, c_code, s)
    if saved:
        rc = lib().gs_grouped_matmul_saved(A._ref, W.data_ptr(), _DTYPES[W.dtype], ldw, step, *rest)
    else:
        rc = lib().gs_grouped_matmul(A.data_ptr(), lda, a_code, shape[0], W.data_ptr(), ldw, step, *rest)
    _raise(rc)
    if out is not None:
        return _written(C)
    return _results((C,), of, keep)[0]


@functools.lru_cache(maxsize=1024)
def _grouped_work(rows: int, groups: int, a: int, b: int) -> int:
    need = _u64()
    _check(lib().gs_grouped_weight_grad_workspace(rows, groups, a, b, ctypes.byref(need)))
    return need.value


def grouped_weight_grad(A, G: torch.Tensor, offsets: torch.Tensor, stream=None) -> torch.Tensor:
    """A_g^T G_g of each group's rows, groups x a x b in fp32, zeros for a group without rows
    (gs_grouped_weight_grad).  A (rows x a): dense in G's type, or a SavedActivation."""
    if stream is not None:
        return _on(stream, grouped_weight_grad, A, G, offsets)
    saved = isinstance(A, SavedActivation)
    of = (None if saved else A, G)
    G, ldg, code, g_shape, s = _dense(G, "G", A.device.index if saved else -1)
    at = G.get_device()
    if saved:
        shape = A.shape
    else:
        A, lda, a_code, shape, _ = _dense(A, "A", at)
        if a_code != code:
            raise ValueError("A and G must have the same type")
    if shape[0] != g_shape[0]:
        raise ValueError("A and G must have the same number of rows")
    if not isinstance(offsets, torch.Tensor) or offsets.dim() != 1 or offsets.shape[0] < 2:
        raise ValueError("offsets must be a 1-D tensor of at least two numbers")
    groups, a, b = offsets.shape[0] - 1, shape[1], g_shape[1]
    bytes_ = _offsets(offsets, groups, at)
    out = torch.empty((groups, a, b), dtype=torch.float32, device=G.device)
    need = _grouped_work(shape[0], groups, a, b)
    work = torch.empty(need, dtype=torch.uint8, device=G.device) if need else None
    if saved:
        rc = lib().gs_grouped_weight_grad_saved(A._ref, G.data_ptr(), ldg, code, b, groups, offsets.data_ptr(), bytes_, out.data_ptr(),
                                                _at(work), need, s)
    else:
        rc = lib().gs_grouped_weight_grad(A.data_ptr(), lda, G.data_ptr(), ldg, code, shape[0], a, b, groups, offsets.data_ptr(),
                                          bytes_, out.data_ptr(), _at(work), need, s)
    _raise(rc)
    return _results((out,), *of)[0]


# ------------------------------------------------------- scores, distillation


class LogProbs(NamedTuple):
    """What log_probs finds in rows of logits (all fp32 but top_ids, which is int32)."""

    logp: torch.Tensor       # log probability of the row's class, 0 where it has none
    entropy: torch.Tensor
    stats: torch.Tensor      # rows x 2: largest logit, sum of exp(logit - largest)
    top_ids: torch.Tensor    # rows x top, from the most probable on, ties to the lower class
    top_logp: torch.Tensor   # and their log probabilities


def log_probs(logits: torch.Tensor, ids: torch.Tensor, top: int = 0, stream=None) -> LogProbs:
    """Log probability of one class a row (ids: int32 or int64, negative for none), entropy and
    the `top` most probable classes of softmax(logits) (gs_log_probs)."""
    if stream is not None:
        return _on(stream, log_probs, logits, ids, top)
    of = logits
    logits, ld, code, (n, v), s = _dense(logits, "logits")
    id_bytes = _array(ids, "ids", (n,), _INTS, logits.get_device())
    if not 0 <= top <= min(v, TOP_MAX):
        raise ValueError(f"top must be 0 to {min(v, TOP_MAX)}")
    dev = logits.device
    # (each for itself: a caller may change one in place, or keep it alone)
    logp, entropy = torch.empty(n, dtype=torch.float32, device=dev), torch.empty(n, dtype=torch.float32, device=dev)
    stats, best = torch.empty((n, 2), dtype=torch.float32, device=dev), torch.empty((n, top), dtype=torch.float32, device=dev)
    top_ids = torch.empty((n, top), dtype=torch.int32, device=dev)
    _raise(lib().gs_log_probs(logits.data_ptr(), ld, code, n, v, ids.data_ptr(), id_bytes, logp.data_ptr(), entropy.data_ptr(),
                              stats.data_ptr(), top, top_ids.data_ptr(), best.data_ptr(), s))
    return LogProbs(*_results((logp, entropy, stats, top_ids, best), of))


def log_probs_grad(logits: torch.Tensor, ids: torch.Tensor, found: LogProbs, dlogp: torch.Tensor | None = None,
                   dentropy: torch.Tensor | None = None, out: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """Gradient of sum(dlogp logp + dentropy entropy) by the logits, in their type, from what
    log_probs found in them (gs_log_probs_grad); out may be the logits themselves."""
    return _scores_grad(logits, ids, found.stats, found.entropy, dlogp, dentropy, out, stream)


def _scores_grad(logits, ids, stats, entropy, dlogp, dentropy, out, stream=None):
    if stream is not None:
        return _on(stream, _scores_grad, logits, ids, stats, entropy, dlogp, dentropy, out)
    of = logits
    logits, ld, code, (n, v), s = _dense(logits, "logits")
    at = logits.get_device()
    id_bytes = _array(ids, "ids", (n,), _INTS, at)
    _array(stats, "stats", (n, 2), _F32, at)
    _array(entropy, "entropy", (n,), _F32, at)
    for t, name in ((dlogp, "dlogp"), (dentropy, "dentropy")):
        if t is not None:
            _array(t, name, (n,), _F32, at)
    D, ldo = _out(out, (n, v), logits.dtype, logits.device, of)
    _raise(lib().gs_log_probs_grad(logits.data_ptr(), ld, code, n, v, ids.data_ptr(), id_bytes, stats.data_ptr(), _at(dlogp),
                                   _at(dentropy), entropy.data_ptr(), D.data_ptr(), ldo, s))
    return _written(D) if out is not None else _results((D,), of, dlogp, dentropy)[0]


def _teacher(top_ids, top_logits, n: int, at: int) -> tuple:
    if not isinstance(top_ids, torch.Tensor) or top_ids.dim() != 2 or not 1 <= top_ids.shape[1] <= TOP_MAX:
        raise ValueError(f"top_ids must be a 2-D tensor of 1 to {TOP_MAX} columns")
    k = top_ids.shape[1]
    return k, _array(top_ids, "top_ids", (n, k), _INTS, at), _array(top_logits, "top_logits", (n, k), _DTYPES, at)


def distill_loss(logits: torch.Tensor, top_ids: torch.Tensor, top_logits: torch.Tensor, temperature: float = 1.0,
                 stream=None) -> tuple:
    """(loss, stats): a student's loss against a teacher's best classes, one number a row, in
    fp32 (gs_distill_loss): temperature^2 times the divergence of softmax(logits / temperature)
    from the teacher's softmax over the classes it names.  top_ids (rows x k, negative: none) and
    top_logits as log_probs gives them (log probabilities serve as logits).  stats: what
    distill_grad takes."""
    if stream is not None:
        return _on(stream, distill_loss, logits, top_ids, top_logits, temperature)
    of = logits
    logits, ld, code, (n, v), s = _dense(logits, "logits")
    k, id_bytes, t_code = _teacher(top_ids, top_logits, n, logits.get_device())
    stats = torch.empty((n, 4), dtype=torch.float32, device=logits.device)
    loss = torch.empty(n, dtype=torch.float32, device=logits.device)
    _raise(lib().gs_distill_loss(logits.data_ptr(), ld, code, n, v, top_ids.data_ptr(), id_bytes, top_logits.data_ptr(), t_code, k,
                                 float(temperature), loss.data_ptr(), stats.data_ptr(), s))
    return _results((loss, stats), of, top_logits)


def distill_grad(logits: torch.Tensor, top_ids: torch.Tensor, top_logits: torch.Tensor, stats: torch.Tensor, dloss: torch.Tensor,
                 temperature: float = 1.0, out: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """Gradient of sum(dloss loss) by the student's logits, in their type, from distill_loss's
    stats (gs_distill_grad); out may be the logits themselves."""
    if stream is not None:
        return _on(stream, distill_grad, logits, top_ids, top_logits, stats, dloss, temperature, out)
    of = logits
    logits, ld, code, (n, v), s = _dense(logits, "logits")
    at = logits.get_device()
    k, id_bytes, t_code = _teacher(top_ids, top_logits, n, at)
    _array(stats, "stats", (n, 4), _F32, at)
    _array(dloss, "dloss", (n,), _F32, at)
    D, ldo = _out(out, (n, v), logits.dtype, logits.device, of)
    _raise(lib().gs_distill_grad(logits.data_ptr(), ld, code, n, v, top_ids.data_ptr(), id_bytes, top_logits.data_ptr(), t_code, k,
                                 float(temperature), stats.data_ptr(), dloss.data_ptr(), D.data_ptr(), ldo, s))
    return _written(D) if out is not None else _results((D,), of, top_logits, dloss)[0]
