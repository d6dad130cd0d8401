"""Differentiable layers of the norm, the products by group, the scores and the distillation.

Each joins the library's forward and gradient calls for autograd; first derivatives only.
They can be captured into a graph, forward and backward pass together, as long as no graph
recorded outside the capture still holds the same parameters, directly or through other
operations (an error where such a graph has one of these layers in it).

    Z, H = norm_grouped_linear(X, w, W, offsets, residual=H0)   # norm(X + H0) in 8 bits, by group
    Z = grouped_linear(X, W, offsets)
    Y, H = rms_norm(X, w, residual=H0)
    logp, entropy = log_probs(logits, ids)                      # -logp.mean() is the usual loss
    loss = distill_loss(logits, top_ids, top_logits, temperature)   # one number a row
"""
from __future__ import annotations

import weakref

import torch

import paper_2111_00352_amd as gs


def _first_order_only():
    if torch.is_grad_enabled():
        raise RuntimeError("these layers cannot be differentiated twice (create_graph=True)")


def _of(t, like):
    """A gradient in the type of what it belongs to."""
    return None if t is None else t.to(like.dtype)


def _rows(t):
    """A tensor whose rows the library reads: a gradient may be expanded from one number."""
    return None if t is None else t.contiguous()


# The nodes of these layers that were recorded eagerly and still live.  Such a node's graph ties its
# leaves' gradients to the stream it was recorded on, and a capture that goes backwards to the same
# leaves, whatever lies between, would have to wait for that stream, which ends the process where the
# capture does: it is refused instead.
_recorded = weakref.WeakSet()


def _capturing(t) -> bool:
    return isinstance(t, torch.Tensor) and t.is_cuda and torch.cuda.is_current_stream_capturing()


def _record(ctx, of):
    if any(ctx.needs_input_grad) and not _capturing(of):
        _recorded.add(ctx)


def _leaves(tensors, nodes=()) -> dict:
    """The leaves, by id, that tensors and nodes have their gradients from."""
    leaves = {id(t): t for t in tensors if t.requires_grad and t.is_leaf}
    left, seen = [t.grad_fn for t in tensors if t.grad_fn is not None] + list(nodes), set()
    while left:
        node = left.pop()
        if node in seen:
            continue
        seen.add(node)
        if (leaf := getattr(node, "variable", None)) is not None:
            leaves[id(leaf)] = leaf
        left += [n for n, _ in node.next_functions if n is not None]
    return leaves


def _may_record(*inputs):
    """Refuses a capture of inputs whose leaves a graph recorded outside it holds."""
    if not torch.is_grad_enabled() or not _capturing(inputs[0]) or not (held := list(_recorded)):
        return
    mine, others = _leaves([t for t in inputs if t is not None]), _leaves((), held)
    if any(leaf is mine.get(at) for at, leaf in others.items()):
        raise RuntimeError("a graph recorded outside this capture holds the same parameter: delete what it computed first")


class _RmsNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, X, weight, residual, eps):
        _record(ctx, X)
        ctx.set_materialize_grads(False)
        Y, H, r = gs.rms_norm(X, weight, residual, eps)
        ctx.save_for_backward(H, r, weight)
        ctx.residual = residual is not None
        return Y, H if ctx.residual else X.view_as(X)

    @staticmethod
    def backward(ctx, dY, dH):
        _first_order_only()
        H, r, weight = ctx.saved_tensors
        dX, dw = dH, None
        if dY is not None:
            dX, dw = gs.rms_norm_grad(H, r, _rows(dY), weight, _rows(dH))
        return dX, None if weight is None else _of(dw, weight), dX if ctx.residual else None, None


def rms_norm(X, weight=None, residual=None, eps: float = 1e-6):
    """(Y, H): H = X + residual, Y its rows divided by their root mean square, times weight."""
    _may_record(X, weight, residual)
    return _RmsNorm.apply(X, weight, residual, eps)


class _GroupedLinear(torch.autograd.Function):
    @staticmethod
    def forward(ctx, X, W, offsets):
        _record(ctx, X)
        ctx.save_for_backward(X, W, offsets)
        return gs.grouped_matmul(X, W, offsets)

    @staticmethod
    def backward(ctx, dZ):
        _first_order_only()
        X, W, offsets = ctx.saved_tensors
        dZ = _rows(dZ)
        dX = gs.grouped_matmul(dZ, W, offsets, transpose=True) if ctx.needs_input_grad[0] else None
        dW = _of(gs.grouped_weight_grad(X, dZ, offsets), W) if ctx.needs_input_grad[1] else None
        return dX, dW, None


def grouped_linear(X, W, offsets):
    """Rows offsets[g] .. offsets[g+1] - 1 of X times W[g]; X and W of one type."""
    _may_record(X, W)
    return _GroupedLinear.apply(X, W, offsets)


class _NormGroupedLinear(torch.autograd.Function):
    @staticmethod
    def forward(ctx, X, weight, W, offsets, residual, eps):
        _record(ctx, X)
        ctx.set_materialize_grads(False)
        S, H, r = gs.rms_norm(X, weight, residual, eps, save=True)
        ctx.save_for_backward(H, r, weight, W, offsets, S.buffer)
        ctx.residual, ctx.shape = residual is not None, S.shape
        return gs.grouped_matmul(S, W, offsets), H if ctx.residual else X.view_as(X)

    @staticmethod
    def backward(ctx, dZ, dH):
        _first_order_only()
        H, r, weight, W, offsets, codes = ctx.saved_tensors
        dX, dw, dW = dH, None, None
        if dZ is None:
            return dX, None, None, None, dX if ctx.residual else None, None
        dZ = _rows(dZ)
        if ctx.needs_input_grad[2]:
            dW = _of(gs.grouped_weight_grad(gs.SavedActivation(ctx.shape, "none", codes.device, codes), dZ, offsets), W)
        if ctx.needs_input_grad[0] or ctx.needs_input_grad[1] or ctx.needs_input_grad[4]:
            dY = gs.grouped_matmul(dZ, W, offsets, transpose=True, dtype=H.dtype)
            dX, dw = gs.rms_norm_grad(H, r, dY, weight, _rows(dH))
        return dX, None if weight is None else _of(dw, weight), dW, None, dX if ctx.residual else None, None


def norm_grouped_linear(X, weight, W, offsets, residual=None, eps: float = 1e-6):
    """(Z, H): H = X + residual and the products by group of its norm, which is held in 8 bits
    between the forward and the backward pass and read so by the products; its rounding to
    8 bits counts as the identity backwards."""
    _may_record(X, weight, W, residual)
    return _NormGroupedLinear.apply(X, weight, W, offsets, residual, eps)


class _LogProbs(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, ids):
        _record(ctx, logits)
        ctx.set_materialize_grads(False)
        found = gs.log_probs(logits, ids)
        ctx.save_for_backward(logits, ids, found.stats, found.entropy)
        return found.logp, found.entropy

    @staticmethod
    def backward(ctx, dlogp, dentropy):
        _first_order_only()
        logits, ids, stats, entropy = ctx.saved_tensors
        none = stats[:0, 0]
        found = gs.LogProbs(none, entropy, stats, none, none)
        return gs.log_probs_grad(logits, ids, found, _rows(dlogp), _rows(dentropy)), None


def log_probs(logits, ids):
    """(log probability of each row's class, entropy); rows with a negative class have 0 and no
    gradient by it."""
    _may_record(logits)
    return _LogProbs.apply(logits, ids)


class _DistillLoss(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, top_ids, top_logits, temperature):
        _record(ctx, logits)
        loss, stats = gs.distill_loss(logits, top_ids, top_logits, temperature)
        ctx.save_for_backward(logits, top_ids, top_logits, stats)
        ctx.temperature = temperature
        return loss

    @staticmethod
    def backward(ctx, dloss):
        _first_order_only()
        logits, top_ids, top_logits, stats = ctx.saved_tensors
        return gs.distill_grad(logits, top_ids, top_logits, stats, _rows(dloss), ctx.temperature), None, None, None


def distill_loss(logits, top_ids, top_logits, temperature: float = 1.0):
    """A student's loss against a teacher's best classes, one number a row; the teacher has no
    gradient."""
    if top_logits.requires_grad:
        raise ValueError("the teacher's logits have no gradient: detach them")
    _may_record(logits)
    return _DistillLoss.apply(logits, top_ids, top_logits, temperature)
