"""A worker's layers with their gradients, as torch.autograd functions around the library's operators.

`layer_norm`, and the three steps of a layer of experts: `route` (which row each token's copies go to), `dispatch`
(the copies) and `combine` (the weighted sum back).  What the experts compute in between is the caller's.  Tensors are
float32 or bfloat16 on a CUDA device, all of a call on the same one; everything runs in the library's kernels, on copies
of inputs whose strides these do not take.  There are no second derivatives: asking for them raises an error.
"""
from __future__ import annotations

import functools
from dataclasses import dataclass

import torch
from torch.autograd.function import once_differentiable

from . import binding as sgdb


def _on_its_device(call):
    """The call with the device of its first tensor as the current one, which is where the library launches."""
    @functools.wraps(call)
    def wrapped(*args):
        x = args[0] if isinstance(args[0], torch.Tensor) else args[1]  # behind an autograd context
        if not x.is_cuda or x.get_device() == torch.cuda.current_device():
            return call(*args)
        with torch.cuda.device(x.device):
            return call(*args)
    return wrapped


def _rows(x):
    """x itself where its rows are contiguous and do not overlap, else a copy."""
    T, D = x.shape
    fine = (D <= 1 or x.stride(1) == 1) and (T <= 1 or x.stride(0) >= D)
    return x if fine else x.contiguous()


def _as_new(x):
    """x itself where its rows lie against 16-byte boundaries as those of a new tensor do, else a copy: layer norm's kernels are
    slow when dy lies otherwise than x, and bound by the edges of chunks where x's rows need not have any."""
    T, D = x.shape
    x = _rows(x)
    alike = x.data_ptr() % 16 == 0 and (T <= 1 or (x.stride(0) - D) * x.element_size() % 16 == 0)
    return x if alike else torch.empty_like(x, memory_format=torch.contiguous_format).copy_(x)


class _LayerNorm(torch.autograd.Function):
    @staticmethod
    @_on_its_device
    def forward(ctx, x, gamma, beta, eps):
        rows = _as_new(x.reshape(-1, x.size(-1)))
        gamma = None if gamma is None else gamma.contiguous()
        beta = None if beta is None else beta.contiguous()
        y = torch.empty_like(rows, memory_format=torch.contiguous_format)
        mean = torch.empty(rows.size(0), dtype=torch.float32, device=x.device)
        rstd = torch.empty_like(mean)
        sgdb.sgdb_layer_norm(rows, gamma, beta, eps, y, mean, rstd)
        ctx.save_for_backward(rows, gamma, beta, mean, rstd)
        return y.view(x.shape)

    @staticmethod
    @once_differentiable
    @_on_its_device
    def backward(ctx, dy):
        rows, gamma, beta, mean, rstd = ctx.saved_tensors
        dx = torch.empty_like(rows, memory_format=torch.contiguous_format)
        dgamma = torch.empty_like(gamma) if gamma is not None and ctx.needs_input_grad[1] else None
        dbeta = torch.empty_like(beta) if beta is not None and ctx.needs_input_grad[2] else None
        workspace = None
        if dgamma is not None or dbeta is not None:
            need = sgdb.sgdb_layer_norm_backward_workspace_bytes(*rows.shape)
            workspace = torch.empty(need, dtype=torch.uint8, device=rows.device)
        sgdb.sgdb_layer_norm_backward(_as_new(dy.reshape(rows.shape)), rows, gamma, mean, rstd, dx, dgamma, dbeta, workspace)
        return dx.view(dy.shape), dgamma, dbeta, None


def layer_norm(x, gamma=None, beta=None, eps: float = 1e-5):
    """(x - mean) / sqrt(var + eps) * gamma + beta over the last dimension."""
    return _LayerNorm.apply(x, gamma, beta, eps)


@dataclass
class Route:
    """Where each token's copies go: expert e owns the rows offsets[e] .. offsets[e + 1] - 1."""
    offsets: torch.Tensor  # int32 [experts + 1]
    slot: torch.Tensor     # int32 [tokens, k]: the copy's row, -1 when dropped
    source: torch.Tensor   # int32 [tokens * k]: the row's copy (token * k + choice), -1 when not in use


@_on_its_device
def route(expert, experts: int) -> Route:
    """expert int32 [tokens, k]: each token's choices; one outside [0, experts) is dropped."""
    tokens, k = expert.shape
    new = lambda *shape: torch.empty(shape, dtype=torch.int32, device=expert.device)  # noqa: E731
    r = Route(new(experts + 1), new(tokens, k), new(tokens * k))
    sgdb.sgdb_route(expert.contiguous(), experts, r.offsets, r.slot, r.source)
    return r


class _Dispatch(torch.autograd.Function):
    @staticmethod
    @_on_its_device
    def forward(ctx, x, slot, offsets):
        x = _rows(x)
        xs = torch.empty(slot.numel(), x.size(1), dtype=x.dtype, device=x.device)
        sgdb.sgdb_dispatch(x, slot, offsets, xs)
        ctx.save_for_backward(slot)
        return xs

    @staticmethod
    @once_differentiable
    @_on_its_device
    def backward(ctx, dxs):
        (slot,) = ctx.saved_tensors
        dx = torch.empty(slot.size(0), dxs.size(1), dtype=dxs.dtype, device=dxs.device)
        sgdb.sgdb_combine(dxs.contiguous(), slot, None, dx)
        return dx, None, None


def dispatch(x, r: Route):
    """x [tokens, width] -> the experts' rows [tokens * k, width]; rows not in use are zero."""
    return _Dispatch.apply(x, r.slot, r.offsets)


class _Combine(torch.autograd.Function):
    @staticmethod
    @_on_its_device
    def forward(ctx, ys, weights, slot, offsets):
        ys = ys.contiguous()
        weights = None if weights is None else weights.contiguous()
        out = torch.empty(slot.size(0), ys.size(1), dtype=ys.dtype, device=ys.device)
        sgdb.sgdb_combine(ys, slot, weights, out)
        ctx.save_for_backward(ys, weights, slot, offsets)
        return out

    @staticmethod
    @once_differentiable
    @_on_its_device
    def backward(ctx, dout):
        ys, weights, slot, offsets = ctx.saved_tensors
        dys = torch.empty_like(ys)
        dweights = torch.empty_like(weights) if weights is not None and ctx.needs_input_grad[1] else None
        sgdb.sgdb_combine_backward(dout.contiguous(), ys, slot, weights, offsets, dys, dweights)
        return dys, dweights, None, None


def combine(ys, weights, r: Route):
    """The experts' rows [tokens * k, width] added up per token with weights float32 [tokens, k] (None: ones)."""
    return _Combine.apply(ys, weights, r.slot, r.offsets)
