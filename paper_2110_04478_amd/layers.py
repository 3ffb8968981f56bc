"""An expert layer and dropout under torch.autograd: a gate, rows into the order of their
experts and back, elements dropped by a counter.

    weights, chosen = gate(x @ router, k=2)
    order = sort(chosen, n_experts, capacity)
    y = experts(dispatch(x, order))                  # [slots, width]; [n_experts, capacity, width] as a view
    x = dropout(combine(y, order, weights), 0.1, seed, call, add=x)

Differentiable once: a derivative through a gradient raises an error.

A backward can be captured into a graph with its forward while no eager graph of the same leaves lives,
and none that was captured on another stream (torch's engine brings that graph's stream into the capture
and ends the process).  Where such a leaf is an argument of these functions both times the captured call
is refused; of leaves that only other functions read they know nothing."""
from __future__ import annotations

from typing import Optional

import torch
from torch.autograd.function import once_differentiable

from . import binding

sort = binding.themis_expert_sort


def _apply(function, leaves, *args):
    """function.apply(*args); what accumulates the gradients of the leaves among `leaves` is marked
    with the stream of the capture that it was made in, if it was."""
    nodes = []   # (held until the graph holds them)
    if torch.is_grad_enabled():
        for t in leaves:
            if t is not None and t.requires_grad and t.is_leaf:
                nodes.append(torch.autograd.graph.get_gradient_edge(t).node)
                here = None
                if torch.cuda.is_current_stream_capturing():
                    here = torch._C._cuda_getCurrentRawStream(t.get_device()) if t.is_cuda else -1
                made = nodes[-1].metadata.setdefault("captured", here)
                if here is not None and made != here:
                    raise binding.ThemisError(binding.INVALID_ARGUMENT,
                                              "captured while %s graph of the same leaf lives" %
                                              ("an eager" if made is None else "another stream's"))
    return function.apply(*args)


class _Gate(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, k, renormalize, dtype):
        weights, experts = binding.themis_expert_gate(logits, k, renormalize, out_dtype=dtype)
        ctx.save_for_backward(logits, experts)
        ctx.renormalize = renormalize
        ctx.mark_non_differentiable(experts)
        return weights, experts

    @staticmethod
    @once_differentiable
    def backward(ctx, grad_weights, _):
        logits, experts = ctx.saved_tensors
        return binding.themis_expert_gate_grad(grad_weights, logits, experts, ctx.renormalize), None, None, None


def gate(logits: torch.Tensor, k: int, renormalize: bool = True, dtype: torch.dtype = torch.float32) -> tuple:
    """(weights, experts) of the k largest logits (binding.themis_expert_gate); the weights are
    differentiable in the logits, the choice is held."""
    return _apply(_Gate, (logits,), logits, int(k), bool(renormalize), dtype)


class _Dispatch(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, order):
        ctx.save_for_backward(order.place, order.source)   # (an order changed in place is an error)
        ctx.args = order, x.dtype
        return binding.themis_expert_dispatch(x, order)

    @staticmethod
    @once_differentiable
    def backward(ctx, grad):
        ctx.saved_tensors
        order, dtype = ctx.args
        return binding.themis_expert_combine(grad, order, out_dtype=dtype), None


def dispatch(x: torch.Tensor, order: binding.ExpertOrder) -> torch.Tensor:
    """Rows of x in the order of their experts, differentiable in x."""
    return _apply(_Dispatch, (x,), x, order)


class _Combine(torch.autograd.Function):
    @staticmethod
    def forward(ctx, y, weights, order, dtype):
        # (only the weights' gradient reads y)
        ctx.save_for_backward(y if ctx.needs_input_grad[1] else None, weights, order.place, order.source)
        ctx.args = order, y.dtype
        return binding.themis_expert_combine(y, order, weights, out_dtype=dtype)

    @staticmethod
    @once_differentiable
    def backward(ctx, grad):
        y, weights = ctx.saved_tensors[:2]
        order, dtype = ctx.args
        if weights is None:
            return binding.themis_expert_dispatch(grad, order, out_dtype=dtype), None, None, None
        if y is None:   # (of its type and size)
            y = grad.new_empty((1, grad.shape[-1]), dtype=dtype).expand(order.slots, -1)
        rows, products = binding.themis_expert_combine_grad(grad, y, order, weights, ctx.needs_input_grad[0],
                                                            ctx.needs_input_grad[1])
        return rows, products, None, None


def combine(y: torch.Tensor, order: binding.ExpertOrder, weights: Optional[torch.Tensor] = None,
            dtype: Optional[torch.dtype] = None) -> torch.Tensor:
    """The (weighted) sum of every token's rows of y, differentiable in y and the weights."""
    return _apply(_Combine, (y, weights), y, weights, order, dtype)


class _Dropout(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, add, p, seed, call, dtype):
        # (a number that has moved on before the backward is an error, not another mask)
        ctx.save_for_backward(*((call,) if isinstance(call, torch.Tensor) else ()))
        ctx.args = p, seed, call if not isinstance(call, torch.Tensor) else None, x.dtype
        return binding.themis_dropout(x, p, seed, call, add, out_dtype=dtype)

    @staticmethod
    @once_differentiable
    def backward(ctx, grad):
        p, seed, call, dtype = ctx.args
        if call is None:
            (call,) = ctx.saved_tensors
        rows = binding.themis_dropout(grad, p, seed, call, out_dtype=dtype) if ctx.needs_input_grad[0] else None
        return rows, grad if ctx.needs_input_grad[1] else None, None, None, None, None


def dropout(x: torch.Tensor, p: float, seed: int, call, add: Optional[torch.Tensor] = None,
            dtype: Optional[torch.dtype] = None) -> torch.Tensor:
    """add + x / (1 - p) with elements of x dropped (binding.themis_dropout), differentiable in x
    and add.  No mask is kept: the backward draws it again."""
    return _apply(_Dropout, (x, add), x, add, float(p), int(seed), call, dtype)
