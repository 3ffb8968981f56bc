"""Between torch.autograd, the gradient operators and the evaluator's traces: a
token table whose gradient the library sums, and the flat buckets that an
iteration's collectives carry."""
from __future__ import annotations

import contextlib
from typing import Optional

import numpy as np
import torch
from torch.autograd.function import once_differentiable

from . import binding


@contextlib.contextmanager
def _behind(stream, *tensors):
    """The current stream of the tensors' GPU waits for what has been put on `stream`."""
    with torch.cuda.device(tensors[0].device):
        here = torch.cuda.current_stream()
        if here != stream:
            here.wait_stream(stream)
            for t in tensors:
                t.record_stream(here)
        yield


def _current_stream(t: torch.Tensor):
    return torch.cuda.current_stream(t.device)


class _Embedding(torch.autograd.Function):
    @staticmethod
    def forward(ctx, table, ids, scale, ignored, into, node):
        ctx.save_for_backward(ids)
        ctx.args = (table.shape[0], table.dtype, scale, ignored, into, node)
        return binding.themis_embedding_lookup(table, ids, scale)

    @staticmethod
    @once_differentiable
    def backward(ctx, grad_out):
        (ids,) = ctx.saved_tensors
        vocab, dtype, scale, ignored, into, node = ctx.args
        if into is not None:
            _add_later(grad_out, ids, vocab, scale, ignored, into, node)
            return None, None, None, None, None, None
        grad = binding.themis_embedding_grad(grad_out, ids, vocab, scale, ignored, out_dtype=dtype)
        return grad, None, None, None, None, None


def _add_later(grad_out, ids, vocab, scale, ignored, into, node):
    """Adds the gradient to `into` where the table's own gradient is accumulated: behind whatever else
    this backward accumulates there, on that stream, which the caller's waits for; and before hooks on the
    accumulated gradient.  Where nothing is accumulated (a table that is not a leaf, torch.autograd.grad)
    at the end of this backward, on the caller's stream."""
    stream, task, left = _current_stream(grad_out), torch._C._current_graph_task_id(), [True]

    def add():
        if not left:
            return
        left.clear()
        with _behind(stream, grad_out, ids):
            binding.themis_embedding_grad(grad_out, ids, vocab, scale, ignored, out=into, accumulate=True)
        torch.autograd.graph.increment_version(into)

    def before_accumulation(_):
        hook.remove()
        if torch._C._current_graph_task_id() == task:   # (not so behind a backward that failed on its way)
            add()

    def at_the_end():
        if hook is not None:
            hook.remove()
        add()

    hook = node.register_prehook(before_accumulation) if node is not None else None
    torch.autograd.Variable._execution_engine.queue_callback(at_the_end)


def embedding(table: torch.Tensor, ids: torch.Tensor, scale: float = 1.0, ignored: int = -1,
              into: Optional[torch.Tensor] = None) -> torch.Tensor:
    """scale * table[ids], differentiable in the table; tokens of number `ignored` have no gradient.

    into: where the gradient is added in place of being returned to autograd (table.grad, say: a
    table that is also the output projection has one already, and only the rows of the tokens at
    hand are touched).  The addition is a change in place of `into` by every backward through the result,
    torch.autograd.grad's among them, whose result for the table lacks it.  Differentiable once: a
    derivative through the gradient raises an error."""
    node = None
    if into is not None and table.requires_grad and table.is_leaf and torch.is_grad_enabled():
        node = torch.autograd.graph.get_gradient_edge(table).node
    return _Embedding.apply(table, ids, float(scale), int(ignored), into, node)


class GradientBuckets:
    """The gradients of a list of parameters, and the flat buckets that carry them.

    The buckets hold the last parameter's gradient first, as gradients become ready, each at least
    bucket_bytes unless it is the last.  Two ways to clip, which are the same on one rank only:

        fill(); sum the buckets over the ranks; clip_summed(max_norm)   the norm of all ranks' sum
        clip(max_norm); sum the buckets over the ranks                  each rank's own norm

    Every parameter gets a .grad of zeros that has to stay: zero_grad(set_to_none=True), a backward
    with create_graph and moves of the module put others in its place, and fill() and clip() are errors
    until zero() has put these back (after moves of the module: new buckets)."""

    def __init__(self, params, bucket_bytes: int, dtype: torch.dtype = torch.bfloat16):
        self.params = [p for p in params if p.requires_grad]
        if not self.params:
            raise binding.ThemisError(binding.INVALID_ARGUMENT)
        self.buckets, groups, size = [], [[]], 0
        for p in reversed(self.params):
            p.grad = torch.zeros_like(p, memory_format=torch.contiguous_format)
            if size >= bucket_bytes:
                groups.append([])
                size = 0
            groups[-1].append(p)
            size += p.numel() * dtype.itemsize
        self.views = {}
        for group in groups:
            flat = torch.zeros(sum(p.numel() for p in group), dtype=dtype, device=group[0].device)
            for p, part in zip(group, flat.split([p.numel() for p in group])):
                self.views[p] = part.view(p.shape)
            self.buckets.append(flat)
        self.plan = binding.themis_gradient_plan([p.grad for p in self.params],
                                                 [self.views[p] for p in self.params])
        self.summed = binding.themis_gradient_plan([self.views[p] for p in self.params])
        self.places = [g.data_ptr() for g in self.plan.grads]

    def _stays(self) -> bool:
        return all(g.data_ptr() == at for g, at in zip(self.plan.grads, self.places))

    def zero(self):
        binding._need(self._stays())
        for p, g in zip(self.params, self.plan.grads):
            p.grad = g.zero_()

    def _need_gradients(self):
        binding._need(self._stays() and all(p.grad is g for p, g in zip(self.params, self.plan.grads)))

    def fill(self):
        """The gradients into the buckets as they are."""
        self._need_gradients()
        torch._foreach_copy_([self.views[p] for p in self.params], self.plan.grads)

    def clip_summed(self, max_norm: float):
        """What the buckets hold clipped in place -> (f32[2]: norm and factor, norms of the
        parameters' parts f32[n])."""
        return binding.themis_gradient_clip(self.summed, max_norm)

    def clip(self, max_norm: float):
        """This rank's gradients, clipped, into the buckets -> (f32[2]: norm and factor, norms of the
        parameters' gradients f32[n])."""
        self._need_gradients()
        return binding.themis_gradient_clip(self.plan, max_norm)

    def sizes(self) -> np.ndarray:
        """Bytes of the buckets: the collectives of an iteration, in the order of their issue."""
        return np.array([b.numel() * b.element_size() for b in self.buckets], dtype=np.float64)
