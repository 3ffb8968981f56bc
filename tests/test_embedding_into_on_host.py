"""embedding(into=...) without a GPU: when the gradient is added, and that autograd knows of it.
Lookup, gradient and streams are stand-ins."""
import contextlib

import pytest
import torch

from paper_2110_04478_amd import binding, gradients


@pytest.fixture
def added(monkeypatch):
    log = []

    def grad(grad_out, ids, vocab, scale, ignored, out=None, out_dtype=None, accumulate=False):
        keep = (ids != ignored)[..., None]
        if not accumulate:
            out = torch.zeros(vocab, grad_out.shape[-1])
        else:
            log.append(torch._C._current_autograd_node())
        out.numpy()[:] += torch.zeros_like(out).index_add_(0, ids.flatten(), (grad_out * keep).flatten(0, -2)).numpy() * scale
        return out

    monkeypatch.setattr(binding, "themis_embedding_lookup", lambda table, ids, scale: table.detach()[ids] * scale)
    monkeypatch.setattr(binding, "themis_embedding_grad", grad)
    monkeypatch.setattr(gradients, "_behind", lambda *_: contextlib.nullcontext(), raising=False)
    monkeypatch.setattr(gradients, "_current_stream", lambda t: None, raising=False)
    return log


def tied(grad=True):
    table = torch.nn.Parameter(torch.arange(12.0).view(4, 3))
    if grad:
        table.grad = torch.zeros(4, 3)
    return table, torch.tensor([1, 3, 1])


def test_autograd_knows_of_the_addition(added):
    """A gradient that a graph holds on to has changed: an error, not another number."""
    table, ids = tied()
    w = torch.ones(4, 3, requires_grad=True)
    penalty = (table.grad * w).sum()
    before = table.grad._version
    gradients.embedding(table, ids, into=table.grad).sum().backward()
    assert table.grad._version > before
    assert table.grad[:, 0].tolist() == [0, 2, 0, 1]
    with pytest.raises(RuntimeError):
        penalty.backward()


def test_the_addition_is_part_of_the_accumulation(added):
    """In turn with what autograd itself accumulates, whichever stream that is on, and before its hooks."""
    table, ids = tied()
    seen = []
    table.register_post_accumulate_grad_hook(lambda t: seen.append(t.grad.clone()))
    for k in range(3):
        x = gradients.embedding(table, ids, 2.0, into=table.grad) + gradients.embedding(table, ids[:1], into=table.grad)
        (x.sum() + 5.0 * table.sum()).backward()
    assert [type(n).__name__ for n in added] == ["AccumulateGrad"] * 6
    assert [s[:, 0].tolist() for s in seen] == [[5 * k, (5 + 7) * k, 5 * k, (5 + 2) * k] for k in (1, 2, 3)]
    assert torch.equal(seen[-1], table.grad)


def test_where_nothing_is_accumulated(added):
    table, ids = tied()
    into = torch.zeros(4, 3)
    x = gradients.embedding(table * 1.0, ids, into=into)
    x.sum().backward()
    assert into[:, 0].tolist() == [0, 2, 0, 1] and len(added) == 1
    x = gradients.embedding(table, ids, into=into)
    torch.autograd.grad(x.sum(), table, allow_unused=True)
    assert into[:, 0].tolist() == [0, 4, 0, 2] and len(added) == 2
    (gradients.embedding(table, ids, into=into).sum() + table.sum()).backward()
    assert into[:, 0].tolist() == [0, 6, 0, 3] and len(added) == 3


def test_behind_a_backward_that_failed(added):
    """Nothing of it is left for the next one."""
    table, ids = tied()

    def fail(_):
        raise ValueError

    first = table * 2.0
    x = gradients.embedding(table, ids, 7.0, into=table.grad)   # (made last, so its gradient is first)
    y = first.sum() + x.sum()
    first.register_hook(fail)
    with pytest.raises(ValueError):
        y.backward()
    assert not added
    (gradients.embedding(table, ids, into=table.grad).sum() + table.sum()).backward()
    assert table.grad[:, 0].tolist() == [1, 3, 1, 2] and len(added) == 1


def test_without_into(added):
    table, ids = tied(grad=False)
    gradients.embedding(table, ids, 3.0, ignored=3).sum().backward()
    assert table.grad[:, 0].tolist() == [0, 6, 0, 0]
    with torch.no_grad():
        assert not gradients.embedding(table, ids, into=table.grad).requires_grad
    assert not gradients.embedding(table.detach(), ids, into=table.grad).requires_grad and not added
