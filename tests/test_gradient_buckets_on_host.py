"""GradientBuckets without a GPU: whose gradients it clips.  The plan and the kernels behind it are
a plan that remembers its tensors and a clip that copies."""
import types

import pytest
import torch

from paper_2110_04478_amd import binding, gradients


@pytest.fixture
def buckets(monkeypatch):
    clipped = []

    def clip(plan, max_norm):
        clipped.append([g.clone() for g in plan.grads])
        return torch.zeros(2), torch.zeros(len(plan.grads))

    monkeypatch.setattr(binding, "themis_gradient_plan", lambda grads, out=None: types.SimpleNamespace(grads=list(grads), out=out))
    monkeypatch.setattr(binding, "themis_gradient_clip", clip)
    params = [torch.nn.Parameter(torch.ones(3)), torch.nn.Parameter(torch.ones(2, 2))]
    b = gradients.GradientBuckets(params, 1000, dtype=torch.float32)
    b.clipped = clipped
    return b


def backward(params, **kw):
    sum((p * p).sum() for p in params).backward(**kw)


def refused(call):
    with pytest.raises(binding.ThemisError) as e:
        call()
    assert e.value.status == binding.INVALID_ARGUMENT


def test_gradients_in_their_place(buckets):
    for _ in range(2):
        buckets.zero()
        backward(buckets.params)
        buckets.clip(1.0)
        assert all(torch.equal(c, 2 * p.detach()) for c, p in zip(buckets.clipped[-1], buckets.params))


def test_gradients_that_were_dropped(buckets):
    """What optimizer.zero_grad() does: the next backward makes gradients of its own."""
    torch.optim.SGD(buckets.params, lr=0.1).zero_grad()
    refused(lambda: buckets.clip(1.0))
    backward(buckets.params)
    refused(lambda: buckets.clip(1.0))
    assert not buckets.clipped
    buckets.zero()                       # puts them back
    backward(buckets.params)
    buckets.clip(1.0)
    assert all(torch.equal(c, 2 * p.detach()) for c, p in zip(buckets.clipped[-1], buckets.params))


@pytest.mark.filterwarnings("ignore:Using backward")
def test_one_gradient_that_was_replaced(buckets):
    backward(buckets.params, create_graph=True)   # (adds out of place)
    refused(lambda: buckets.clip(1.0))
    buckets.zero()
    buckets.params[1].grad = torch.full((2, 2), 3.0)
    refused(lambda: buckets.clip(1.0))


def test_gradients_that_were_moved(buckets):
    """The tensor is the same, its memory another (Module.to and the like)."""
    buckets.params[0].grad.data = torch.full((3,), 5.0)
    refused(lambda: buckets.clip(1.0))
    refused(buckets.zero)


def test_filled_and_summed(buckets):
    """The gradients as they are; the sum is clipped where it stands."""
    buckets.zero()
    backward(buckets.params)
    buckets.fill()
    assert torch.equal(buckets.buckets[0], torch.full((7,), 2.0)) and not buckets.clipped
    buckets.buckets[0] *= 3.0                         # (three ranks alike)
    buckets.clip_summed(1.0)
    assert [c.tolist() for c in buckets.clipped[-1]] == [[6.0] * 3, [[6.0] * 2] * 2]
    assert buckets.summed.out is None                 # in place
    buckets.params[0].grad = None
    refused(buckets.fill)
