"""The example of a training iteration on several ranks: the norm is that of the ranks' sum."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    if not torch.cuda.is_available():
        pytest.fail("no GPU visible: the gpu-marked tests need an MI355X")
    spec = importlib.util.spec_from_file_location("training_iteration", os.path.join(ROOT, "examples", "training_iteration.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.mark.parametrize("ranks", [1, 2, 4])
def test_the_norm_of_the_sum(example, ranks):
    """Ranks with equal gradients: the buckets come back as a multiple, and so does the norm.  (The same
    step in two runs: matrix products whose order of sums may differ are far within 1e-5.)"""
    sums = []

    def all_reduce(buckets):
        for b in buckets:
            b.mul_(ranks)
        sums.append(torch.cat(buckets).double().norm().item())

    sizes = dict(steps=1, vocab=300, width=64, batch=8, length=48)
    one = example.main(**sizes)["norms"][0]
    got = example.main(**sizes, max_norm=0.25, all_reduce=all_reduce)
    # binary64 sums rounded to binary32
    assert abs(got["norms"][0] - sums[0]) <= 2.0 ** -23 * sums[0]
    assert abs(got["norms"][0] - ranks * one) <= 1e-5 * ranks * one


def test_buckets_are_clipped_by_the_norm_of_the_sum():
    from paper_2110_04478_amd.gradients import GradientBuckets
    g = torch.Generator().manual_seed(4)
    params = [torch.nn.Parameter(torch.randn(s, generator=g).cuda()) for s in ((300, 7), (33,), (4001,))]
    b = GradientBuckets(params, bucket_bytes=1000, dtype=torch.float32)
    own = [torch.randn(p.shape, generator=g).cuda() for p in params]
    other = [torch.randn(x.numel(), generator=g).cuda() for x in b.buckets]
    for p, x in zip(params, own):
        p.grad.copy_(x)
    b.fill()
    for x, y in zip(b.buckets, other):
        x += y
    want = torch.cat(b.buckets).double()
    norm = want.norm().item()
    total, norms = b.clip_summed(0.5)
    # norm and factor are rounded once, the product twice
    assert abs(total[0].item() - norm) <= 2.0 ** -23 * norm
    assert bool(((torch.cat(b.buckets).double() - want * (0.5 / norm)).abs() <= 4 * 2.0 ** -24 * want.abs() * (0.5 / norm)).all())
    assert abs(norms.double().norm().item() - norm) <= 2.0 ** -22 * norm
    assert all(torch.equal(p.grad, x) for p, x in zip(params, own))
