"""The example of a training iteration with experts and dropout: it runs, its gradients are those of the
formulas and reach the buckets."""
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


def test_it_runs_and_its_buckets_are_a_trace(example):
    got = example.main(steps=3, vocab=300, width=64, batch=8, length=48, experts=4, dropout=0.1)
    assert len(got["losses"]) == 3 and all(0 < x < float("inf") for x in got["losses"] + got["norms"])
    assert got["sizes"].sum() == 2 * (300 * 64 + 4 * 64 + 2 * 4 * 64 * 256) and (got["times"] > 0).all()


def test_its_gradients(example):
    """Of the experts' layer alone, against autograd in binary64 on the same choice and mask: chains of sums
    of at most 256 terms (products with the weights), each within 256 u of its magnitudes, ten links."""
    from paper_2110_04478_amd import layers
    from test_gpu_dropout import kept_of
    width, n_experts, n = 32, 4, 48
    p = example.model(50, width, "cuda", 3, n_experts)
    x = torch.randn((2, n // 2, width), generator=torch.Generator().manual_seed(5)).cuda().requires_grad_()
    y = example.feed_forward(p, x)
    out = layers.dropout(y, 0.25, example.SEED, 7, add=x)
    names = ("router", "up", "down")
    g = torch.randn(out.shape, generator=torch.Generator().manual_seed(6)).cuda()
    got = torch.autograd.grad(out, [x] + [p[k] for k in names], g)
    _, chosen = layers.gate(x.detach() @ p["router"].detach().t(), example.CHOSEN)
    capacity = -(-int(example.CAPACITY * example.CHOSEN * n) // n_experts)
    place = layers.sort(chosen, n_experts, capacity).place.cpu().view(n, -1)
    chosen = chosen.cpu().long().view(n, -1)
    z, q = x.detach().cpu().double().requires_grad_(), {k: p[k].detach().cpu().double().requires_grad_() for k in names}
    rows = z.view(n, width)
    weights = torch.softmax((rows @ q["router"].t()).gather(1, chosen), 1)
    want = torch.zeros_like(rows)
    for j in range(example.CHOSEN):
        mine = torch.stack([torch.relu(r @ q["up"][e]) @ q["down"][e] for r, e in zip(rows, chosen[:, j].tolist())])
        want = want + torch.where(place[:, j, None] >= 0, weights[:, j, None] * mine, 0.0)
    kept = torch.from_numpy(kept_of(n, width, 0.25, example.SEED, 7))
    want = (rows + torch.where(kept, want / 0.75, 0.0)).view(x.shape)
    for a, b in zip(got, torch.autograd.grad(want, [z] + [q[k] for k in names], g.cpu().double())):
        assert float((a.cpu().double() - b).abs().max()) <= 2560 * 2.0 ** -24 * float(b.abs().max())


@pytest.mark.parametrize("experts", [1, 2, 3])
def test_few_experts(example, experts):
    """Fewer than a token's choices, too; of one expert the layer is that expert's, every weight 1."""
    got = example.main(steps=2, vocab=100, width=32, batch=4, length=24, experts=experts, dropout=0.1)
    assert all(0 < x < float("inf") for x in got["losses"] + got["norms"])
    if experts == 1:
        p = example.model(50, 32, "cuda", 3, 1)
        x = torch.randn((2, 20, 32), generator=torch.Generator().manual_seed(5)).cuda()
        y = example.feed_forward(p, x).detach().cpu().double()
        z, up, down = x.cpu().double(), p["up"][0].detach().cpu().double(), p["down"][0].detach().cpu().double()
        want = torch.relu(z @ up) @ down
        # sums of 32 and 128 terms in binary32 (and the sign of a hidden value below its error), relative to
        # the terms' magnitudes
        size = (z.abs() @ up.abs()) @ down.abs()
        assert bool(((y - want).abs() <= (32 + 128 + 8) * 2.0 ** -24 * size).all())
