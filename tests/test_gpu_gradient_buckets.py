"""The gradient operators under torch.autograd, and an iteration through all of them."""
import importlib.util
import math
import os

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
U = 2.0 ** -24


@pytest.fixture(scope="module")
def gradients():
    if not torch.cuda.is_available():
        pytest.fail("no GPU visible: the gpu-marked tests need an MI355X")
    from paper_2110_04478_amd.csrc.build import ensure_built
    ensure_built()
    from paper_2110_04478_amd import gradients
    return gradients


@pytest.mark.parametrize("into", [False, True])
def test_embedding_under_autograd(gradients, into):
    g = torch.Generator().manual_seed(1)
    table = torch.randn(90, 40, generator=g).cuda().requires_grad_()
    ids = torch.randint(0, 90, (6, 50), generator=g).cuda()
    weight = torch.randn(6, 50, 40, generator=g).cuda()
    table.grad = torch.ones_like(table)
    out = gradients.embedding(table, ids, 1.5, ignored=7, into=table.grad if into else None)
    assert torch.equal(out, table.detach()[ids] * 1.5)
    (out * weight).sum().backward()
    keep = (ids != 7)[..., None].double()
    want = torch.zeros(90, 40, dtype=torch.float64, device="cuda")
    want.index_add_(0, ids.flatten(), (weight.double() * keep).flatten(0, 1)).mul_(1.5).add_(1.0)
    mass = torch.zeros_like(want).index_add_(0, ids.flatten(), weight.double().abs().flatten(0, 1)).mul_(1.5).add_(1.0)
    # 300 terms at most in a sum, the factor and the addition: a rounding each
    assert bool(((table.grad.double() - want).abs() <= 303 * U * mass).all())


def test_buckets_hold_the_clipped_gradients(gradients):
    g = torch.Generator().manual_seed(2)
    params = [torch.nn.Parameter(torch.randn(s, generator=g).cuda()) for s in ((100, 7), (33,), (5, 5, 5), (1,), (4000,))]
    b = gradients.GradientBuckets(params, bucket_bytes=1000, dtype=torch.float32)
    assert b.sizes().tolist() == [4 * 4000, 4 * (1 + 125 + 33 + 700)]
    for k, p in enumerate(params):
        p.grad.copy_(torch.randn(p.shape, generator=g) * 10.0 ** -k)
    total, norms = b.clip(0.25)
    want = torch.stack([p.grad.double().square().sum() for p in params]).cpu()
    assert bool(((norms.double().cpu() - want.sqrt()).abs() <= 2 * U * want.sqrt()).all())
    norm = want.sum().sqrt().item()
    assert abs(total[0].item() - norm) <= 2 * U * norm
    flat = torch.cat([p.grad.flatten() for p in (params[4], params[3], params[2], params[1], params[0])]).double()
    got = torch.cat([x for x in b.buckets]).double()
    assert bool(((got - flat * (0.25 / norm)).abs() <= 4 * U * flat.abs() * (0.25 / norm)).all())
    b.zero()
    assert not any(p.grad.any() for p in params)


def test_a_training_iteration(gradients):
    spec = importlib.util.spec_from_file_location("training_iteration", os.path.join(ROOT, "examples", "training_iteration.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    got = example.main(steps=30, vocab=300, width=64, batch=8, length=48)
    assert all(math.isfinite(x) for x in got["losses"] + got["norms"])
    assert got["losses"][-1] < got["losses"][0] - 0.5          # it learns
    assert got["sizes"].sum() == 2 * (300 * 64 + 2 * 4 * 64 * 64)
    baseline, fifo, scf = got["times"]
    assert np.isfinite(got["times"]).all() and (got["times"] > 0).all()
    assert scf.mean() < baseline.mean()
    # one step by hand: the same model in plain torch, gradients and norm in binary32
    p = example.model(300, 64, "cuda:0", 1)
    tokens = example.batch_of(300, 8, 48, "cuda:0", 0)
    table, up, down = (p[k].detach().clone().double().requires_grad_() for k in ("table", "up", "down"))
    ids = tokens[:, :-1]
    x = table[ids] * math.sqrt(64)
    x = torch.where((ids == example.PAD)[..., None], x.detach(), x)
    x = x + torch.relu(x @ up.t()) @ down.t()
    x = x / (x.square().mean(-1, keepdim=True) + 1e-6).sqrt()
    logits = x @ table.t()
    loss = torch.nn.functional.cross_entropy(logits.flatten(0, 1), tokens[:, 1:].flatten(), ignore_index=example.PAD)
    loss.backward()
    norm = torch.cat([t.grad.flatten() for t in (table, up, down)]).norm().item()
    # (binary32 products over up to 376 tokens and 256 elements: far within 1e-3)
    assert abs(got["losses"][0] - loss.item()) < 1e-3 * loss.item()
    assert abs(got["norms"][0] - norm) < 1e-3 * norm


@pytest.mark.parametrize("n", [3, 5000])
def test_workspaces_elsewhere_are_refused(gradients, n):
    """Host memory, and memory with gaps or of one element that a stride of zero makes long."""
    binding = gradients.binding
    ids = torch.zeros(n, dtype=torch.int64, device="cuda")
    g = torch.zeros((n, 8), device="cuda")
    need = 2 * max(16, binding.themis_embedding_grad_workspace_bytes(n, 8, 5))
    for work in (torch.empty(need, dtype=torch.uint8), torch.empty(need, dtype=torch.uint8, device="cuda")[::2],
                 torch.empty(1, dtype=torch.uint8, device="cuda").expand(need)):
        with pytest.raises(binding.ThemisError) as e:
            binding.themis_embedding_grad(g, ids, 5, workspace=work)
        assert e.value.status == -1


def test_embedding_is_differentiable_once(gradients):
    """A second derivative is an error, not a graph that ends without one."""
    table = torch.ones((5, 8), device="cuda", requires_grad=True)
    ids = torch.tensor([1, 4, 1], device="cuda")
    out = gradients.embedding(table, ids)
    (grad,) = torch.autograd.grad(out.square().sum(), table, create_graph=True)
    assert torch.equal(grad.detach()[:, 0].cpu(), torch.tensor([0.0, 4.0, 0.0, 0.0, 2.0]))
    with pytest.raises(RuntimeError):
        grad.sum().backward()
