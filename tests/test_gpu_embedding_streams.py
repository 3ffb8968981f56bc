"""embedding(into=...) where the lookup's stream, the accumulation's and the caller's are not one."""
import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


@pytest.fixture(scope="module")
def gradients():
    if not torch.cuda.is_available():
        pytest.fail("no GPU visible: the gpu-marked tests need an MI355X")
    from paper_2110_04478_amd.csrc.build import ensure_built
    ensure_built()
    from paper_2110_04478_amd import gradients
    return gradients


@pytest.mark.parametrize("tied", [False, True])
@pytest.mark.parametrize("n", [300, 6000])
def test_the_caller_reads_the_whole_gradient(gradients, n, tied):
    """The lookup runs on a stream of its own, and its gradient comes late there; what the caller's
    stream reads behind backward() is complete."""
    vocab, width = 500, 64
    g = torch.Generator().manual_seed(n)
    table = torch.nn.Parameter(torch.randn(vocab, width, generator=g).cuda())
    table.grad = torch.zeros_like(table)
    ids = torch.randint(0, vocab, (n,), generator=g).cuda()
    weight = torch.randn(n, width, generator=g).cuda()
    slow = torch.full((4096, 4096), 2.0 ** -12, device="cuda")   # (a product with it keeps a matrix of ones)
    node = torch.autograd.graph.get_gradient_edge(table).node     # on the caller's stream
    other = torch.cuda.Stream()
    for k in range(3):
        table.grad.zero_()
        other.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(other):
            x = gradients.embedding(table, ids, 1.5, into=table.grad)
            def late(grad):
                one = torch.ones(4096, 4096, device="cuda")
                for _ in range(20):
                    one = one @ slow
                return grad * one[0, 0]

            x.register_hook(late)
            loss = (x * weight).sum()
        torch.cuda.current_stream().wait_stream(other)
        if tied:
            loss = loss + 2.0 * table.sum()
        loss.backward()
        got = table.grad.clone()                                  # at once, on the caller's stream
        want = torch.zeros(vocab, width, dtype=torch.float64, device="cuda")
        want.index_add_(0, ids, weight.double()).mul_(1.5).add_(2.0 if tied else 0.0)
        mass = torch.zeros_like(want).index_add_(0, ids, weight.double().abs()).mul_(1.5).add_(2.0)
        # fewer than 300 terms in a sum, the factor and the addition: a rounding each
        assert bool(((got.double() - want).abs() <= 303 * U * mass).all()), k
    assert torch.equal(got, table.grad)
    del node
