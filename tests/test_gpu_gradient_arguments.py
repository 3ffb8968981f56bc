"""Arguments of the gradient operators that are refused, and their neighbours that are not."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def gpu():
    if not torch.cuda.is_available():
        pytest.fail("no GPU visible: the gpu-marked tests need an MI355X")
    from paper_2110_04478_amd import binding
    from paper_2110_04478_amd.csrc.build import ensure_built
    ensure_built()
    return binding


def refused(gpu, call):
    with pytest.raises(gpu.ThemisError) as e:
        call()
    assert e.value.status == -1


@pytest.mark.parametrize("n", [9, 5000])
def test_results_on_what_is_read(gpu, n):
    """A lookup into its own table, a gradient on the rows that are summed: refused; beside them,
    in the same matrix: not."""
    big = torch.randn(2 * n, 40, device="cuda")
    ids = torch.arange(n, device="cuda") // 2
    before = big.clone()
    refused(gpu, lambda: gpu.themis_embedding_lookup(big, ids, out=big[:n]))
    refused(gpu, lambda: gpu.themis_embedding_lookup(big[:, :16], ids, out=big[n:, 8:24]))
    refused(gpu, lambda: gpu.themis_embedding_grad(big[:n], ids, n, out=big[n - 1:2 * n - 1]))
    refused(gpu, lambda: gpu.themis_embedding_grad(big[:n, :16], ids, n, out=big[:n, 15:31], accumulate=True))
    assert torch.equal(big, before)
    gpu.themis_embedding_lookup(big[:, :16], ids, 2.0, out=big[n:, 16:32])
    assert torch.equal(big[n:, 16:32], 2.0 * before[ids, :16])
    gpu.themis_embedding_grad(big[:n, :8], ids, n, out=big[:n, 8:16], accumulate=True)
    want = before[:n, 8:16].double().index_add_(0, ids, before[:n, :8].double())
    # two terms and what was held: an addition each
    mass = before[:n, 8:16].double().abs().index_add_(0, ids, before[:n, :8].double().abs())
    assert bool(((big[:n, 8:16].double() - want).abs() <= 4 * 2.0 ** -24 * mass).all())
