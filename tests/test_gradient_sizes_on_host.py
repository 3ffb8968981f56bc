"""Sizes and workspaces of the table's gradient that are refused, without a GPU."""
import pytest

from test_gradients_on_host import FAKE, F32, I64, binding, rows  # noqa: F401

MOST = (1 << 31) - 1


def call(binding, n, width, vocab, work, work_bytes):  # noqa: F811
    return binding.lib().themis_embedding_grad(rows(binding, F32, inner=1 << 31, inner_stride=width), width,
                                               rows(binding, I64, inner=1 << 31, inner_stride=1), n, 1.0, -1, 0,
                                               rows(binding, F32, inner=1 << 31, inner_stride=width), vocab,
                                               work, work_bytes, None)


@pytest.mark.parametrize("n,width,vocab", [(1 << 20, (1 << 24) + 1, 1000), (1 << 26, 1 << 20, 1000), (4097, 1 << 26, 7),
                                           (MOST, 1 << 16, MOST), (1 << 31, 8, 8), (5, 1 << 31, 8)])
def test_sizes_beyond_the_grids(binding, n, width, vocab):  # noqa: F811
    """Unsupported, whatever the workspace, and none is asked for."""
    assert binding.lib().themis_embedding_grad_workspace_bytes(n, width, vocab) == 0
    assert call(binding, n, width, vocab, None, 0) == -2
    assert call(binding, n, width, vocab, FAKE, 1 << 60) == -2


@pytest.mark.parametrize("n,width,vocab", [(4097, 8, 10), (5000, 65, 1023), (200000, 4096, 1 << 20)])
def test_workspaces_that_are_refused(binding, n, width, vocab):  # noqa: F811
    need = binding.lib().themis_embedding_grad_workspace_bytes(n, width, vocab)
    assert need > 8 * n
    assert call(binding, n, width, vocab, None, need) == -4
    assert call(binding, n, width, vocab, FAKE, need - 1) == -4
    assert call(binding, n, width, vocab, FAKE + 8, need) == -4
