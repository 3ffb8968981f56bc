"""Which targets of a list of gradients share memory: against the sets of their bytes, and the
lists whose clipping would scale an element twice."""
import random

import pytest
import torch

from paper_2110_04478_amd import binding, overlap


def bytes_of(t):
    at = torch.zeros((), dtype=torch.int64)
    for n, s in zip(t.shape, t.stride()):
        at = at[..., None] + torch.arange(n) * s
    at = (at.flatten() * t.element_size()).tolist()
    return [t.data_ptr() + a + k for a in at for k in range(t.element_size())]


def view_in(r, base):
    """Some view of a flat array: slices, steps, windows, transposed, of up to four levels."""
    while True:
        dims = r.randint(0, 4)
        shape = [r.choice((1, 2, 3, 4, 7)) for _ in range(dims)]
        strides = [r.choice((0, 1, 1, 2, 3, 4, 5, 8, 12, 24, 60)) for _ in range(dims)]
        reach = sum((n - 1) * s for n, s in zip(shape, strides))
        if reach < base.numel():
            return torch.as_strided(base, shape, strides, r.randint(0, base.numel() - 1 - reach))


@pytest.mark.parametrize("seed", range(8))
def test_against_the_bytes_themselves(seed):
    r = random.Random(seed)
    base = torch.zeros(200)
    half = base.view(torch.bfloat16)
    yes = 0
    for _ in range(400):
        views = [view_in(r, r.choice((base, base, half))) for _ in range(r.randint(1, 5))]
        cut = r.randint(0, len(views))
        for t in views:
            assert overlap.repeats(t) == (len(set(bytes_of(t))) != t.numel() * t.element_size())
        sets = [set(bytes_of(t)) for t in views]
        want = any(sets[i] & sets[j] for i in range(cut) for j in range(i + 1, len(views)))
        assert overlap.shared([overlap.view_of(t) for t in views[:cut]], [overlap.view_of(t) for t in views[cut:]]) == want
        yes += want
    assert 40 < yes < 400


def test_lists_with_gaps_that_share_elements():
    base, a, c = torch.zeros(8, 12), torch.zeros(8, 5), torch.zeros(8, 12)
    weight = torch.zeros(12, 16)
    windows = torch.zeros(64).as_strided((2, 2, 4), (6, 5, 1))
    for grads in ([base, base[:, :5]], [base[:, :5], base[:, 3:8]], [base, base.t()], [windows],
                  [weight[:, :12].unfold(0, 4, 2)], [base[:6, :9], base[3:, :9]], [base[::2], base[::3]], [base[:1, :3].expand(5, 3)]):
        assert binding._targets_share(grads, grads), [g.shape for g in grads]
    assert binding._targets_share([a, base], [base[:, :5], c])      # a target on another gradient
    assert binding._targets_share([base[:, :5]], [base[:, 1:6]])


def test_lists_between_one_another():
    """Parts of one matrix that have no element in common, many of them: neither refused nor slow."""
    w = torch.zeros(64, 4096)
    cube = torch.zeros(12, 34, 56)
    for grads in (list(w.split(7, dim=1)), list(w.unbind(1)), list(w.t().unbind(0)), [w[:, 1::2], w[:, ::2].t()],
                  [w[::2, :100], w[1::2], w[::2, 100:]], [w[:, :100], w[:, 100:].view(64, 999, 4)[..., ::2],
                                                         w[:, 101:].reshape(-1)[:0], w[:, 100:].view(64, 999, 4)[..., 1::2]],
                  [cube.permute(2, 0, 1)[1:50, 2:9, 3:], cube[:2], cube[9:, ::3], cube[9:, 1::3].transpose(0, 2)],
                  [w.view(64, 16, 256)[:, k].t() for k in range(16)]):
        assert not binding._targets_share(grads, grads), [g.shape for g in grads]
    assert not binding._targets_share([w[:, :5]], [w[:, 5:10]])


def test_a_search_that_is_too_long(monkeypatch):
    """It ends, and what is not shown to be apart counts as shared."""
    r = random.Random(1)
    steps = [2 * r.randrange(10 ** 6, 2 * 10 ** 6) for _ in range(24)]
    odd = [(k, [(s, 9) for s in steps], 1) for k in (0, 5 * 10 ** 6 + 1)]
    monkeypatch.setattr(overlap, "_STEPS", 4000)
    monkeypatch.setattr(overlap, "_MODULI", 0)
    assert overlap.shared(odd, [])
    few = [(k, [(s, 1) for s in steps[:3]], 1) for k in (0, 5 * 10 ** 6 + 1)]
    assert not overlap.shared(few, [])


def test_results_on_what_is_read():
    big, ids = torch.zeros(40, 20), torch.zeros(9, dtype=torch.int64)
    apart = binding._apart
    assert apart(big[:9, :8], big[:, 8:16], ids) and apart(big[:9], big[9:], ids) and apart(big[::2, :4], big[1::2, :4])
    assert apart(big[:9, :8], big[:0, :8], ids) and apart(big, big.clone(), ids)
    assert not apart(big[:9], big, ids) and not apart(big[:9, :8], big[8:, 7:15], ids)
    assert not apart(big[20:29, :8], big[:, :8], ids) and not apart(ids.view(torch.float32)[None], big, ids)
