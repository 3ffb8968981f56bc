"""The gradient operators against plain implementations in binary64.

Bounds, from the number formats (u = 2^-24 for binary32; u_out = 2^-24, 2^-8, 2^-11 for the
three element types, the largest relative error of one rounding; tiny_out = half the distance
of the type's subnormal numbers):
  lookup     the binary32 product rounded once more: no difference at all
  gradient   a sum of m terms in binary32, in any order, is within (m - 1) u of the sum of the
             terms' magnitudes (first order); the factor, the addition to what was held and the
             rounding to the type add one each:
             (m + 2) u (|scale| sum |g| + |held|) + u_out |result| + tiny_out
  norms      binary64 sums, rounded once to binary32: 2^-24 relative; 2^-23 covers the sums
  clipped    factor and product are binary32 (2^-24 each) and the result is rounded once
"""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
U_OUT = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.float32: 2.0 ** -150, torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25}
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
I32, I64 = torch.int32, torch.int64


@pytest.fixture(scope="module")
def gpu():
    if not torch.cuda.is_available():
        pytest.fail("no GPU visible: the gpu-marked tests need an MI355X")
    from paper_2110_04478_amd import binding
    from paper_2110_04478_amd.csrc.build import ensure_built
    ensure_built()
    binding.lib()
    return binding


def normal(shape, dtype, seed, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * scale).to(dtype)


def numbers(n, vocab, dtype, seed, hot=0.0):
    r = np.random.default_rng(seed)
    ids = np.minimum((np.exp(r.random(n) * math.log(vocab + 1)) - 1).astype(np.int64), vocab - 1)
    ids[r.random(n) < hot] = vocab // 2
    return torch.from_numpy(ids).to(dtype)


def same(got, want):
    """Equal bit for bit, NaN for NaN."""
    got, want = got.cpu(), want.cpu()
    assert got.dtype == want.dtype and got.shape == want.shape
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    ok = ~torch.isnan(want)
    assert torch.equal(got[ok], want[ok])


# -- lookup -------------------------------------------------------------------------------

def lookup_64(table, ids, scale, dtype):
    """In binary64 (the product of two binary32 numbers is exact there), rounded as the
    operator rounds: to binary32 and then to the type."""
    t, vocab = ids.long(), table.shape[0]
    ok = (t >= 0) & (t < vocab)
    rows = table.double()[torch.where(ok, t, 0)] if vocab else torch.zeros(*ids.shape, table.shape[1]).double()
    rows = rows * float(np.float32(scale))
    rows[~ok] = float("nan")
    return rows.float().to(dtype)


@pytest.mark.parametrize("n", [1, 2, 3, 7, 63, 64, 65, 257, 1000, 4097])
@pytest.mark.parametrize("width", [1, 7, 8, 9, 64, 777, 1000, 2048, 2049, 4100])
def test_lookup_sizes(gpu, n, width):
    if n * width > 1 << 21:
        pytest.skip("covered by the smaller products")
    vocab = 501
    table, ids = normal((vocab, width), BF16, n), numbers(n, vocab, I64, width)
    got = gpu.themis_embedding_lookup(table.cuda(), ids.cuda(), 1.7)
    same(got, lookup_64(table, ids, 1.7, BF16))


@pytest.mark.parametrize("index", [I32, I64])
@pytest.mark.parametrize("to", [F32, BF16, F16])
@pytest.mark.parametrize("kind", [F32, BF16, F16])
def test_lookup_types(gpu, kind, to, index):
    table, ids = normal((333, 129), kind, 3, 30.0), numbers(200, 333, index, 4)
    table[5, :4] = torch.tensor([float("inf"), -float("inf"), float("nan"), 0.0])
    ids[:3] = 5
    got = gpu.themis_embedding_lookup(table.cuda(), ids.cuda(), 11.3, out_dtype=to)
    same(got, lookup_64(table, ids, 11.3, to))


def test_lookup_beyond_the_types_range(gpu):
    """Products too large for the type are infinite, those too small subnormal or zero."""
    table = torch.tensor([[6e4, 1e-4, 3e-8, -65519.0, -65520.0, 1e-7, 65504.0, 5.9e-8]])
    ids = torch.zeros(4, dtype=I64)
    for scale in (1.0, 1e-3, 2.0, 0.0):
        same(gpu.themis_embedding_lookup(table.cuda(), ids.cuda(), scale, out_dtype=F16),
             lookup_64(table, ids, scale, F16))


@pytest.mark.parametrize("index", [I32, I64])
def test_lookup_numbers_outside_the_table(gpu, index):
    table = normal((10, 33), F32, 1)
    wrong = [-1, 10, 11, -2 ** 31, 2 ** 31 - 1] + ([2 ** 32, 2 ** 32 + 3, -2 ** 63, 2 ** 63 - 1] if index == I64 else [])
    ids = torch.tensor([0, 9] + wrong + [3], dtype=index)
    got = gpu.themis_embedding_lookup(table.cuda(), ids.cuda())
    same(got, lookup_64(table, ids, 1.0, F32))
    assert torch.isnan(got[2:2 + len(wrong)]).all()
    none = gpu.themis_embedding_lookup(table[:0].cuda(), ids.cuda())
    assert torch.isnan(none).all()


def test_lookup_strides(gpu):
    """Slices of token numbers (the inputs of next-token training), a table inside a wider one, targets
    inside a larger array in another order; rows that begin at odd addresses."""
    table, tokens = normal((300, 90), BF16, 5), numbers(7 * 33, 300, I64, 6).view(7, 33)
    t, k = table.cuda(), tokens.cuda()
    for ids, ids_g in ((tokens[:, :-1], k[:, :-1]), (tokens[:, 1:], k[:, 1:]), (tokens[::2, ::3], k[::2, ::3]),
                       (tokens.t(), k.t()), (tokens[2:3].expand(5, 33), k[2:3].expand(5, 33)),
                       (tokens[:, :, None].expand(7, 33, 2)[:, 1:], k[:, :, None].expand(7, 33, 2)[:, 1:])):
        same(gpu.themis_embedding_lookup(t[:, 1:78], ids_g, 0.3), lookup_64(table[:, 1:78], ids, 0.3, BF16))
    big = torch.full((33, 7, 101), 7.0, dtype=F32, device="cuda")
    out = big.transpose(0, 1)[:, :32, 3:93]
    got = gpu.themis_embedding_lookup(t, k[:, :-1], 2.0, out=out)
    assert got is out
    same(out, lookup_64(table, tokens[:, :-1], 2.0, F32))
    kept = big.transpose(0, 1).clone()
    kept[:, :32, 3:93] = 7.0
    assert bool((kept == 7.0).all())   # nothing beside the rows was written


def test_lookup_offsets_beyond_32_bits(gpu):
    """Rows more than 2^32 elements apart."""
    whole = torch.zeros(2 ** 32 + 2 ** 20, dtype=BF16, device="cuda")
    table = torch.as_strided(whole, (3, 40), (2 ** 31 + 3, 1))
    rows = normal((3, 40), BF16, 9)
    table.copy_(rows)
    ids = torch.tensor([2, 0, 1, 2], dtype=I32)
    same(gpu.themis_embedding_lookup(table, ids.cuda(), 3.0), lookup_64(rows, ids, 3.0, BF16))


def test_lookup_of_nothing(gpu):
    table = torch.zeros((5, 4), device="cuda")
    assert gpu.themis_embedding_lookup(table, torch.zeros((0,), dtype=I64, device="cuda")).shape == (0, 4)
    assert gpu.themis_embedding_lookup(table, torch.zeros((3, 0), dtype=I64, device="cuda")).shape == (3, 0, 4)
    assert gpu.themis_embedding_lookup(table[:, :0], torch.zeros((3,), dtype=I64, device="cuda")).shape == (3, 0)
    one = torch.tensor(4, device="cuda")
    assert gpu.themis_embedding_lookup(table, one).shape == (4,)


# -- the table's gradient -----------------------------------------------------------------

def check_grad(got, g, ids, vocab, scale, ignored=-1, held=None):
    g, ids = g.cpu().reshape(-1, g.shape[-1]), ids.cpu().reshape(-1).long()
    scale = float(np.float32(scale))
    has = ((ids >= 0) & (ids < vocab) & (ids != ignored)).nonzero().view(-1)
    rows = g[has].double()
    want = torch.zeros((vocab, g.shape[-1]), dtype=torch.float64).index_add_(0, ids[has], rows) * scale
    mass = torch.zeros_like(want).index_add_(0, ids[has], rows.abs()) * abs(scale)
    terms = torch.bincount(ids[has], minlength=vocab).double()[:, None]
    if held is not None:
        want, mass = want + held.cpu().double(), mass + held.cpu().double().abs()
        untouched = terms[:, 0] == 0
        same(got.cpu()[untouched], held.cpu()[untouched])
    else:
        assert not got.cpu()[terms[:, 0] == 0].float().abs().any()
    bound = (terms + 2) * U * mass + U_OUT[got.dtype] * want.abs() + TINY[got.dtype]
    off = (got.cpu().double() - want).abs()
    assert not torch.isnan(off).any()
    worst = (off / bound).max().item() if off.numel() else 0.0
    assert worst <= 1.0, worst


@pytest.mark.parametrize("add", [False, True])
@pytest.mark.parametrize("width", [1, 8, 63, 520, 1000, 2056])
@pytest.mark.parametrize("n", [1, 2, 31, 64, 65, 129, 1000, 5001])
def test_grad_sizes(gpu, n, width, add):
    if n * width > 1 << 22:
        pytest.skip("covered by the smaller products")
    vocab = 777
    g, ids = normal((n, width), BF16, n + width), numbers(n, vocab, I64, n, hot=0.2)
    held = normal((vocab, width), F32, 8) if add else None
    out = held.cuda() if add else None
    got = gpu.themis_embedding_grad(g.cuda(), ids.cuda(), vocab, 1.3, out=out, out_dtype=F32, accumulate=add)
    check_grad(got, g, ids, vocab, 1.3, held=held)


@pytest.mark.parametrize("vocab", [1, 2, 63, 64, 65, 255, 256, 257, 1023, 1025, 65535, 65537, 300001])
def test_grad_vocabularies(gpu, vocab):
    n, width = 3000, 24
    g, ids = normal((n, width), F32, 1), torch.randint(0, vocab, (n,), generator=torch.Generator().manual_seed(vocab))
    ids[0], ids[-1] = vocab - 1, 0
    check_grad(gpu.themis_embedding_grad(g.cuda(), ids.cuda(), vocab), g, ids, vocab, 1.0)


@pytest.mark.parametrize("add", [False, True])
@pytest.mark.parametrize("index", [I32, I64])
@pytest.mark.parametrize("to", [F32, BF16, F16])
@pytest.mark.parametrize("kind", [F32, BF16, F16])
def test_grad_types(gpu, kind, to, index, add):
    n, vocab, width = 900, 400, 130
    g, ids = normal((n, width), kind, 1), numbers(n, vocab, index, 2)
    held = normal((vocab, width), to, 3) if add else None
    got = gpu.themis_embedding_grad(g.cuda(), ids.cuda(), vocab, 0.7, ignored=int(ids[5]),
                                    out=held.cuda() if add else None, out_dtype=to, accumulate=add)
    check_grad(got, g, ids, vocab, 0.7, ignored=int(ids[5]), held=held)


@pytest.mark.parametrize("n", [1, 64, 255, 257, 4096, 20000, 70001])
@pytest.mark.parametrize("share", [0.3, 1.0])
def test_grad_of_one_frequent_token(gpu, n, share):
    """All or many tokens of one number: a row that is the sum of thousands."""
    vocab, width = 5000, 40
    g, ids = normal((n, width), BF16, n), numbers(n, vocab, I32, n, hot=share)
    got = gpu.themis_embedding_grad(g.cuda(), ids.cuda(), vocab, out_dtype=F32)
    check_grad(got, g, ids, vocab, 1.0)


@pytest.mark.parametrize("each", [2, 33, 64, 65, 100, 129, 1000])
def test_grad_of_runs(gpu, each):
    """Every number the same number of times: sums that end wherever work is divided."""
    n, width = 10000, 72
    vocab = -(-n // each)
    ids = (torch.arange(n) // each)[torch.randperm(n, generator=torch.Generator().manual_seed(each))]
    g = normal((n, width), F32, each)
    check_grad(gpu.themis_embedding_grad(g.cuda(), ids.cuda(), vocab), g, ids, vocab, 1.0)


def test_grad_large_sorted_and_reversed(gpu):
    n, vocab, width = 150000, 70000, 16
    g = normal((n, width), BF16, 2)
    for ids in (torch.arange(n) % vocab, (n - 1 - torch.arange(n)) // 3, torch.full((n,), vocab - 1)):
        check_grad(gpu.themis_embedding_grad(g.cuda(), ids.cuda(), vocab, out_dtype=F32), g, ids, vocab, 1.0)


def test_grad_ignored_and_outside(gpu):
    """Tokens without a gradient: their rows may hold anything."""
    n, vocab, width = 500, 60, 50
    g, ids = normal((n, width), F32, 1), numbers(n, vocab, I64, 2)
    ids[::7], ids[1::7], ids[2::7], ids[3::7] = -1, vocab, 2 ** 40, 17
    g[::7], g[1::7], g[2::7], g[3::7] = float("nan"), float("inf"), -float("inf"), float("nan")
    g[(ids == 17)] = float("nan")
    got = gpu.themis_embedding_grad(g.cuda(), ids.cuda(), vocab, 2.0, ignored=17)
    check_grad(got, g, ids, vocab, 2.0, ignored=17)
    held = normal((vocab, width), BF16, 3)
    got = gpu.themis_embedding_grad(g.cuda(), ids.cuda(), vocab, 2.0, ignored=17, out=held.cuda(), accumulate=True)
    check_grad(got, g, ids, vocab, 2.0, ignored=17, held=held)
    # all of them: zeros, or what was held
    ids[:] = 17
    got = gpu.themis_embedding_grad(g.cuda(), ids.cuda(), vocab, 2.0, ignored=17)
    assert not got.any()
    got = gpu.themis_embedding_grad(g.cuda(), ids.cuda(), vocab, 2.0, ignored=17, out=held.cuda(), accumulate=True)
    same(got, held)


def test_grad_special_values_stay_in_their_place(gpu):
    g, ids = normal((400, 70), F32, 1), torch.arange(400) % 90
    g[13, 5], g[50, 69], g[399, 0] = float("nan"), float("inf"), -float("inf")
    got = gpu.themis_embedding_grad(g.cuda(), ids.cuda(), 100).cpu()
    wrong = ~torch.isfinite(got)
    assert wrong.nonzero().tolist() == [[13, 5], [399 % 90, 0], [50, 69]] or \
        sorted(wrong.nonzero().tolist()) == sorted([[13, 5], [50, 69], [399 % 90, 0]])
    assert math.isnan(got[13, 5]) and got[50, 69] == float("inf") and got[39, 0] == -float("inf")


def test_grad_strides(gpu):
    """Gradients of sliced sequences, of a broadcast, in a wider array; a target inside a larger table."""
    tokens, wide = numbers(6 * 41, 200, I64, 1).view(6, 41), normal((6, 41, 100), BF16, 2)
    k, w = tokens.cuda(), wide.cuda()
    views = [(wide[:, :-1, 3:90], w[:, :-1, 3:90], tokens[:, 1:], k[:, 1:]),
             (wide[::2, ::2], w[::2, ::2], tokens[::2, ::2], k[::2, ::2]),
             (wide[:, :1].expand(6, 41, 100), w[:, :1].expand(6, 41, 100), tokens, k),
             (wide[:1, :1, :1].expand(6, 41, 30), w[:1, :1, :1].expand(6, 41, 30), tokens, k),
             (wide[..., ::2], w[..., ::2], tokens, k),
             (wide.transpose(0, 1), w.transpose(0, 1), tokens.t(), k.t())]
    for g, gg, ids, ii in views:
        check_grad(gpu.themis_embedding_grad(gg, ii, 200, 1.5, out_dtype=F32), g, ids, 200, 1.5)
    big = torch.full((400, 111), 5.0, device="cuda")
    out = big[::2, 4:104]
    assert gpu.themis_embedding_grad(w, k, 200, out=out) is out
    check_grad(out, wide, tokens, 200, 1.0)
    big[::2, 4:104] = 5.0
    assert bool((big == 5.0).all())


def test_grad_of_nothing(gpu):
    none = torch.zeros((0, 12), device="cuda")
    ids = torch.zeros((0,), dtype=I64, device="cuda")
    out = torch.full((9, 12), 3.0, device="cuda")
    assert bool((gpu.themis_embedding_grad(none, ids, 9, out=out, accumulate=True) == 3.0).all())
    assert not gpu.themis_embedding_grad(none, ids, 9, out=out).any()
    assert gpu.themis_embedding_grad(torch.zeros((4, 0), device="cuda"),
                                     torch.zeros((4,), dtype=I64, device="cuda"), 9).shape == (9, 0)
    assert gpu.themis_embedding_grad(torch.zeros((4, 3), device="cuda"),
                                     torch.zeros((4,), dtype=I64, device="cuda"), 0).shape == (0, 3)


def test_grad_offsets_beyond_32_bits(gpu):
    whole = torch.zeros(2 ** 32 + 2 ** 20, dtype=BF16, device="cuda")
    g = torch.as_strided(whole, (3, 40), (2 ** 31 + 3, 1))
    rows, ids = normal((3, 40), BF16, 9), torch.tensor([2, 0, 2])
    g.copy_(rows)
    check_grad(gpu.themis_embedding_grad(g, ids.cuda(), 3, 3.0), rows, ids, 3, 3.0)
    got = gpu.themis_embedding_grad(rows.cuda(), ids.cuda(), 3, 3.0, out=g)
    check_grad(got, rows, ids, 3, 3.0)


def test_grad_is_the_same_in_every_call(gpu):
    n, vocab, width = 30000, 1000, 200
    g, ids = normal((n, width), F32, 1).cuda(), numbers(n, vocab, I64, 2, hot=0.3).cuda()
    first = gpu.themis_embedding_grad(g, ids, vocab)
    for _ in range(5):
        assert torch.equal(gpu.themis_embedding_grad(g, ids, vocab), first)


def test_grad_against_differences(gpu):
    """The lookup is linear in the table, so a difference over any step is the gradient's product
    with it, up to the rounding of the binary32 products (u each) and of the gradient's sums."""
    n, vocab, width, scale = 300, 50, 48, 1.9
    table, ids = normal((vocab, width), F32, 1).cuda(), numbers(n, vocab, I64, 2).cuda()
    weight = normal((n, width), F32, 3).cuda()
    grad = gpu.themis_embedding_grad(weight, ids, vocab, scale).double()

    def value(t):
        return (gpu.themis_embedding_lookup(t, ids, scale).double() * weight.double()).sum().item()

    size = scale * (weight.double().abs().sum().item()) * 8.0   # of the sums below (|table| < 8)
    for seed in range(4):
        step = torch.zeros_like(table)
        step[seed * 7 % vocab] = 0.5   # (table + step differs from table by the step but for u * 8)
        moved = table + step
        want = (grad * (moved.double() - table.double())).sum().item()
        assert abs(value(moved) - value(table) - want) <= (n + 4) * U * size


@pytest.mark.parametrize("kinds", [(F32, F32), (BF16, BF16), (F16, F32), (F32, BF16)])
@pytest.mark.parametrize("width", [2, 3, 4, 5, 7, 9, 11, 15, 17, 259, 511, 513, 515, 1023, 2047, 2049, 2051, 4099])
def test_rows_that_end_inside_an_access(gpu, width, kinds):
    """Every element is written once, and nothing beside the row: the last access of a row is moved
    back over the one before."""
    kind, to = kinds
    for n in (40, 4500):
        vocab = 70
        table, ids = normal((vocab, width), kind, n), numbers(n, vocab, I64, width)
        wide = torch.full((n, width + 5), 7.0, dtype=to, device="cuda")
        gpu.themis_embedding_lookup(table.cuda(), ids.cuda(), 1.7, out=wide[:, 2:-3])
        same(wide[:, 2:-3], lookup_64(table, ids, 1.7, to))
        g, held = normal((n, width), kind, 1), normal((vocab, width), to, 2)
        for add in (False, True):
            whole = torch.full((vocab, width + 5), 7.0, dtype=to, device="cuda")
            whole[:, 3:-2] = held.cuda()
            gpu.themis_embedding_grad(g.cuda(), ids.cuda(), vocab, 1.3, out=whole[:, 3:-2], accumulate=add)
            check_grad(whole[:, 3:-2], g, ids, vocab, 1.3, held=held if add else None)
            whole[:, 3:-2] = 7.0
            assert bool((whole == 7.0).all())
        wide[:, 2:-3] = 7.0
        assert bool((wide == 7.0).all())


@pytest.mark.parametrize("pad", [0, 1, 4, 8])
@pytest.mark.parametrize("width", [40, 1001, 2400])
def test_large_tables_cleared_before_the_sums(gpu, width, pad):
    """Tables beyond 64 MiB: rows that follow each other, and rows that do not; at odd addresses."""
    vocab = (80 << 20) // (4 * width)
    whole = torch.full((vocab * (width + pad) + 3,), 7.0, device="cuda")
    out = torch.as_strided(whole, (vocab, width), (width + pad, 1), 1)
    n = 50
    g, ids = normal((n, width), F32, 1), torch.randint(0, vocab, (n,), generator=torch.Generator().manual_seed(5))
    gpu.themis_embedding_grad(g.cuda(), ids.cuda(), vocab, 2.0, out=out)
    check_grad(out, g, ids, vocab, 2.0)
    out.fill_(7.0)
    assert bool((whole == 7.0).all())


@pytest.mark.parametrize("n", [4095, 4096, 4097, 4160, 8192, 9001])
@pytest.mark.parametrize("width", [1, 9, 64, 65, 300, 777, 1032])
def test_grad_on_both_sides_of_the_sort(gpu, n, width):
    """Up to 4,096 tokens one launch, beyond a sort and tiles."""
    vocab = 3000
    g, ids = normal((n, width), BF16, n + width), numbers(n, vocab, I64, n, hot=0.1)
    ids[::9] = vocab - 1
    held = normal((vocab, width), F32, 8)
    got = gpu.themis_embedding_grad(g.cuda(), ids.cuda(), vocab, 1.3, ignored=vocab - 1, out_dtype=F32)
    check_grad(got, g, ids, vocab, 1.3, ignored=vocab - 1)
    got = gpu.themis_embedding_grad(g.cuda(), ids.cuda(), vocab, 1.3, out=held.cuda(), accumulate=True)
    check_grad(got, g, ids, vocab, 1.3, held=held)


@pytest.mark.parametrize("add", [False, True])
@pytest.mark.parametrize("to", [F32, BF16, F16])
@pytest.mark.parametrize("kind", [F32, BF16, F16])
@pytest.mark.parametrize("width", [33, 520])
def test_grad_types_of_many_tokens(gpu, width, kind, to, add):
    n, vocab = 6000, 2500
    g, ids = normal((n, width), kind, 1), numbers(n, vocab, I32, 2)
    held = normal((vocab, width), to, 3) if add else None
    got = gpu.themis_embedding_grad(g.cuda(), ids.cuda(), vocab, 0.7, ignored=int(ids[5]),
                                    out=held.cuda() if add else None, out_dtype=to, accumulate=add)
    check_grad(got, g, ids, vocab, 0.7, ignored=int(ids[5]), held=held)


def test_grad_strides_of_many_tokens(gpu):
    tokens, wide = numbers(90 * 81, 200, I64, 1).view(90, 81), normal((90, 81, 100), BF16, 2)
    k, w = tokens.cuda(), wide.cuda()
    for g, gg, ids, ii in ((wide[:, :-1, 3:90], w[:, :-1, 3:90], tokens[:, 1:], k[:, 1:]),
                           (wide[:, :1].expand(90, 81, 100), w[:, :1].expand(90, 81, 100), tokens, k),
                           (wide.transpose(0, 1), w.transpose(0, 1), tokens.t(), k.t())):
        check_grad(gpu.themis_embedding_grad(gg, ii, 200, 1.5, out_dtype=F32), g, ids, 200, 1.5)
    big = torch.full((400, 111), 5.0, device="cuda")
    out = big[::2, 4:104]
    assert gpu.themis_embedding_grad(w, k, 200, out=out) is out
    check_grad(out, wide, tokens, 200, 1.0)
    big[::2, 4:104] = 5.0
    assert bool((big == 5.0).all())


def test_grad_ignored_and_outside_among_many_tokens(gpu):
    n, vocab, width = 9000, 60, 50
    g, ids = normal((n, width), F32, 1), numbers(n, vocab, I64, 2)
    ids[::7], ids[1::7], ids[2::7], ids[3::7] = -1, vocab, 2 ** 40, 17
    g[(ids < 0) | (ids >= vocab) | (ids == 17)] = float("nan")
    got = gpu.themis_embedding_grad(g.cuda(), ids.cuda(), vocab, 2.0, ignored=17)
    check_grad(got, g, ids, vocab, 2.0, ignored=17)
    held = normal((vocab, width), BF16, 3)
    got = gpu.themis_embedding_grad(g.cuda(), ids.cuda(), vocab, 2.0, ignored=17, out=held.cuda(), accumulate=True)
    check_grad(got, g, ids, vocab, 2.0, ignored=17, held=held)
    ids[:] = 17
    assert not gpu.themis_embedding_grad(g.cuda(), ids.cuda(), vocab, 2.0, ignored=17).any()
    got = gpu.themis_embedding_grad(g.cuda(), ids.cuda(), vocab, 2.0, ignored=17, out=held.cuda(), accumulate=True)
    same(got, held)


def test_grad_workspace_of_many_tokens(gpu):
    n, vocab, width = 20000, 900, 65
    g, ids = normal((n, width), BF16, 3).cuda(), numbers(n, vocab, I64, 2, hot=0.2).cuda()
    want = gpu.themis_embedding_grad(g, ids, vocab, out_dtype=F32)
    need = gpu.themis_embedding_grad_workspace_bytes(n, width, vocab)
    assert need > 0
    for fill in (0, 0xFF, 0x7F):
        work = torch.full((need + 64,), fill, dtype=torch.uint8, device="cuda")
        same(gpu.themis_embedding_grad(g, ids, vocab, out_dtype=F32, workspace=work[:need]), want)
        assert bool((work[need:] == fill).all())
    for bad in (work[:need - 1], work[4:]):
        with pytest.raises(gpu.ThemisError) as e:
            gpu.themis_embedding_grad(g, ids, vocab, workspace=bad)
        assert e.value.status == -4


# -- norm and clipping --------------------------------------------------------------------

def squares_64(grads):
    return torch.stack([g.double().square().sum() for g in grads]).cpu() if len(grads) else torch.zeros(0).double()


def check_norms(total, norms, grads):
    want = squares_64(grads)
    got = torch.cat([norms, total[:1]]).double().cpu()
    want = torch.cat([want, want.sum()[None]]).sqrt()
    same(torch.isfinite(got), torch.isfinite(want))
    ok = torch.isfinite(want)
    assert bool(((got[ok] - want[ok]).abs() <= 2.0 ** -23 * want[ok]).all()), (got, want)
    return want[-1].item()


def check_clipped(outs, grads, total, norm, max_norm):
    factor = total[1].item()
    want_factor = 1.0 if norm <= max_norm else max_norm / norm
    assert abs(factor - want_factor) <= 2.0 ** -23 * want_factor
    for o, g in zip(outs, grads):
        want = g.double() * want_factor
        bound = (U_OUT[o.dtype] + 4 * U) * want.abs() + TINY[o.dtype]
        assert bool(((o.double() - want).abs() <= bound).all())


SIZES = [1, 2, 7, 8, 9, 255, 2047, 2048, 2049, 8191, 8192, 65535, 65536, 65537, 200003]


@pytest.mark.parametrize("kind", [F32, BF16, F16])
@pytest.mark.parametrize("n", SIZES)
def test_norm_and_clip_sizes(gpu, n, kind):
    g = normal((n,), kind, n).cuda()
    total, norms = gpu.themis_gradient_norm(gpu.themis_gradient_plan([g]))
    norm = check_norms(total, norms, [g])
    for to in (F32, BF16, F16):
        for max_norm in (norm / 3, norm * 3):
            out = torch.empty(n, dtype=to, device="cuda")
            total, norms = gpu.themis_gradient_clip(gpu.themis_gradient_plan([g], [out]), max_norm)
            check_norms(total, norms, [g])
            check_clipped([out], [g], total, norm, max_norm)


@pytest.mark.parametrize("count", [1, 3, 64, 700, 3001])
def test_clip_of_lists_into_a_packed_bucket(gpu, count):
    """Many tensors of any size and type, none at a round address in the bucket."""
    r = np.random.default_rng(count)
    kinds = [F32, BF16, F16]
    grads = [normal((int(np.exp(r.uniform(0, 9))),), kinds[r.integers(3)], i, float(np.exp(r.uniform(-6, 1)))).cuda()
             for i in range(count)]
    for to in kinds:
        whole = torch.full((sum(g.numel() for g in grads) + 2,), 9.0, dtype=to, device="cuda")
        outs = list(whole[1:-1].split([g.numel() for g in grads]))
        plan = gpu.themis_gradient_plan(grads, outs)
        total, norms = gpu.themis_gradient_clip(plan, 0.5)
        norm = check_norms(total, norms, grads)
        check_clipped(outs, grads, total, norm, 0.5)
        assert whole[0] == 9.0 and whole[-1] == 9.0


def test_clip_in_place(gpu):
    grads = [normal(s, k, i).cuda() for i, (s, k) in enumerate([((100, 33), F32), ((5,), BF16), ((70001,), F16)])]
    before = [g.clone() for g in grads]
    plan = gpu.themis_gradient_plan(grads)
    total, norms = gpu.themis_gradient_clip(plan, 1e9)
    norm = check_norms(total, norms, before)
    assert total[1] == 1.0
    for g, b in zip(grads, before):
        same(g, b)
    total, norms = gpu.themis_gradient_clip(plan, norm / 2)
    check_clipped(grads, before, total, norm, norm / 2)
    total, norms = gpu.themis_gradient_norm(plan)   # (the plan takes the values of the time)
    check_norms(total, norms, grads)


def test_clip_strides(gpu):
    """Views, transposed and permuted tensors, slices with steps, broadcasts, more than two levels."""
    base = normal((12, 34, 56), F32, 1).cuda()
    views = [base[:, 3:20], base[..., ::3], base.transpose(0, 2), base[::2, ::5, ::7], base[:, :, 4], base[3],
             base.permute(2, 0, 1)[1:50, 2:9, 3:], base[:, 1:2], base[4:4], base[0, 0, 0]]
    fan = base[0, 0, :1].expand(500)
    total, norms = gpu.themis_gradient_norm(gpu.themis_gradient_plan(views + [fan, base[:, :1].expand(12, 9, 56)]))
    check_norms(total, norms, views + [fan, base[:, :1].expand(12, 9, 56)])
    outs = [torch.empty(v.shape, dtype=BF16, device="cuda") for v in views]
    total, norms = gpu.themis_gradient_clip(gpu.themis_gradient_plan(views, outs), 2.0)
    check_clipped(outs, views, total, check_norms(total, norms, views), 2.0)
    # dense gradients into strided targets
    dense = [v.contiguous() for v in views]
    into = torch.full((12, 34, 56), 4.0, device="cuda")
    total, norms = gpu.themis_gradient_clip(gpu.themis_gradient_plan([dense[3]], [into[::2, ::5, ::7]]), 2.0)
    check_clipped([into[::2, ::5, ::7]], [dense[3]], total, check_norms(total, norms, [dense[3]]), 2.0)
    into[::2, ::5, ::7] = 4.0
    assert bool((into == 4.0).all())
    # in place on views that share no element
    whole = base.clone()
    parts = [whole[:, :10], whole[:, 10:, ::2], whole[:, 10:, 1::2].transpose(0, 1)]
    before = [p.clone() for p in parts]
    total, norms = gpu.themis_gradient_clip(gpu.themis_gradient_plan(parts), 1.0)
    check_clipped(parts, before, total, check_norms(total, norms, before), 1.0)


def test_gradients_that_share_elements(gpu):
    """A tensor given twice, windows over one another: norms as of any other, but no scaling in place."""
    g = normal((400,), F32, 3).cuda()
    for grads in ([g, g], [g, g[:0], g.view(20, 20), g], [g.unfold(0, 50, 7)], [g[:5], g.unfold(0, 3, 1)]):
        plan = gpu.themis_gradient_plan(grads)
        total, norms = gpu.themis_gradient_norm(plan)
        norm = check_norms(total, norms, grads)
        if any(a is b for k, a in enumerate(grads) for b in grads[k + 1:]) or any(a.dim() == 2 and a.stride(0) < a.shape[1] for a in grads):
            with pytest.raises(gpu.ThemisError) as e:
                gpu.themis_gradient_clip(plan, 1.0)
            assert e.value.status == -1
        outs = [torch.empty(x.shape, device="cuda") for x in grads]
        total, norms = gpu.themis_gradient_clip(gpu.themis_gradient_plan(grads, outs), 1.0)
        check_clipped(outs, grads, total, norm, 1.0)
    with pytest.raises(gpu.ThemisError):
        gpu.themis_gradient_plan([g, g], [g, g])


def test_many_tiny_gradients(gpu):
    grads = list(normal((9000 * 3,), BF16, 4).cuda().split(3))
    total, norms = gpu.themis_gradient_norm(gpu.themis_gradient_plan(grads))
    want = torch.cat(grads).double().view(-1, 3).square().sum(1).cpu()
    assert bool(((norms.double().cpu() - want.sqrt()).abs() <= 2.0 ** -23 * want.sqrt()).all())
    assert abs(total.item() - want.sum().sqrt().item()) <= 2.0 ** -23 * total.item()


def test_norm_needs_no_scaling(gpu):
    """Squares beyond binary32's range, in both directions, and sums of them."""
    for value in (1e-30, 1e-44, 1e25, 3e38):
        g = torch.full((3000,), value, device="cuda")
        total, norms = gpu.themis_gradient_norm(gpu.themis_gradient_plan([g[:1000], g[:1]]))
        want = math.sqrt(1001) * g[0].item()
        if want > 3.4028235e38:
            assert math.isinf(total.item())
        else:
            assert abs(total.item() - want) <= max(2.0 ** -23 * want, 2.0 ** -149)
        assert norms[1] == g[0]
    # a norm beyond binary32 still gives the factor
    g = torch.full((1000,), 3e38, device="cuda")
    out = torch.empty_like(g)
    total, _ = gpu.themis_gradient_clip(gpu.themis_gradient_plan([g], [out]), 1.0)
    assert abs(total[1].item() * math.sqrt(1000) * g[0].item() - 1.0) < 1e-5
    assert abs(out.double().norm().item() - 1.0) < 1e-5


@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("kind", [F32, BF16, F16])
def test_clip_of_special_values(gpu, kind, value):
    grads = [normal((5000,), kind, 1).cuda(), normal((77,), kind, 2).cuda()]
    grads[0][4321] = value
    outs = [torch.empty_like(g) for g in grads]
    total, norms = gpu.themis_gradient_clip(gpu.themis_gradient_plan(grads, outs), 1.0)
    if math.isnan(value):
        assert torch.isnan(total).all() and torch.isnan(norms[0]) and all(torch.isnan(o).all() for o in outs)
    else:
        assert math.isinf(total[0]) and total[1] == 0 and math.isinf(norms[0])
        assert torch.isnan(outs[0][4321]) and not outs[0][:4321].any() and not outs[1].any()
    assert torch.isfinite(norms[1])


def test_lists_of_nothing(gpu):
    empty = torch.zeros((0, 4), device="cuda")
    for grads in ([], [empty], [empty, empty, torch.zeros(0, dtype=BF16, device="cuda")]):
        plan = gpu.themis_gradient_plan(grads)
        total, norms = gpu.themis_gradient_norm(plan)
        assert total.tolist() == [0.0] and norms.tolist() == [0.0] * len(grads)
        total, norms = gpu.themis_gradient_clip(plan, 1.0)
        assert total.tolist() == [0.0, 1.0] and norms.tolist() == [0.0] * len(grads)
    g = normal((10,), F32, 1).cuda()
    total, norms = gpu.themis_gradient_norm(gpu.themis_gradient_plan([empty, g, empty, g[:0]]))
    check_norms(total, norms, [empty, g, empty, g[:0]])
    zeros = torch.zeros(1000, device="cuda")
    total, norms = gpu.themis_gradient_clip(gpu.themis_gradient_plan([zeros]), 1.0)
    assert total.tolist() == [0.0, 1.0] and not zeros.any()


def test_norm_of_billions_of_elements(gpu):
    """More than 2^32 bytes and 2^31 elements in one tensor, a value at each end."""
    n = 2 ** 31 + 12345
    g = torch.zeros(n, dtype=BF16, device="cuda")
    g[0], g[2 ** 31 + 7], g[n - 1] = 3.0, 4.0, 12.0
    total, norms = gpu.themis_gradient_norm(gpu.themis_gradient_plan([g]))
    assert total.item() == 13.0 and norms.item() == 13.0
    total, _ = gpu.themis_gradient_clip(gpu.themis_gradient_plan([g]), 6.5)
    assert total.tolist() == [13.0, 0.5]
    assert (g[0], g[2 ** 31 + 7], g[n - 1]) == (1.5, 2.0, 6.0)


# -- streams, graphs, workspaces, refusals ------------------------------------------------

def _all_calls(gpu, state):
    table, ids, g, grads, plan = state
    a = gpu.themis_embedding_lookup(table, ids, 2.0)
    b = gpu.themis_embedding_grad(g, ids, table.shape[0], 2.0, out_dtype=F32)
    return (a, b, *gpu.themis_gradient_clip(plan, 0.5), *gpu.themis_gradient_norm(plan), *plan.out)


def _state(gpu, n=3000):
    table, ids = normal((900, 65), BF16, 1).cuda(), numbers(n, 900, I64, 2, hot=0.2).cuda()
    g = normal((n, 65), BF16, 3).cuda()
    grads = [normal((s,), F32, s).cuda() for s in (10, 70000, 333)]
    return table, ids, g, grads, gpu.themis_gradient_plan(grads, [torch.empty_like(x) for x in grads])


def test_calls_on_another_stream(gpu):
    state = _state(gpu)
    want = [t.clone() for t in _all_calls(gpu, state)]
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(other):
        got = _all_calls(gpu, state)
    other.synchronize()
    for x, y in zip(got, want):
        same(x, y)


@pytest.mark.parametrize("n", [500, 20000])
def test_calls_replay_inside_a_hip_graph(gpu, n):
    state = _state(gpu, n)
    _all_calls(gpu, state)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = _all_calls(gpu, state)
    for seed in range(3):
        state[2].copy_(normal((n, 65), BF16, 10 + seed))
        state[3][1].copy_(normal((70000,), F32, 20 + seed))
        state[1].copy_(numbers(n, 900, I64, 30 + seed, hot=0.4))
        graph.replay()
        torch.cuda.synchronize()
        replayed = [t.clone() for t in got]
        for x, y in zip(replayed, _all_calls(gpu, state)):
            same(x, y)


def test_workspaces_are_the_callers_and_need_no_contents(gpu):
    state = _state(gpu)
    table, ids, g, _, plan = state
    want = [t.clone() for t in _all_calls(gpu, state)]
    need = gpu.themis_embedding_grad_workspace_bytes(ids.numel(), 65, 900)
    for fill in (0, 0xFF, 0x7F):
        work = torch.full((need + 64,), fill, dtype=torch.uint8, device="cuda")
        got = gpu.themis_embedding_grad(g, ids, 900, 2.0, out_dtype=F32, workspace=work[:need])
        same(got, want[1])
        assert bool((work[need:] == fill).all())
        plan.workspace.fill_(fill)
        total, norms = gpu.themis_gradient_clip(plan, 0.5)
        same(total, want[2])
        same(norms, want[3])
    if need:
        with pytest.raises(gpu.ThemisError) as e:
            gpu.themis_embedding_grad(g, ids, 900, workspace=work[:need - 1])
        assert e.value.status == -4
        with pytest.raises(gpu.ThemisError) as e:
            gpu.themis_embedding_grad(g, ids, 900, workspace=work[4:])
        assert e.value.status == -4


def test_refusals(gpu):
    t, ids = torch.zeros((5, 8), device="cuda"), torch.zeros(3, dtype=I64, device="cuda")
    g = torch.zeros((3, 8), device="cuda")
    calls = [
        lambda: gpu.themis_embedding_lookup(t.double(), ids),
        lambda: gpu.themis_embedding_lookup(t, ids.short()),
        lambda: gpu.themis_embedding_lookup(t, ids.float()),
        lambda: gpu.themis_embedding_lookup(t[0], ids),
        lambda: gpu.themis_embedding_lookup(t, ids.cpu()),
        lambda: gpu.themis_embedding_lookup(t, ids, out=torch.zeros((3, 7), device="cuda")),
        lambda: gpu.themis_embedding_lookup(t, ids, out=torch.zeros((3, 8), device="cuda"), out_dtype=BF16),
        lambda: gpu.themis_embedding_lookup(t, ids, out=torch.zeros((1, 8), device="cuda").expand(3, 8)),
        lambda: gpu.themis_embedding_lookup(t, ids, out=torch.zeros((3, 16), device="cuda")[:, ::2]),
        lambda: gpu.themis_embedding_lookup(t, ids, out=torch.as_strided(torch.zeros(30, device="cuda"), (3, 8), (7, 1))),
        lambda: gpu.themis_embedding_grad(g, ids[:2], 5),
        lambda: gpu.themis_embedding_grad(g, ids, -1),
        lambda: gpu.themis_embedding_grad(g, ids, 5, accumulate=True),
        lambda: gpu.themis_embedding_grad(g, ids, 5, out=torch.zeros((6, 8), device="cuda")),
        lambda: gpu.themis_embedding_grad(g, ids, 5, out=torch.zeros((1, 8), device="cuda").expand(5, 8)),
        lambda: gpu.themis_embedding_grad(g.long(), ids, 5),
        lambda: gpu.themis_gradient_plan([g.double()]),
        lambda: gpu.themis_gradient_plan([g.cpu()]),
        lambda: gpu.themis_gradient_plan([g], [g[:2]]),
        lambda: gpu.themis_gradient_plan([g], [g, g]),
        lambda: gpu.themis_gradient_plan([g], [torch.zeros((1, 8), device="cuda").expand(3, 8)]),
        lambda: gpu.themis_gradient_clip(gpu.themis_gradient_plan([g]), 0.0),
        lambda: gpu.themis_gradient_clip(gpu.themis_gradient_plan([g]), -1.0),
        lambda: gpu.themis_gradient_clip(gpu.themis_gradient_plan([g]), float("nan")),
        lambda: gpu.themis_gradient_clip(gpu.themis_gradient_plan([g]), float("inf")),
        lambda: gpu.themis_gradient_clip(gpu.themis_gradient_plan([g[:, :1].expand(3, 8)]), 1.0),
    ]
    for k, call in enumerate(calls):
        with pytest.raises(gpu.ThemisError) as e:
            call()
        assert e.value.status == -1, k


def test_gradients_that_overlap_in_part(gpu):
    """Windows over one another would be scaled twice in place, and a target on another gradient
    before that is read: the first have norms alone, the second are refused."""
    x, y = normal((400,), F32, 3).cuda(), normal((400,), F32, 4).cuda()
    before = x.clone()
    plan = gpu.themis_gradient_plan([x[:201], x[200:]])
    check_norms(*gpu.themis_gradient_norm(plan), [x[:201], x[200:]])
    with pytest.raises(gpu.ThemisError) as e:
        gpu.themis_gradient_clip(plan, 1e-3)
    assert e.value.status == -1
    same(x, before)
    for grads, outs in (([x, y], [y, x]), ([x[:200]], [x[1:201]]), ([x, y], [torch.empty_like(x), x])):
        with pytest.raises(gpu.ThemisError) as e:
            gpu.themis_gradient_plan(grads, outs)
        assert e.value.status == -1
    halves = [x[:200], x[200:]]
    total, norms = gpu.themis_gradient_clip(gpu.themis_gradient_plan(halves), 1.0)
    check_clipped(halves, [before[:200], before[200:]], total, check_norms(total, norms, [before[:200], before[200:]]), 1.0)


def test_plans_given_up_while_another_stream_uses_them(gpu):
    """The memory of a plan is not handed out again before a call on another stream has ended."""
    grads = [normal((70001,), F32, 5).cuda()]
    outs = [torch.empty_like(grads[0])]
    slow = torch.ones((8192, 8192), dtype=BF16, device="cuda")
    plan = gpu.themis_gradient_plan(grads, outs)
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(other):
        for _ in range(40):
            slow @ slow
        total, norms = gpu.themis_gradient_clip(plan, 1.0)
        done = torch.cuda.Event()
        done.record()
    sizes, held = (plan.image.numel() * 8, plan.workspace.numel()), {plan.image.data_ptr(), plan.workspace.data_ptr()}
    del plan
    taken = [torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda") for n in sizes for _ in range(8)]
    if not done.query():
        assert not held & {t.data_ptr() for t in taken}
    other.synchronize()
    check_clipped(outs, grads, total, check_norms(total, norms, grads), 1.0)
