"""The table's gradient and the lookup in the layouts that only long lists get: tiles of 16 and 32
tokens, many workgroups, keys of one to four digits, a table cleared before a sort, lookups of two
rows a lane.  Against sums in binary64; the bound is that of a sum of m binary32 terms in any order,
(m - 1) 2^-24 of their magnitudes, with one rounding each for the factor, what was held and the
result: (m + 2) 2^-24 (|scale| sum |g| + |held|) + u_out |result| + tiny_out."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
U_OUT = {F32: 2.0 ** -24, BF16: 2.0 ** -8, F16: 2.0 ** -11}
TINY = {F32: 2.0 ** -150, BF16: 2.0 ** -134, F16: 2.0 ** -25}


@pytest.fixture(scope="module")
def gpu():
    if not torch.cuda.is_available():
        pytest.fail("no GPU visible: the gpu-marked tests need an MI355X")
    from paper_2110_04478_amd import binding
    from paper_2110_04478_amd.csrc.build import ensure_built
    ensure_built()
    return binding


def normal(shape, dtype, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(shape, generator=g, device="cuda").to(dtype)


def numbers(n, vocab, seed, hot=0.0):
    """Rank r with probability ~ 1 / (r + 1), a share of one number."""
    r = np.random.default_rng(seed)
    ids = np.minimum((np.exp(r.random(n) * math.log(vocab + 1)) - 1).astype(np.int64), vocab - 1)
    ids[r.random(n) < hot] = vocab // 2
    return torch.from_numpy(ids).cuda()


def check(got, g, ids, scale, ignored=-1, held=None):
    vocab, scale = got.shape[0], float(np.float32(scale))
    has = ((ids >= 0) & (ids < vocab) & (ids != ignored)).nonzero().view(-1)
    rows, at, terms = ids[has].long().unique(return_inverse=True, return_counts=True)
    # (a row's terms in several sums, which are added: thousands of additions to one place take seconds)
    sums = max(1, min(256, (1 << 25) // max(1, rows.numel() * g.shape[1])))
    at = at * sums + torch.arange(at.numel(), device="cuda") % sums

    def summed(x):
        total = torch.zeros((rows.numel() * sums, g.shape[1]), dtype=torch.float64, device="cuda")
        return total.index_add_(0, at, x).view(rows.numel(), sums, g.shape[1]).sum(1)

    want, mass = summed(g[has].double()).mul_(scale), summed(g[has].double().abs()).mul_(abs(scale))
    rest = got.clone()
    if held is None:
        rest[rows] = 0
        assert not rest.any()
    else:
        want += held[rows]
        mass += held[rows].abs()
        rest[rows] = held[rows]
        assert torch.equal(rest, held)
    off = (got[rows].double() - want).abs()
    bound = (terms.double()[:, None] + 2) * U * mass + U_OUT[got.dtype] * want.abs() + TINY[got.dtype]
    assert bool((off <= bound).all()), (off / bound).max().item()


# (tokens, elements of a row): a tile is the longest of 32, 16, 8 tokens that leaves 4,096 wavefronts,
# of 64 lanes with eight elements each; a join has four wavefronts beyond 2,048 workgroups of sums
LAYOUTS = [
    (40001, 520),     # 16 tokens
    (70001, 520),     # 32
    (140001, 513),    # 32, 2,188 workgroups: joins of four wavefronts
    (60001, 2049),    # 32, 2,345, five slabs
    (600001, 40),     # 16, eight lanes a row
    (1100001, 61),    # 32
    (1100001, 7),     # 32, element by element
    (300001, 130),    # 32, 32 lanes a row
]


@pytest.mark.parametrize("n,width", LAYOUTS)
@pytest.mark.parametrize("which", ["usual", "half one", "runs", "each once", "one"])
def test_tiles(gpu, n, width, which):
    """Sums that end in a tile, go from one turn of its loop to the next, and cross tiles, workgroups
    and blocks."""
    vocab = {"usual": 5003, "half one": 5003, "runs": -(-n // 37), "each once": n, "one": 3}[which]
    if vocab * width > 1 << 27:
        pytest.skip("a large table, covered by the other widths")
    if which in ("usual", "half one"):
        ids = numbers(n, vocab, n, 0.5 if which == "half one" else 0.0)
        ids[::11] = -1
    elif which == "one":
        ids = torch.ones(n, dtype=torch.int64, device="cuda")
    else:
        order = torch.randperm(n, generator=torch.Generator().manual_seed(n))
        ids = ((torch.arange(n) // (37 if which == "runs" else 1))[order]).cuda()
    g = normal((n, width), BF16, width)
    check(gpu.themis_embedding_grad(g, ids, vocab, 1.3, ignored=17, out_dtype=F32), g, ids, 1.3, ignored=17)
    held = normal((vocab, width), BF16, 2)
    got = gpu.themis_embedding_grad(g, ids, vocab, 0.7, out=held.clone(), accumulate=True)
    check(got, g, ids, 0.7, held=held)


@pytest.mark.parametrize("kind,to", [(F32, F32), (F32, BF16), (F16, F32), (BF16, BF16), (F16, F16)])
@pytest.mark.parametrize("n,width", LAYOUTS[1:4])
def test_types_in_long_tiles(gpu, n, width, kind, to):
    vocab = 6007
    g, ids = normal((n, width), kind, 1), numbers(n, vocab, 2, 0.1).int()
    check(gpu.themis_embedding_grad(g, ids, vocab, 0.3, out_dtype=to), g, ids, 0.3)
    held = normal((vocab, width), to, 3)
    check(gpu.themis_embedding_grad(g, ids, vocab, 0.3, out=held.clone(), accumulate=True), g, ids, 0.3, held=held)


@pytest.mark.parametrize("n", [3000, 5000, 60000])
@pytest.mark.parametrize("vocab", [1, 2, 3, 63, 64, 255, 256, 1022, 1023, 1024, 1025, 65535, 65536, (1 << 20) - 2,
                                   (1 << 20) - 1, 1 << 20, 3000001])
@pytest.mark.parametrize("width", [3, 9])
def test_keys(gpu, n, vocab, width):
    """Digits of the sort: one pass up to 1,023 rows, two up to 2^20 - 1, then three; a token without a
    gradient has the key behind the last row's."""
    ids = torch.randint(0, vocab, (n,), generator=torch.Generator().manual_seed(vocab)).cuda()
    ids[::5], ids[1::7], ids[2::9], ids[3::11] = vocab - 1, vocab, -1, 0
    ids[4::13] = 1 << 40
    g = normal((n, width), F32, n)
    for ignored in (-1, vocab - 1, 0):
        check(gpu.themis_embedding_grad(g, ids, vocab, 2.0, ignored=ignored), g, ids, 2.0, ignored=ignored)
    held = normal((vocab, width), F32, 3)
    got = gpu.themis_embedding_grad(g, ids, vocab, 2.0, ignored=vocab // 2, out=held.clone(), accumulate=True)
    check(got, g, ids, 2.0, ignored=vocab // 2, held=held)


def test_keys_of_four_digits(gpu):
    vocab, n = (1 << 30) + 5, 5000
    ids = torch.randint(0, vocab, (n,), generator=torch.Generator().manual_seed(3)).cuda()
    ids[::3], ids[1::50], ids[2::50] = vocab - 1, 0, vocab
    g = normal((n, 1), BF16, 4)
    check(gpu.themis_embedding_grad(g, ids, vocab, 2.0), g, ids, 2.0)


@pytest.mark.parametrize("pad", [0, 5])
@pytest.mark.parametrize("n,width,vocab", [(5000, 512, 40001), (4097, 1001, 30001), (9000, 4096, 72001), (70001, 513, 140002)])
def test_clear_before_a_sort(gpu, n, width, vocab, pad):
    """Tables beyond 64 MiB with many more rows than tokens: zeros first, then sums of sorted tokens."""
    whole = torch.full((vocab, width + pad), 7.0, device="cuda")
    out = whole[:, pad:]
    g, ids = normal((n, width), BF16, 1), numbers(n, vocab, 2, 0.2)
    ids[:3] = torch.tensor([vocab - 1, 0, vocab], device="cuda")
    gpu.themis_embedding_grad(g, ids, vocab, 1.1, ignored=5, out=out)
    check(out, g, ids, 1.1, ignored=5)
    assert bool((whole[:, :pad] == 7.0).all())


@pytest.mark.parametrize("kind,to", [(F32, F32), (F32, BF16), (BF16, F32), (F16, F16)])
@pytest.mark.parametrize("n,width", [(4099, 2049), (9001, 801), (17001, 513), (70003, 130), (140001, 64), (300007, 9)])
def test_lookups_of_two_rows_a_lane(gpu, n, width, kind, to):
    """Several rows side by side, the last turn not full; a number outside the table among them."""
    vocab = 3001
    table, ids = normal((vocab, width), kind, 1), numbers(n, vocab, 2)
    ids[::101], ids[-1] = vocab, -1
    whole = torch.full((n, width + 3), 7.0, dtype=to, device="cuda")
    gpu.themis_embedding_lookup(table, ids, 1.7, out=whole[:, 2:-1])
    outside = (ids < 0) | (ids >= vocab)
    want = table[torch.where(outside, 0, ids)].double() * float(np.float32(1.7))   # exact; rounded as the operator does
    got = whole[:, 2:-1]
    assert torch.equal(got[~outside], want[~outside].float().to(to)) and bool(torch.isnan(got[outside]).all())
    whole[:, 2:-1] = 7.0
    assert bool((whole == 7.0).all())
