"""Dropout against its definition: the generator's published answers, then bit for bit (a product
rounded to binary32, a sum rounded to binary32, a rounding to the type)."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
LOW = np.uint64(0xFFFFFFFF)


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


def philox(counter, key):
    """Philox4x32-10 on four and two arrays of whole numbers below 2^32."""
    c, k = [np.asarray(x, dtype=np.uint64) for x in counter], [int(x) for x in key]
    for _ in range(10):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [b >> np.uint64(32) ^ c[1] ^ np.uint64(k[0]), b & LOW, a >> np.uint64(32) ^ c[3] ^ np.uint64(k[1]), a & LOW]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return c


def test_the_generators_published_answers():
    """The known answers that the generator's authors publish with it."""
    f, z = 0xFFFFFFFF, 0
    for counter, key, want in (
            ([z] * 4, [z] * 2, "6627e8d5 e169c58d bc57ac4c 9b00dbd8"),
            ([f] * 4, [f] * 2, "408f276d 41c83b0e a20bc7c6 6d5451fd"),
            ([0x243f6a88, 0x85a308d3, 0x13198a2e, 0x03707344], [0xa4093822, 0x299f31d0],
             "d16cfe09 94fdcceb 5001e420 24126ea1")):
        assert " ".join("%08x" % int(x) for x in philox(counter, key)) == want


def kept_of(rows, width, p, seed, call, first=0):
    """Of the rows from `first` on."""
    seed, call, low = seed % 2 ** 64, call % 2 ** 64, 0xFFFFFFFF
    blocks = -(-width // 4)
    c0, c1 = np.meshgrid(np.arange(blocks, dtype=np.uint64), np.arange(first, first + rows, dtype=np.uint64))
    words = philox((c0, c1, np.full_like(c0, call & low), np.full_like(c0, call >> 32)), (seed & low, seed >> 32))
    return np.stack(words, -1).reshape(rows, -1)[:, :width] >= round(p * 2.0 ** 32)


def dropout_of(x, p, seed, call, add, dtype):
    width = x.shape[-1]
    kept = torch.from_numpy(kept_of(x.numel() // width, width, p, seed, call)).reshape(x.shape)
    scale = np.float32(1.0 / (1.0 - p)) if p < 1 else np.float32(0)
    out = torch.where(kept, x.float() * float(scale), 0.0)
    return (out if add is None else out + add.float()).to(dtype)


def same(got, want):
    got, want = got.cpu(), want.cpu()
    assert got.dtype == want.dtype and got.shape == want.shape
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    ok = ~torch.isnan(want)
    assert torch.equal(got[ok], want[ok])


@pytest.mark.parametrize("kind", [F32, BF16])
@pytest.mark.parametrize("width", [1, 3, 7, 8, 9, 10, 11, 12, 15, 16, 64, 777, 1000, 1023, 1025, 2048, 2049, 2055, 4100])
def test_sizes(gpu, width, kind):
    for n in (1, 2, 65, 300):
        x, held = normal((n, width), kind, n), normal((n, width), kind, n + 1)
        same(gpu.themis_dropout(x.cuda(), 0.3, 11, 5), dropout_of(x, 0.3, 11, 5, None, kind))
        same(gpu.themis_dropout(x.cuda(), 0.1, 12, 6, add=held.cuda()), dropout_of(x, 0.1, 12, 6, held, kind))


@pytest.mark.parametrize("to", [F32, BF16, F16])
@pytest.mark.parametrize("kind", [F32, BF16, F16])
def test_types(gpu, kind, to):
    for width in (5, 130, 1025):
        x, held = normal((33, width), kind, 1, 9.0), normal((33, width), to, 2)
        same(gpu.themis_dropout(x.cuda(), 0.5, 1, 2, out_dtype=to), dropout_of(x, 0.5, 1, 2, None, to))
        same(gpu.themis_dropout(x.cuda(), 0.5, 1, 2, add=held.cuda()), dropout_of(x, 0.5, 1, 2, held, to))


@pytest.mark.parametrize("seed,call", [(0, 0), (2 ** 32 - 1, 2 ** 32), (2 ** 64 - 1, 2 ** 64 - 1), (-1, -5),
                                       (0x299f31d0a4093822, 0x0370734413198a2e)])
def test_seeds_and_calls(gpu, seed, call):
    x = normal((9, 100), F32, 1)
    same(gpu.themis_dropout(x.cuda(), 0.4, seed, call), dropout_of(x, 0.4, seed, call, None, F32))
    at = torch.tensor([(call + 2 ** 63) % 2 ** 64 - 2 ** 63]).cuda()
    same(gpu.themis_dropout(x.cuda(), 0.4, seed, at), dropout_of(x, 0.4, seed, call, None, F32))


@pytest.mark.parametrize("p", [0.0, 2.0 ** -32, 2.0 ** -34, 1e-3, 0.5, 0.999, 1 - 2.0 ** -33, 1.0])
def test_probabilities(gpu, p):
    x = normal((64, 1000), F32, 1)
    x[0, :3] = torch.tensor([float("inf"), float("nan"), -float("inf")])
    same(gpu.themis_dropout(x.cuda(), p, 3, 4), dropout_of(x, p, 3, 4, None, F32))
    held = normal((64, 1000), F32, 2)
    same(gpu.themis_dropout(x.cuda(), p, 3, 4, add=held.cuda()), dropout_of(x, p, 3, 4, held, F32))


def test_what_is_dropped_is_zero(gpu):
    """Whatever it was; and about as many as asked for (64,000 draws at 0.25: a deviation is 110)."""
    x = torch.full((64, 1000), float("nan")).cuda()
    got = gpu.themis_dropout(x, 0.25, 5, 6)
    dropped = int((got == 0).sum())
    assert dropped + int(torch.isnan(got).sum()) == 64000 and abs(dropped - 16000) < 6 * 110


def test_the_mask_goes_by_row_and_column(gpu):
    """Not by strides, types, row lengths or places in memory; rows of a batch are counted through."""
    big = normal((6, 11, 90), BF16, 1)
    x = big[:, 1:, 3:80]
    want = dropout_of(x, 0.3, 1, 2, None, BF16)
    same(gpu.themis_dropout(big.cuda()[:, 1:, 3:80], 0.3, 1, 2), want)
    same(gpu.themis_dropout(x.contiguous().cuda().view(60, 77), 0.3, 1, 2).view(6, 10, 77), want)
    turned = big.cuda().transpose(0, 2)
    same(gpu.themis_dropout(turned, 0.3, 1, 2), dropout_of(big.transpose(0, 2), 0.3, 1, 2, None, BF16))
    ones = torch.ones(5, 100).cuda()
    short, long = gpu.themis_dropout(ones[:, :40], 0.3, 1, 2), gpu.themis_dropout(ones, 0.3, 1, 2)
    assert torch.equal(short, long[:, :40])
    one = normal((1, 77), F32, 3)
    same(gpu.themis_dropout(one.cuda().expand(9, 77), 0.3, 1, 2), dropout_of(one.expand(9, 77), 0.3, 1, 2, None, F32))
    room = torch.full((20, 100), 7.0).cuda()
    gpu.themis_dropout(ones, 0.3, 1, 2, out=room[::4])
    assert torch.equal(room[::4], long) and (room[1::4] == 7).all()


@pytest.mark.parametrize("width", [9, 100, 1027, 2100])
def test_in_place(gpu, width):
    x, held = normal((70, width), BF16, 1), normal((70, width), BF16, 2)
    d = x.cuda()
    assert gpu.themis_dropout(d, 0.3, 1, 2, out=d) is d
    same(d, dropout_of(x, 0.3, 1, 2, None, BF16))
    d = held.cuda()
    gpu.themis_dropout(x.cuda(), 0.3, 1, 2, add=d, out=d)
    same(d, dropout_of(x, 0.3, 1, 2, held, BF16))
    d = x.cuda()
    gpu.themis_dropout(d, 0.3, 1, 2, add=d, out=d)
    same(d, dropout_of(x, 0.3, 1, 2, x, BF16))


@pytest.mark.parametrize("kind,width,n", [(BF16, 4096, 20000), (F16, 1001, 70001), (F32, 2055, 20001)])
def test_more_than_the_last_cache_level_holds(gpu, kind, width, n):
    """Another kernel there: the first rows as a small call gives them, the last ones by the definition."""
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn(n, width, generator=g, device="cuda").to(kind)
    held = torch.randn(n, width, generator=g, device="cuda").to(kind)
    assert x.numel() * x.element_size() * 2 >= 1 << 28
    kept = torch.from_numpy(kept_of(n, width, 0.3, 3, 4)[-200:])
    for add in (None, held):
        got = gpu.themis_dropout(x, 0.3, 3, 4, add=add)
        few = gpu.themis_dropout(x[:1000], 0.3, 3, 4, add=None if add is None else add[:1000])
        same(got[:1000], few)
        last = torch.where(kept, x[-200:].cpu().float() * float(np.float32(1 / (1 - 0.3))), 0.0)
        same(got[-200:], (last if add is None else last + add[-200:].cpu().float()).to(kind))
        out = x.clone() if add is None else add.clone()
        gpu.themis_dropout(out if add is None else x, 0.3, 3, 4, add=None if add is None else out, out=out)
        same(out, got)


def test_more_rows_than_a_grid_has_lanes(gpu):
    """1.07 G rows of nine elements, two lanes each: in two segments."""
    n, width = (2 ** 31 - 257) // 2 + 3000, 9
    x = torch.arange(1.0, 10.0).cuda().expand(n, width)
    got = gpu.themis_dropout(x, 0.4, 8, 9, out_dtype=BF16)
    scale = float(np.float32(1 / (1 - 0.4)))
    for first in (0, 10 ** 9, n - 3500, n - 100):
        kept = torch.from_numpy(kept_of(100, width, 0.4, 8, 9, first))
        want = torch.where(kept, torch.arange(1.0, 10.0) * scale, 0.0).to(BF16)
        same(got[first:first + 100], want)


def test_nothing(gpu):
    assert gpu.themis_dropout(torch.ones(0, 5).cuda(), 0.3, 1, 2).shape == (0, 5)
    assert gpu.themis_dropout(torch.ones(5, 0).cuda(), 0.3, 1, 2).shape == (5, 0)
    assert gpu.themis_dropout(torch.ones(7).cuda(), 0.0, 1, 2).tolist() == [1.0] * 7


def test_a_captured_call_draws_another_mask_in_every_replay(gpu):
    x = normal((50, 300), F32, 1).cuda()
    call, out = torch.zeros(1, dtype=torch.int64, device="cuda"), torch.empty_like(x)
    gpu.themis_dropout(x, 0.3, 7, call, out=out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        gpu.themis_dropout(x, 0.3, 7, call, out=out)
    for replay in range(4):
        call.fill_(replay * 10 ** 12)
        graph.replay()
        torch.cuda.synchronize()
        same(out, dropout_of(x.cpu(), 0.3, 7, replay * 10 ** 12, None, F32))
        same(gpu.themis_dropout(x, 0.3, 7, replay * 10 ** 12), out)
