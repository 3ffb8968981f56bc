"""The expert layer's operators against plain implementations in binary64.

Bounds, from the number formats (u = 2^-24 for binary32; u_out = 2^-24, 2^-8, 2^-11, the largest
relative error of one rounding; tiny_out = half the distance of the type's subnormal numbers):
  order      whole numbers: no difference
  rows       into the order: no difference; a product of weight and gradient is rounded to binary32
             and from there to the type: no difference
  weights    a difference d = l - largest is rounded once, which changes exp(d) by |d| u; exp itself is
             within 2 u, the sum of N such terms within N + 2 more (a term's |d| u is largest, relative to
             a sum of at least 1, at |d| e^-|d| < 0.4), the quotient 1: (|d| + N + 8) u w + u_out w + tiny
  logits     a sum of k products w_i g_i of such weights, subtracted and multiplied by one:
             (D + N + k + 16) u (w_e |g_e| + p_e sum |w_i g_i|) + u_out |result| + tiny, D the largest |d|
  sums       m terms in binary32: (m + 2) u (sum |w y| + |held|) + u_out |result| + tiny
"""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
U_OUT = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.float32: 2.0 ** -149, torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25}
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
I32, I64 = torch.int32, torch.int64
INF = float("inf")


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


def same(got, want):
    """Equal bit for bit, NaN for NaN."""
    got, want = got.cpu(), want.cpu()
    assert got.dtype == want.dtype and got.shape == want.shape
    if got.is_floating_point():
        assert torch.equal(torch.isnan(got), torch.isnan(want))
        ok = ~torch.isnan(want)
        got, want = got[ok], want[ok]
    assert torch.equal(got, want)


def within(got, want, bound):
    got = got.cpu().double()
    assert got.shape == want.shape
    off = (got - want).abs()
    assert bool((off <= bound).all()), float((off - bound).max())


# -- gate ---------------------------------------------------------------------------------

def gate_64(logits, k, renormalize):
    """(weights, experts, |d| of the chosen) of rows without NaN or +inf."""
    rows = logits.double().numpy().reshape(-1, logits.shape[-1])
    n, e = rows.shape
    order = np.argsort(-rows, axis=1, kind="stable")[:, :k]
    value = np.take_along_axis(rows, order, 1)
    chosen = np.where(value == -INF, -1, order)
    top = np.where(value[:, :1] == -INF, 0.0, value[:, :1])
    over = np.exp((value if renormalize else rows) - top)
    weights = np.exp(value - top) / np.maximum(over.sum(1, keepdims=True), 1e-300)
    shape = (*logits.shape[:-1], k)
    d = np.where(chosen < 0, 0.0, top - np.where(chosen < 0, 0.0, value))
    return (torch.from_numpy(np.where(chosen < 0, 0.0, weights)).reshape(shape),
            torch.from_numpy(chosen).reshape(shape), torch.from_numpy(np.abs(d)).reshape(shape))


def check_gate(gpu, logits, k, renormalize, out=F32, index=I32, device_logits=None):
    weights, experts = gpu.themis_expert_gate(logits.cuda() if device_logits is None else device_logits, k,
                                              renormalize, out_dtype=out, index_dtype=index)
    want, chosen, d = gate_64(logits, k, renormalize)
    assert weights.dtype == out
    same(experts, chosen.to(index))
    terms = k if renormalize else logits.shape[-1]
    within(weights, want, ((d + terms + 8) * U + U_OUT[out]) * want + TINY[out])
    return weights, experts


@pytest.mark.parametrize("renormalize", [True, False])
@pytest.mark.parametrize("experts", [1, 2, 7, 8, 9, 16, 31, 60, 64, 65, 128, 200, 256, 300, 512, 513, 1000, 1024])
def test_gate_sizes(gpu, experts, renormalize):
    for n, k in ((1, 1), (3, 2), (33, 8), (130, 6), (70, 3), (67, 5), (40, 9), (1000, 64)):
        k = min(k, experts)
        check_gate(gpu, normal((n, experts), BF16, n + experts, 2.0), k, renormalize)
        check_gate(gpu, normal((n, experts), F32, n + experts, 2.0), k, renormalize)


@pytest.mark.parametrize("index", [I32, I64])
@pytest.mark.parametrize("out", [F32, BF16, F16])
@pytest.mark.parametrize("kind", [F32, BF16, F16])
def test_gate_types(gpu, kind, out, index):
    check_gate(gpu, normal((77, 40), kind, 5, 3.0), 5, True, out, index)
    check_gate(gpu, normal((77, 140), kind, 6, 3.0), 9, False, out, index)


@pytest.mark.parametrize("kind", [F32, BF16, F16])
def test_gate_equal_logits(gpu, kind):
    """Of equal ones the lower index; -0 and 0 are equal."""
    g = torch.Generator().manual_seed(3)
    few = torch.randint(-2, 3, (500, 96), generator=g).to(kind)
    few[few == 0] *= torch.where(torch.rand((few == 0).sum(), generator=g) < 0.5, -1.0, 1.0).to(kind)
    for k in (1, 2, 4, 7, 64):
        check_gate(gpu, few, k, True)
        check_gate(gpu, few * 1e-30 if kind == F32 else few, k, True)
    check_gate(gpu, torch.full((9, 1000), -0.5, dtype=kind), 8, False)
    check_gate(gpu, torch.zeros((9, 1024), dtype=kind), 8, False)
    check_gate(gpu, torch.full((9, 1000), 0.5, dtype=kind), 64, False)


@pytest.mark.parametrize("renormalize", [True, False])
@pytest.mark.parametrize("kind", [F32, BF16, F16])
def test_gate_masks(gpu, kind, renormalize):
    """Masked experts are not chosen; rows that leave fewer than k, or nothing; the type's lowest value
    is no mask."""
    for experts in (6, 64, 130, 600):
        x = normal((200, experts), kind, experts)
        g = torch.Generator().manual_seed(experts)
        x[torch.rand(x.shape, generator=g) < torch.linspace(0, 1, 200)[:, None]] = -INF
        x[7] = -INF
        x[8, 1:] = -INF
        x[9] = torch.finfo(kind).min
        x[10, :] = -INF
        x[10, 3] = torch.finfo(kind).min
        x[11, 0] = torch.finfo(kind).max
        weights, chosen = check_gate(gpu, x, min(6, experts), renormalize)
        assert (chosen[7] == -1).all() and (weights[7] == 0).all()
        assert chosen[10].tolist()[:2] == [3, -1] and weights[10, 0] == 1


@pytest.mark.parametrize("kind", [F32, BF16, F16])
def test_gate_nan_and_infinity(gpu, kind):
    x = normal((4, 20), kind, 1)
    x[0, 7] = float("nan")
    x[1, 5] = INF
    x[2, 3], x[2, 11] = -float("nan"), float("nan")
    for renormalize in (True, False):
        many, numbers = gpu.themis_expert_gate(x.cuda(), 12, renormalize)
        weights, experts = gpu.themis_expert_gate(x.cuda(), 3, renormalize)
        assert torch.equal(experts, numbers[:, :3]) and torch.isnan(many[:3]).all()
        assert torch.isnan(weights[:3]).all() and not torch.isnan(weights[3]).any()
        assert experts[0, 0] == 7 and experts[1, 0] == 5 and experts[2, :2].tolist() == [3, 11]
        grad = gpu.themis_expert_gate_grad(torch.ones_like(weights), x.cuda(), experts, renormalize)
        assert not torch.isnan(grad[3]).any() and torch.isnan(grad[0, 7])


def test_gate_strides(gpu):
    """Rows of a wider matrix, of a transposed batch, one row for all, odd addresses."""
    wide = normal((50, 91), BF16, 1)
    d = wide.cuda()
    check_gate(gpu, wide[:, 3:70], 4, True, device_logits=d[:, 3:70])
    check_gate(gpu, wide[::2, 1:60], 4, False, device_logits=d[::2, 1:60])
    check_gate(gpu, wide[:1].expand(9, 91), 4, True, device_logits=d[:1].expand(9, 91))
    cube = normal((6, 5, 33), F32, 2)
    check_gate(gpu, cube.transpose(0, 1), 3, True, device_logits=cube.cuda().transpose(0, 1))
    check_gate(gpu, cube.transpose(1, 2), 3, True, device_logits=cube.cuda().transpose(1, 2))


def gate_grad_64(g, logits, chosen, renormalize):
    """(gradient, magnitude) from the softmax's derivative, element by element."""
    e = logits.shape[-1]
    rows, g, chosen = logits.double().reshape(-1, e), g.double().reshape(-1, g.shape[-1]), chosen.long()
    chosen = chosen.reshape(-1, chosen.shape[-1])
    ok = (chosen >= 0) & (chosen < e)
    value = torch.where(ok, rows.gather(1, torch.where(ok, chosen, 0)), -INF)
    over = value if renormalize else rows
    top = over.amax(1, keepdim=True) if over.shape[1] else torch.full((len(rows), 1), -INF)
    top = torch.where(top == -INF, 0.0, top)
    total = torch.exp(over - top).sum(1, keepdim=True)
    total = torch.where(total == 0, 1.0, total)
    w = torch.where(ok, torch.exp(value - top) / total, 0.0)
    dot, size = (w * g).sum(1, keepdim=True), (w * g).abs().sum(1, keepdim=True)
    hot = (chosen[:, :, None] == torch.arange(e)).double()
    if renormalize:
        p = (hot * w[:, :, None]).sum(1)
    else:
        p = torch.exp(rows - top) / total
    want = (hot * (w * g)[:, :, None]).sum(1) - p * dot
    magnitude = (hot * (w * g).abs()[:, :, None]).sum(1) + p * size
    near = torch.where(torch.isinf(over), 0.0, (over - top).abs()).amax(1, keepdim=True) if over.shape[1] else top
    return want.reshape(logits.shape), magnitude.reshape(logits.shape), near.clamp(max=110).reshape(*logits.shape[:-1], 1)


def check_gate_grad(gpu, g, logits, chosen, renormalize, out=None, device_logits=None):
    got = gpu.themis_expert_gate_grad(g.cuda(), logits.cuda() if device_logits is None else device_logits,
                                      chosen.cuda(), renormalize, out)
    out = out or logits.dtype
    assert got.dtype == out
    want, magnitude, near = gate_grad_64(g, logits, chosen, renormalize)
    terms = chosen.shape[-1] if renormalize else logits.shape[-1]
    within(got, want, (near + terms + chosen.shape[-1] + 16) * U * magnitude + U_OUT[out] * want.abs() + TINY[out])


@pytest.mark.parametrize("renormalize", [True, False])
@pytest.mark.parametrize("experts", [1, 2, 7, 8, 9, 16, 31, 60, 64, 65, 128, 200, 256, 300, 512, 513, 1000, 1024])
def test_gate_gradient_sizes(gpu, experts, renormalize):
    for n, k in ((1, 1), (3, 2), (33, 8), (130, 6), (100, 64)):
        k = min(k, experts)
        x = normal((n, experts), F32, n + experts, 2.0)
        check_gate_grad(gpu, normal((n, k), F32, n), x, gate_64(x, k, True)[1], renormalize)


@pytest.mark.parametrize("out", [F32, BF16, F16])
@pytest.mark.parametrize("kind", [F32, BF16, F16])
def test_gate_gradient_types(gpu, kind, out):
    for grad, index in ((F32, I64), (BF16, I32), (F16, I64)):
        x = normal((77, 40), kind, 5, 3.0)
        check_gate_grad(gpu, normal((77, 5), grad, 2), x, gate_64(x, 5, True)[1].to(index), True, out)
        check_gate_grad(gpu, normal((77, 5), grad, 2), x, gate_64(x, 5, True)[1].to(index), False, out)


@pytest.mark.parametrize("experts", [65, 130, 300, 1001])
@pytest.mark.parametrize("out", [F32, BF16, F16])
@pytest.mark.parametrize("kind", [F32, BF16, F16])
def test_gate_gradient_types_of_several_chunks(gpu, kind, out, experts):
    """Two and four accesses a lane, the last one moved back; masked logits, in it too; a row with none left."""
    x = normal((50, experts), kind, experts, 3.0)
    g = torch.Generator().manual_seed(experts)
    x[torch.rand(x.shape, generator=g) < torch.linspace(0, 1, 50)[:, None]] = -INF
    x[3, -8:], x[4, -5:], x[5, :-3], x[6] = -INF, -INF, -INF, -INF
    for k in (3, 8, 20):
        chosen = gate_64(x, k, True)[1]
        assert bool((chosen[6] == -1).all())
        for renormalize in (True, False):
            check_gate_grad(gpu, normal((50, k), F32, 2), x, chosen.to(I32), renormalize, out)


@pytest.mark.parametrize("renormalize", [True, False])
def test_gate_gradient_lists(gpu, renormalize):
    """Experts that stand twice, none, numbers outside; more chosen than lanes; masked logits."""
    x = normal((64, 12), F32, 1, 2.0)
    x[5], x[6, 2:] = -INF, -INF
    r = np.random.default_rng(0)
    chosen = torch.from_numpy(r.integers(-3, 14, (64, 7)))
    chosen[0] = 4
    chosen[1] = -1
    chosen[2, 0], chosen[2, 1] = 2 ** 40, -2 ** 40
    check_gate_grad(gpu, normal((64, 7), F32, 3), x, chosen, renormalize)
    x = normal((20, 11), F32, 4)
    check_gate_grad(gpu, normal((20, 30), F32, 5), x, torch.from_numpy(r.integers(0, 11, (20, 30))), renormalize)
    none = gpu.themis_expert_gate_grad(torch.ones(20, 0).cuda(), x.cuda(), torch.zeros((20, 0), dtype=I64).cuda(), renormalize)
    same(none, torch.zeros(20, 11))


def test_gate_gradient_strides(gpu):
    wide = normal((50, 91), BF16, 1)
    x, chosen = wide[::2, 3:70], gate_64(wide[::2, 3:70], 4, True)[1]
    check_gate_grad(gpu, normal((25, 4), F32, 1), x, chosen, False, device_logits=wide.cuda()[::2, 3:70])
    every = normal((25, 8), F32, 1)
    got = gpu.themis_expert_gate_grad(every.cuda()[:, ::2], x.cuda(), chosen.cuda())
    same(got, gpu.themis_expert_gate_grad(every[:, ::2].contiguous().cuda(), x.cuda(), chosen.cuda()))
    same(gpu.themis_expert_gate_grad(torch.ones(1, 1).cuda().expand(25, 4), x.cuda(), chosen.cuda()),
         gpu.themis_expert_gate_grad(torch.ones(25, 4).cuda(), x.cuda(), chosen.cuda()))


def test_gate_gradient_against_differences(gpu):
    """Central differences of the definition in binary64: h^2 times a third derivative (below 1 for a
    softmax times |g| < 4, four products) and 2^-53 / h."""
    x, g = normal((6, 9), F32, 8), normal((6, 3), F32, 9).clamp(-4, 4)
    chosen = gate_64(x, 3, True)[1]
    for renormalize in (True, False):
        def value(z):
            v = z.gather(1, chosen)
            w = torch.softmax(v, 1) if renormalize else torch.softmax(z, 1).gather(1, chosen)
            return (w * g.double()).sum(1)
        h, diff = 1e-5, torch.zeros(6, 9, dtype=torch.float64)
        for e in range(9):
            step = torch.zeros(6, 9, dtype=torch.float64)
            step[:, e] = h
            diff[:, e] = (value(x.double() + step) - value(x.double() - step)) / (2 * h)
        got = gpu.themis_expert_gate_grad(g.cuda(), x.cuda(), chosen.cuda(), renormalize).cpu().double()
        assert float((got - diff).abs().max()) < 100 * 24 * U + 12 * h * h + 16 * 2.0 ** -53 / h


# -- order --------------------------------------------------------------------------------

def order_of(experts, n_experts, capacity):
    flat = experts.numpy().reshape(-1).astype(np.int64)
    slots = n_experts * capacity if capacity else flat.size
    counts = np.bincount(flat[(flat >= 0) & (flat < n_experts)], minlength=n_experts)
    starts = np.concatenate([[0], np.cumsum(counts)]) if not capacity else np.arange(n_experts + 1) * capacity
    place, source = np.full(flat.size, -1), np.full(slots, -1)
    order = np.argsort(np.where((flat < 0) | (flat >= n_experts), n_experts, flat), kind="stable")[:counts.sum()]
    first = np.concatenate([[0], np.cumsum(counts)])
    rank = np.arange(len(order)) - first[flat[order]]
    kept = rank < (capacity or flat.size + 1)
    at = starts[flat[order]] + rank
    place[order[kept]], source[at[kept]] = at[kept], order[kept]
    return place.reshape(experts.shape), counts, starts, source


def check_order(gpu, experts, n_experts, capacity=0, device_experts=None):
    got = gpu.themis_expert_sort(experts.cuda() if device_experts is None else device_experts, n_experts, capacity)
    for name, want in zip(("place", "counts", "starts", "source"), order_of(experts, n_experts, capacity)):
        same(getattr(got, name), torch.from_numpy(want).to(I32))
    return got


def choices(shape, n_experts, seed, dtype=I32, outside=0.0, hot=0.0):
    r = np.random.default_rng(seed)
    x = r.integers(0, n_experts, shape)
    x[r.random(shape) < hot] = n_experts // 2
    away = r.random(shape) < outside
    x[away] = r.choice([-1, -7, n_experts, n_experts + 5, 2 ** 31 - 1], int(away.sum()))
    return torch.from_numpy(x).to(dtype)


@pytest.mark.parametrize("capacity", [0, 1, 37])
@pytest.mark.parametrize("n_experts", [1, 2, 8, 61, 64, 1000, 1024])
@pytest.mark.parametrize("n,k", [(1, 1), (1, 8), (7, 3), (64, 1), (1000, 2), (5000, 8), (40960, 1), (40961, 1), (70001, 3)])
def test_order_sizes(gpu, n, k, n_experts, capacity):
    check_order(gpu, choices((n, k), n_experts, n + k, outside=0.1), n_experts, capacity)


@pytest.mark.parametrize("index", [I32, I64])
@pytest.mark.parametrize("n_experts", [1, 8, 61, 1024])
@pytest.mark.parametrize("pairs", [1023, 1024, 1025, 4095, 4096, 4097, 6000, 8191, 8192, 8193, 12289])
def test_order_around_one_workgroup(gpu, pairs, n_experts, index):
    """Turns of a wavefront, one and several, in one workgroup, and the first lists that two launches sort."""
    for capacity in (0, 37, 3000):
        for outside, hot in ((0.0, 0.0), (0.2, 0.0), (0.0, 0.7), (0.1, 1.0)):
            check_order(gpu, choices((pairs, 1), n_experts, pairs, index, outside, hot), n_experts, capacity)
    if pairs % 3 == 0:
        check_order(gpu, choices((pairs // 3, 3), n_experts, pairs, index, 0.1, 0.3), n_experts, 11)


@pytest.mark.parametrize("index", [I32, I64])
@pytest.mark.parametrize("hot", [0.0, 0.5, 1.0])
def test_order_of_hot_experts(gpu, index, hot):
    for n in (100, 30000, 200000):
        for capacity in (0, 1000):
            check_order(gpu, choices((n, 2), 64, n, index, 0.0, hot), 64, capacity)


def test_order_of_large_lists(gpu):
    check_order(gpu, choices((300000, 8), 256, 1, hot=0.3), 256)
    check_order(gpu, choices((1 << 20, 2), 128, 2, I64, outside=0.5), 128, 20000)


def test_order_without_pairs(gpu):
    check_order(gpu, torch.zeros((0, 4), dtype=I32), 5)
    check_order(gpu, torch.zeros((0, 4), dtype=I32), 5, 3)
    check_order(gpu, torch.zeros((6, 0), dtype=I64), 5, 3)
    check_order(gpu, torch.full((9, 2), -1, dtype=I64), 5)
    check_order(gpu, torch.full((9, 2), -1, dtype=I64), 5, 2)
    wide = torch.tensor([2 ** 32, 2 ** 32 + 1, -2 ** 63, 2 ** 63 - 1, 1])[:, None]
    check_order(gpu, wide, 4)


def test_order_strides(gpu):
    x = choices((40, 30, 6), 16, 3)
    d = x.cuda()
    check_order(gpu, x[:, 1:, :4], 16, device_experts=d[:, 1:, :4])
    check_order(gpu, x[::2, :, 2:], 16, 20, device_experts=d[::2, :, 2:])
    check_order(gpu, x.transpose(0, 1), 16, device_experts=d.transpose(0, 1))
    check_order(gpu, x[..., ::2], 16, device_experts=d[..., ::2])
    check_order(gpu, x[:1, :1].expand(5, 4, 6), 16, device_experts=d[:1, :1].expand(5, 4, 6))


# -- rows ---------------------------------------------------------------------------------

def an_order(gpu, shape, n_experts, capacity, seed, outside=0.05):
    experts = choices(shape, n_experts, seed, outside=outside)
    return gpu.themis_expert_sort(experts.cuda(), n_experts, capacity), order_of(experts, n_experts, capacity)


def dispatch_of(x, place, source, dtype):
    rows = x.reshape(-1, x.shape[-1])
    ok, k = source >= 0, place.shape[-1]
    out = rows[torch.from_numpy(np.where(ok, source, 0) // max(k, 1))].float()
    out[torch.from_numpy(~ok)] = 0
    return out.to(dtype)


def combine_64(y, place, weights, held):
    """(sum, magnitude), the terms added in binary64."""
    k = place.shape[-1]
    flat = torch.from_numpy(place.reshape(-1, k))
    rows = y.double()[flat.clamp(min=0)] if y.shape[0] else torch.zeros(*flat.shape, y.shape[-1]).double()
    if weights is not None:
        rows = rows * weights.double().reshape(-1, k, 1)
    rows = torch.where(flat[:, :, None] >= 0, rows, 0.0)
    out, size = rows.sum(1), rows.abs().sum(1)
    if held is not None:
        out, size = out + held.double().reshape(out.shape), size + held.double().abs().reshape(out.shape)
    return out, size


WIDTHS = [1, 7, 8, 9, 64, 65, 100, 777, 1000, 2048, 2049, 4100]


@pytest.mark.parametrize("capacity", [0, 3, 90])
@pytest.mark.parametrize("width", WIDTHS)
def test_dispatch_and_combine_sizes(gpu, width, capacity):
    for n, k, n_experts in ((1, 1, 1), (1, 8, 9), (5, 3, 4), (130, 2, 8), (257, 5, 13)):
        order, (place, _, _, source) = an_order(gpu, (n, k), n_experts, capacity, n + width)
        x = normal((n, width), BF16, n)
        same(gpu.themis_expert_dispatch(x.cuda(), order), dispatch_of(x, place, source, BF16))
        y, w, held = normal((len(source), width), BF16, 2), normal((n, k), F32, 3), normal((n, width), BF16, 4)
        y[torch.from_numpy(source < 0)] = float("nan")   # not read
        for weights, add in ((w, None), (None, None), (w, held)):
            out = None if add is None else add.cuda()
            got = gpu.themis_expert_combine(y.cuda(), order, None if weights is None else weights.cuda(), out=out,
                                            accumulate=add is not None)
            assert out is None or got is out
            want, size = combine_64(y, place, weights, add)
            within(got, want, (k + 3) * U * size + U_OUT[BF16] * want.abs() + TINY[BF16])


@pytest.mark.parametrize("to", [F32, BF16, F16])
@pytest.mark.parametrize("kind", [F32, BF16, F16])
def test_dispatch_and_combine_types(gpu, kind, to):
    order, (place, _, _, source) = an_order(gpu, (60, 3), 7, 20, 1)
    for width in (5, 129, 520):
        x = normal((60, width), kind, 2, 30.0)
        x[3, :4] = torch.tensor([INF, -INF, float("nan"), 0.0])
        same(gpu.themis_expert_dispatch(x.cuda(), order, out_dtype=to), dispatch_of(x, place, source, to))
        y = normal((len(source), width), kind, 2, 3.0)
        for kw in (F32, BF16, F16):
            w, held = normal((60, 3), kw, 3), normal((60, width), to, 4)
            got = gpu.themis_expert_combine(y.cuda(), order, w.cuda(), out=held.cuda(), accumulate=True)
            want, size = combine_64(y, place, w, held)
            within(got, want, 6 * U * size + U_OUT[to] * want.abs() + TINY[to])


@pytest.mark.parametrize("capacity", [0, 3, 90])
@pytest.mark.parametrize("width", WIDTHS)
def test_combine_gradient_sizes(gpu, width, capacity):
    for n, k, n_experts in ((1, 1, 1), (1, 8, 9), (5, 3, 4), (130, 2, 8), (257, 5, 13)):
        order, orders = an_order(gpu, (n, k), n_experts, capacity, n + width)
        y, w, g = normal((len(orders[3]), width), BF16, 2), normal((n, k), F32, 3), normal((n, width), BF16, 4)
        check_combine_gradient(gpu, g, y, order, orders, w)


def check_combine_gradient(gpu, g, y, order, orders, w, at=None):
    """at: tensors on the GPU in the place of copies."""
    at = at or {}
    place, _, _, source = orders
    rows, products = gpu.themis_expert_combine_grad(at.get("g", g.cuda()), at.get("y", y.cuda()), order,
                                                    at.get("w", w.cuda()))
    k, width = place.shape[-1], g.shape[-1]
    flat, slot = g.reshape(-1, width), torch.from_numpy(source).clamp(min=0)
    want = (flat.float()[slot // k] * w.reshape(-1)[slot].float()[:, None])
    want[torch.from_numpy(source < 0)] = 0
    same(rows, want.to(y.dtype))
    at = torch.from_numpy(place.reshape(-1, k))
    terms = flat.double()[:, None] * (y.double()[at.clamp(min=0)] if y.shape[0] else torch.zeros(*at.shape, width))
    terms = torch.where(at[:, :, None] >= 0, terms, 0.0)
    dot, size = terms.sum(-1).reshape(w.shape), terms.abs().sum(-1).reshape(w.shape)
    within(products, dot, (width + 2) * U * size + U_OUT[w.dtype] * dot.abs() + TINY[w.dtype])
    alone = gpu.themis_expert_combine_grad(g.cuda(), y.cuda(), order, w.cuda(), need_weights=False)
    same(alone[0], rows)
    other = gpu.themis_expert_combine_grad(g.cuda(), y.cuda(), order, w.cuda(), need_rows=False)
    same(other[1], products)
    assert alone[1] is None and other[0] is None


@pytest.mark.parametrize("kg", [F32, BF16, F16])
@pytest.mark.parametrize("ky", [F32, BF16, F16])
def test_combine_gradient_types(gpu, kg, ky):
    for width in (5, 129, 520):
        for kw in (F32, BF16, F16):
            order, orders = an_order(gpu, (60, 3), 7, 20, 1)
            check_combine_gradient(gpu, normal((60, width), kg, 1), normal((140, width), ky, 2), order, orders,
                                   normal((60, 3), kw, 3))


def test_infinite_neighbours_stay_out_of_products(gpu):
    """Rows whose last access begins before the last elements of the one before."""
    order, (place, _, _, _) = an_order(gpu, (4, 2), 3, 0, 1, outside=0.0)
    for width in (9, 13, 516, 2049):
        y, g = normal((8, width), BF16, 1), torch.zeros(4, width, dtype=BF16)
        y[:, width - 5] = INF
        g[:, width - 5] = 1
        _, products = gpu.themis_expert_combine_grad(g.cuda(), y.cuda(), order, torch.ones(4, 2).cuda())
        want = (g.double()[:, None] * y.double()[torch.from_numpy(place)]).sum(-1)
        assert torch.equal(torch.isnan(products.cpu()), torch.isnan(want))


def test_rows_without_pairs(gpu):
    """No experts a token, no tokens, no slots that anybody has, no columns."""
    order = gpu.themis_expert_sort(torch.zeros((6, 0), dtype=I32).cuda(), 3, 2)
    x = normal((6, 20), BF16, 1).cuda()
    assert not gpu.themis_expert_dispatch(x, order).any()
    assert not gpu.themis_expert_combine(normal((6, 20), BF16, 2).cuda(), order).any()
    held = x.clone()
    assert torch.equal(gpu.themis_expert_combine(normal((6, 20), BF16, 2).cuda(), order, out=held, accumulate=True), x)
    rows, products = gpu.themis_expert_combine_grad(x, normal((6, 20), BF16, 3).cuda(), order, torch.zeros(6, 0).cuda())
    assert not rows.any() and products.shape == (6, 0)
    order = gpu.themis_expert_sort(torch.zeros((0, 2), dtype=I32).cuda(), 3, 2)
    assert not gpu.themis_expert_dispatch(x[:0], order).any()
    assert gpu.themis_expert_combine(x, order).shape == (0, 20)
    order = gpu.themis_expert_sort(torch.full((6, 2), -1, dtype=I32).cuda(), 3)
    assert not gpu.themis_expert_dispatch(x, order).any()
    nan = torch.full((12, 20), float("nan"), dtype=BF16).cuda()
    assert not gpu.themis_expert_combine(nan, order, torch.ones(6, 2).cuda()).any()
    rows, products = gpu.themis_expert_combine_grad(x, nan, order, torch.ones(6, 2).cuda())
    assert not rows.any() and not products.any()
    order = gpu.themis_expert_sort(torch.zeros((6, 2), dtype=I32).cuda(), 3)
    rows, products = gpu.themis_expert_combine_grad(x[:, :0], nan[:, :0], order, torch.ones(6, 2).cuda())
    assert rows.shape == (12, 0) and not products.any() and gpu.themis_expert_dispatch(x[:, :0], order).shape == (12, 0)


def test_one_token_without_a_batch(gpu):
    """Every shape may be a token's alone: [experts], [k], [width]."""
    logits = normal((40,), F32, 1)
    weights, chosen = check_gate(gpu, logits, 3, True)
    grad = gpu.themis_expert_gate_grad(weights, logits.cuda(), chosen)
    same(grad, gpu.themis_expert_gate_grad(weights[None], logits[None].cuda(), chosen[None])[0])
    order = check_order(gpu, chosen.cpu(), 40, 2)
    x = normal((30,), BF16, 2).cuda()
    rows = gpu.themis_expert_dispatch(x, order)
    assert all(torch.equal(rows[2 * int(e)], x) for e in chosen) and int(rows.any(1).sum()) == 3
    back = gpu.themis_expert_combine(rows, order, torch.tensor([0.5, 0.25, 0.25]).cuda())
    assert torch.equal(back, x)
    _, products = gpu.themis_expert_combine_grad(x, rows, order, weights)
    assert products.shape == (3,) and bool((products - x.float().square().sum()).abs().max() <= 32 * U * x.float().square().sum())


def test_weights_of_pairs_without_a_slot_have_no_part(gpu):
    order, (place, _, _, _) = an_order(gpu, (50, 3), 4, 10, 2)
    w, y, g = normal((50, 3), F32, 1), normal((40, 30), F32, 2), normal((50, 30), F32, 3)
    spoiled = torch.where(torch.from_numpy(place) < 0, float("nan"), w)
    assert torch.isnan(spoiled).any()
    same(gpu.themis_expert_combine(y.cuda(), order, spoiled.cuda()), gpu.themis_expert_combine(y.cuda(), order, w.cuda()))
    for a, b in zip(gpu.themis_expert_combine_grad(g.cuda(), y.cuda(), order, spoiled.cuda()),
                    gpu.themis_expert_combine_grad(g.cuda(), y.cuda(), order, w.cuda())):
        same(a, b)


def test_row_strides(gpu):
    """Tokens in two levels, slots that are every other row, rows at odd addresses, one row for all."""
    order, orders = an_order(gpu, (6, 10, 2), 5, 30, 3)
    place, _, _, source = orders
    big = normal((6, 11, 40), BF16, 1)
    x = big[:, 1:, 3:36]
    got = gpu.themis_expert_dispatch(big.cuda()[:, 1:, 3:36], order)
    same(got, dispatch_of(x.reshape(60, 33), place, source, BF16))
    room = torch.full((300, 41), 7.0, dtype=BF16).cuda()
    gpu.themis_expert_dispatch(x.cuda(), order, out=room[::2, 1:34])
    same(room[::2, 1:34], got)
    assert (room[1::2] == 7).all() and (room[:, 0] == 7).all() and (room[:, 34:] == 7).all()
    y, w = normal((300, 40), F16, 2), normal((6, 10, 5), F32, 3)
    held = torch.full((6, 12, 37), 3.0, dtype=F32).cuda()
    gpu.themis_expert_combine(y.cuda()[::2, 1:34], order, w.cuda()[..., 1:3], out=held[:, 2:, 2:35], accumulate=True)
    want, size = combine_64(y[::2, 1:34], place, w[..., 1:3], torch.full((60, 33), 3.0))
    within(held[:, 2:, 2:35].reshape(60, 33), want, 5 * U * size + U * want.abs())
    assert (held[:, :2] == 3).all() and (held[:, :, :2] == 3).all() and (held[:, :, 35:] == 3).all()
    g = normal((6, 10, 1), BF16, 5)
    check_combine_gradient(gpu, g.expand(6, 10, 33), y[::2, 1:34].to(BF16), order, orders, w[..., 1:3],
                           dict(y=y.to(BF16).cuda()[::2, 1:34], w=w.cuda()[..., 1:3]))
    one = normal((1, 33), BF16, 6)
    check_combine_gradient(gpu, one.expand(6, 10, 33), y[::2, 1:34].to(BF16), order, orders, w[..., 1:3],
                           dict(g=one.cuda().expand(6, 10, 33)))


def test_an_order_that_is_none_is_not_followed(gpu):
    """Places and sources beyond the slots are taken as none."""
    order, (place, _, _, source) = an_order(gpu, (20, 2), 4, 0, 1, outside=0.0)
    order.place[3, 0], order.place[4, 1], order.source[5] = 10 ** 6, 40, 40
    place[3, 0] = place[4, 1] = -1
    y, w = normal((40, 24), F32, 1), normal((20, 2), F32, 2)
    want, size = combine_64(y, place, w, None)
    within(gpu.themis_expert_combine(y.cuda(), order, w.cuda()), want, 4 * U * size + U * want.abs())
    _, products = gpu.themis_expert_combine_grad(normal((20, 24), F32, 1).cuda(), y.cuda(), order, w.cuda())
    assert products[3, 0] == 0 and products[4, 1] == 0


CHANGES = dict(place_none=lambda place, source: place.view(-1)[3:9:2].fill_(-1),
               place_outside=lambda place, source: place.view(-1)[3:9:2].fill_(10 ** 6),
               place_of_another=lambda place, source: place.view(-1)[3:6].copy_(place.view(-1)[6:9].clone()),
               source_none=lambda place, source: source[:5].fill_(-1),
               source_outside=lambda place, source: source[2:7].fill_(10 ** 6),
               source_of_another=lambda place, source: source[2:4].copy_(source[4:6].clone()),
               places_swapped=lambda place, source: place.copy_(place.flip(0).clone()),
               all_sources_none=lambda place, source: source.fill_(-1))


@pytest.mark.parametrize("width", [5, 24, 520, 2049])
@pytest.mark.parametrize("capacity", [0, 14])
@pytest.mark.parametrize("change", list(CHANGES))
def test_rows_by_slots_of_an_order_that_was_changed(gpu, change, capacity, width):
    """Slot s is pair a's where source[s] is a and place[a] is s, and holds zeros otherwise: every slot is
    written, and by one pair."""
    order, orders = an_order(gpu, (40, 3), 9, capacity, 1)
    CHANGES[change](order.place, order.source)
    place, source = order.place.cpu().view(-1).long(), order.source.cpu().long()
    slots, pairs = len(source), place.numel()
    inside = (source >= 0) & (source < pairs)
    own = inside & (place[torch.where(inside, source, 0)] == torch.arange(slots))
    assert int(own.sum()) < int((orders[3] >= 0).sum())
    agreed = torch.where(own, source, -1).numpy()
    for kind in (F32, BF16):
        x, w, y = normal((40, width), kind, 1), normal((40, 3), F32, 2), normal((slots, width), kind, 3)
        out = torch.full((slots, width), float("nan"), dtype=kind).cuda()
        same(gpu.themis_expert_dispatch(x.cuda(), order, out=out), dispatch_of(x, place.view(40, 3).numpy(), agreed, kind))
        want = (x.float()[torch.from_numpy(agreed).clamp(min=0) // 3] *
                w.reshape(-1)[torch.from_numpy(agreed).clamp(min=0)][:, None])
        want[~own] = 0
        dx, dy, dw = x.cuda(), y.cuda(), w.cuda()
        for need in (True, False):
            spoiled = torch.full_like(dy, float("nan"))
            del spoiled   # (the result's memory: what is not written shows)
            same(gpu.themis_expert_combine_grad(dx, dy, order, dw, need_weights=need)[0], want.to(kind))


@pytest.mark.parametrize("kind,width,k,capacity", [(BF16, 4096, 3, 0), (F32, 1030, 2, 9000), (F16, 500, 8, 0)])
def test_rows_beyond_the_last_cache_level(gpu, kind, width, k, capacity):
    """Read another way there: the same as in two calls on half of the columns, which are not; products
    of the halves add up (two sums of width / 2 terms in binary32, one addition)."""
    n = (1 << 28) // (width * k * kind.itemsize) + 5
    g = torch.Generator(device="cuda").manual_seed(2)
    chosen = torch.randint(0, 8, (n, k), generator=g, device="cuda", dtype=I32)
    order = gpu.themis_expert_sort(chosen, 8, n * k // 8 + 100 if capacity else 0)
    make = lambda *shape: torch.randn(shape, generator=g, device="cuda")   # noqa: E731
    y, w, grad = make(order.slots, width).to(kind), make(n, k), make(n, width).to(BF16)
    whole, (rows, products) = gpu.themis_expert_combine(y, order, w), gpu.themis_expert_combine_grad(grad, y, order, w)
    half, sums = width // 2, []
    for c in (slice(0, half), slice(half, width)):
        same(gpu.themis_expert_combine(y[:, c], order, w), whole[:, c])
        part, product = gpu.themis_expert_combine_grad(grad[:, c], y[:, c], order, w)
        same(part, rows[:, c])
        sums.append(product.double())
    at = order.place.long().clamp(min=0)
    size = torch.stack([(grad.double() * y[at[:, j]].double()).abs().sum(1) for j in range(k)], 1)
    assert bool(((products.double() - sum(sums)).abs() <= (width + 4) * U * size + 2.0 ** -149).all())


def test_places_beyond_32_bits(gpu):
    """4.5 G elements in the order and back."""
    n, k, width = 140000, 8, 4096
    g = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn((n, width), generator=g, device="cuda").to(BF16)
    order = gpu.themis_expert_sort(torch.randint(0, 16, (n, k), generator=g, device="cuda", dtype=I32), 16)
    rows = gpu.themis_expert_dispatch(x, order)
    assert rows.numel() > 1 << 32
    for s in range(0, order.slots, 1 << 17):
        assert torch.equal(rows[s:s + (1 << 17)], x[(order.source[s:s + (1 << 17)] // k).long()])
    # eight equal rows times weights of a power of two: exact
    w = torch.full((n, k), 0.125, device="cuda")
    assert torch.equal(gpu.themis_expert_combine(rows, order, w), x)
    back, products = gpu.themis_expert_combine_grad(x, rows, order, w)
    for s in range(0, order.slots, 1 << 17):
        assert torch.equal(back[s:s + (1 << 17)], rows[s:s + (1 << 17)] * 0.125)
    norms = x.double().square().sum(1, keepdim=True)
    assert bool(((products.double() - norms).abs() <= (width + 3) * U * norms).all())


def test_rows_in_several_segments_of_a_grid(gpu):
    """More lanes than 2^31: long rows, then many short ones, there and back."""
    n, width = 515, 1 << 25
    base = torch.randn(width + n, generator=torch.Generator(device="cuda").manual_seed(4), device="cuda").to(BF16)
    x = base.as_strided((n, width), (1, 1))   # (row t is base from t on)
    order = gpu.themis_expert_sort(torch.arange(n - 1, -1, -1, device="cuda", dtype=I32)[:, None], n)
    rows = gpu.themis_expert_dispatch(x, order)
    for t in range(n):
        assert torch.equal(rows[n - 1 - t], base[t:t + width]), t
    sums = gpu.themis_expert_combine(rows, order, torch.full((n, 1), 0.5, device="cuda"))
    half = base * 0.5
    for t in range(n):
        assert torch.equal(sums[t], half[t:t + width]), t
    del rows, sums
    n, width = (2 ** 31 - 257) // 2 + 3000, 9
    base = torch.randn(n + 8, generator=torch.Generator(device="cuda").manual_seed(5), device="cuda", dtype=F32).to(BF16)
    x = base.as_strided((n, width), (1, 1))
    order = gpu.themis_expert_sort(torch.zeros((1, 1), device="cuda", dtype=I32).expand(n, 1), 1)
    for got in (gpu.themis_expert_dispatch(x, order), gpu.themis_expert_combine(x, order)):
        for t in range(0, n, 1 << 26):
            assert torch.equal(got[t:t + (1 << 26)], x[t:t + (1 << 26)]), t
        del got


def test_equal_calls_give_equal_bits(gpu):
    order, _ = an_order(gpu, (3000, 4), 16, 600, 1)
    y, w, g = normal((9600, 1000), BF16, 1).cuda(), normal((3000, 4), F32, 2).cuda(), normal((3000, 1000), F32, 3).cuda()
    one = [gpu.themis_expert_combine(y, order, w, out_dtype=F32), *gpu.themis_expert_combine_grad(g, y, order, w)]
    for _ in range(3):
        for a, b in zip(one, [gpu.themis_expert_combine(y, order, w, out_dtype=F32),
                              *gpu.themis_expert_combine_grad(g, y, order, w)]):
            same(a, b)
