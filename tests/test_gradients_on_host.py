"""The host side of the gradient operators, without a GPU: what is refused before anything is
launched, and the layout of a list of gradients (every element in one piece, its tensor's).  The
pointers are numbers that nobody dereferences."""
import ctypes

import numpy as np
import pytest

F32, BF16, F16, I32, I64 = range(5)
FAKE = 0x100000


@pytest.fixture(scope="module")
def binding():
    from paper_2110_04478_amd.csrc.build import ensure_built
    ensure_built()
    from paper_2110_04478_amd import binding
    return binding


def rows(binding, type_, inner=1 << 20, outer_stride=0, inner_stride=8, data=FAKE):
    return binding._Rows(data, type_, inner, outer_stride, inner_stride)


def test_lookup_refusals(binding):
    L = binding.lib()

    def call(table=None, vocab=10, width=8, ids=None, n=5, out=None, **_):
        table = table or rows(binding, F32)
        ids = ids or rows(binding, I64, inner_stride=1)
        out = out or rows(binding, BF16)
        return L.themis_embedding_lookup(table, vocab, width, ids, n, 1.0, out, None)

    assert call(n=0) == 0 and call(width=0) == 0
    assert call(table=rows(binding, I32)) == -1 and call(table=rows(binding, 7)) == -1
    assert call(ids=rows(binding, F32)) == -1 and call(out=rows(binding, I64)) == -1
    assert call(table=rows(binding, F32, data=0)) == -1 and call(out=rows(binding, F32, data=0)) == -1
    assert call(table=rows(binding, F32, data=FAKE + 2)) == -1 and call(ids=rows(binding, I64, data=FAKE + 4)) == -1
    assert call(out=rows(binding, BF16, data=FAKE + 1)) == -1
    assert call(ids=rows(binding, I64, inner=0)) == -1
    assert call(n=1 << 31) == -2 and call(vocab=1 << 31) == -2 and call(width=1 << 31) == -2
    # rows of the result that share elements
    for bad in (dict(inner_stride=7), dict(inner_stride=0), dict(inner_stride=-7), dict(inner=2, outer_stride=15),
                dict(inner=2, outer_stride=0), dict(inner=3, outer_stride=8, inner_stride=8)):
        assert call(out=rows(binding, F32, **bad)) == -1, bad
    assert L.themis_embedding_lookup(None, 10, 8, rows(binding, I64), 5, 1.0, rows(binding, F32), None) == -1
    assert L.themis_embedding_lookup(rows(binding, F32), 10, 8, None, 5, 1.0, rows(binding, F32), None) == -1
    assert L.themis_embedding_lookup(rows(binding, F32), 10, 8, rows(binding, I64), 5, 1.0, None, None) == -1


def test_grad_refusals(binding):
    L = binding.lib()

    def call(g=None, width=8, ids=None, n=5, add=0, grad=None, vocab=10, work=FAKE, work_bytes=1 << 40):
        g = g or rows(binding, F32)
        ids = ids or rows(binding, I64, inner_stride=1)
        grad = grad or rows(binding, BF16)
        return L.themis_embedding_grad(g, width, ids, n, 1.0, -1, add, grad, vocab, work, work_bytes, None)

    assert call(width=0) == 0 and call(vocab=0) == 0 and call(n=0, add=1) == 0
    assert call(g=rows(binding, I32)) == -1 and call(ids=rows(binding, BF16)) == -1
    assert call(grad=rows(binding, I64)) == -1 and call(grad=rows(binding, F32, data=0)) == -1
    assert call(g=rows(binding, F32, data=FAKE + 1)) == -1 and call(ids=rows(binding, I32, data=FAKE + 2)) == -1
    assert call(grad=rows(binding, F32, inner_stride=4)) == -1 and call(grad=rows(binding, F32, inner_stride=0)) == -1
    assert call(n=1 << 31) == -2 and call(vocab=1 << 31) == -2 and call(width=1 << 31) == -2
    need = L.themis_embedding_grad_workspace_bytes(5, 8, 10)
    if need:
        assert call(work=None) == -4 and call(work_bytes=need - 1) == -4 and call(work=FAKE + 8) == -4


PIECE = np.dtype([("in", "u8"), ("out", "u8"), ("count", "u4"), ("cols", "u4"), ("tensor", "u4"), ("kind", "u4"),
                  ("in_row", "i8"), ("in_col", "i8"), ("out_row", "i8"), ("out_col", "i8")])
BYTES = {F32: 4, BF16: 2, F16: 2}


def layout(binding, parts, n_tensors):
    L, plan = binding.lib(), binding._GradientPlan()
    array = (binding._Gradient * max(1, len(parts)))(*[binding._Gradient(*p) for p in parts])
    assert L.themis_gradient_plan(array, len(parts), n_tensors, plan, None, 0) == 0
    image = np.zeros((plan.image_bytes + 7) // 8, dtype=np.uint64)
    assert L.themis_gradient_plan(array, len(parts), n_tensors, plan, image.ctypes.data, plan.image_bytes - 1) == -4
    assert L.themis_gradient_plan(array, len(parts), n_tensors, plan, image.ctypes.data, image.nbytes) == 0
    raw = image.view(np.uint8)[:plan.image_bytes].tobytes()
    pieces = np.frombuffer(raw[:plan.n_pieces * PIECE.itemsize], dtype=PIECE)
    first = np.frombuffer(raw[plan.n_pieces * PIECE.itemsize:][:4 * (n_tensors + 1)], dtype=np.uint32)
    return plan, pieces, first


def addresses(base, type_, rows_, cols, rs, cs):
    return base + BYTES[type_] * (np.arange(rows_)[:, None] * rs + np.arange(cols)[None, :] * cs)


@pytest.mark.parametrize("scale", [1, 40])
def test_every_element_is_in_one_piece(binding, scale):
    r = np.random.default_rng(scale)
    parts, at = [], 1 << 32
    for tensor in range(60):
        for _ in range(int(r.integers(0, 4))):
            it, ot = int(r.integers(3)), int(r.integers(3))
            rows_, cols = int(np.exp(r.uniform(0, 5))), int(np.exp(r.uniform(0, 6))) * scale
            kind = int(r.integers(6))
            rs, cs = {0: (cols, 1), 1: (cols + 3, 1), 2: (1, rows_), 3: (2 * cols, 2), 4: (0, 1), 5: (-cols, 1)}[kind]
            ors, ocs = [(cols, 1), (cols + 5, 1), (1, rows_), (-cols, 1)][int(r.integers(4))]
            if r.random() < 0.05:
                rows_ = 0
            parts.append((at + 4 * rows_ * cols, at + (1 << 40), tensor, it, ot, rows_, cols, rs, cs, ors, ocs))
            at += 64 * max(1, rows_) * cols
    plan, pieces, first = layout(binding, parts, 60)
    assert plan.has_out == 1 and plan.n_pieces == len(pieces)
    assert first[0] == 0 and first[-1] == len(pieces) and (np.diff(first.astype(np.int64)) >= 0).all()
    for t in range(60):
        assert (pieces["tensor"][first[t]:first[t + 1]] == t).all()
    seen_in, seen_out = [], []
    for p in pieces:
        it, ot = int(p["kind"] & 0xFF), int(p["kind"] >> 8 & 0xFF)
        assert 0 < p["count"] <= 65536 and p["count"] % p["cols"] == 0
        n, c = int(p["count"]), int(p["cols"])
        a = addresses(int(p["in"]), it, n // c, c, int(p["in_row"]), int(p["in_col"])).ravel()
        b = addresses(int(p["out"]), ot, n // c, c, int(p["out_row"]), int(p["out_col"])).ravel()
        if p["kind"] >> 16 & 1:
            assert (a == int(p["in"]) + BYTES[it] * np.arange(n)).all()
        if p["kind"] >> 17 & 1:
            assert (b == int(p["out"]) + BYTES[ot] * np.arange(n)).all()
        seen_in.append(a)
        seen_out.append(b)
    want = [(addresses(q[0], q[3], q[5], q[6], q[7], q[8]).ravel(), addresses(q[1], q[4], q[5], q[6], q[9], q[10]).ravel())
            for q in parts if q[5]]
    got = np.stack([np.concatenate(seen_in), np.concatenate(seen_out)])
    want = np.stack([np.concatenate([w[0] for w in want]), np.concatenate([w[1] for w in want])])
    order = lambda x: x[:, np.lexsort(x)]   # noqa: E731
    assert np.array_equal(order(got), order(want))


def test_pieces_of_long_tensors(binding):
    """One run is cut into pieces of one size, whatever its two given levels."""
    for rows_, cols in ((1, 10_000_003), (1000, 10_000), (10_000_000, 1), (1, 2 ** 33 + 5)):
        plan, pieces, _ = layout(binding, [(FAKE, FAKE, 0, BF16, BF16, rows_, cols, cols, 1, cols, 1)], 1)
        size = int(pieces["count"][0])
        assert (pieces["count"][:-1] == size).all() and size % 2048 == 0 and pieces["count"].sum(dtype=np.uint64) == rows_ * cols
        assert (pieces["in"] == FAKE + 2 * size * np.arange(len(pieces), dtype=np.uint64)).all()
        assert (pieces["kind"] >> 16 == 7).all() and plan.strided == 0


def test_plan_refusals(binding):
    L, plan = binding.lib(), binding._GradientPlan()

    def call(*parts, n_tensors=4):
        array = (binding._Gradient * max(1, len(parts)))(*[binding._Gradient(*p) for p in parts])
        return L.themis_gradient_plan(array, len(parts), n_tensors, plan, None, 0)

    ok = dict(in_=FAKE, out=FAKE * 2, tensor=1, it=F32, ot=BF16, rows_=3, cols=5, rs=5, cs=1, ors=5, ocs=1)

    def part(**kw):
        return tuple({**ok, **kw}.values())

    assert call(part()) == 0 and plan.has_out == 1 and call() == 0 and call(n_tensors=0) == 0
    assert call(part(out=0)) == 0 and plan.has_out == 0
    assert call(part(), part(tensor=0)) == -1 and call(part(tensor=4)) == -1
    assert call(part(it=I32)) == -1 and call(part(ot=9)) == -1
    assert call(part(in_=0)) == -1 and call(part(in_=FAKE + 2)) == -1 and call(part(out=FAKE + 1)) == -1
    assert call(part(in_=0, rows_=0)) == 0 and call(part(in_=0, cols=0)) == 0
    assert call(part(out=FAKE)) == -1                                    # in place, another type
    assert call(part(out=FAKE, ot=F32, ocs=2, ors=10)) == -1             # .., other strides
    assert call(part(out=FAKE, ot=F32)) == 0
    for bad in (dict(ocs=0), dict(ors=0), dict(ors=4), dict(ors=-4), dict(ors=1, ocs=2), dict(ors=3, ocs=2)):
        assert call(part(**bad)) == -1, bad                              # an element written twice
    assert call(part(rows_=1 << 40, cols=1 << 40)) == -2
    assert call(part(), n_tensors=1 << 25) == -2
    assert L.themis_gradient_plan(None, 1, 1, plan, None, 0) == -1
    assert L.themis_gradient_plan(None, 0, 0, None, None, 0) == -1


def test_pass_refusals(binding):
    L, plan = binding.lib(), binding._GradientPlan()
    array = (binding._Gradient * 1)(binding._Gradient(FAKE, FAKE, 0, F32, F32, 1, 100, 100, 1, 100, 1))
    assert L.themis_gradient_plan(array, 1, 1, plan, None, 0) == 0
    need = plan.workspace_bytes
    assert need > 0
    for name, args in (("themis_gradient_norm", ()), ("themis_gradient_clip", (ctypes.c_double(1.0),))):
        call = getattr(L, name)
        assert call(plan, *args, FAKE, None, FAKE, need, None) == -1       # no image
        plan.image = FAKE + 8
        assert call(plan, *args, FAKE, None, FAKE, need, None) == -1
        plan.image = FAKE
        assert call(plan, *args, None, None, FAKE, need, None) == -1
        assert call(plan, *args, FAKE, None, None, need, None) == -4
        assert call(plan, *args, FAKE, None, FAKE, need - 1, None) == -4
        assert call(plan, *args, FAKE, None, FAKE + 8, need, None) == -4
        plan.image = None
    plan.image = FAKE
    for bad in (0.0, -1.0, float("nan"), float("inf")):
        assert L.themis_gradient_clip(plan, bad, FAKE, None, FAKE, need, None) == -1
    plan.has_out = 0
    assert L.themis_gradient_clip(plan, 1.0, FAKE, None, FAKE, need, None) == -1


def test_views_of_tensors(binding):
    """Any tensor as views of two levels, element for element with its target."""
    import torch
    base = torch.arange(3 * 4 * 5 * 6).view(3, 4, 5, 6)
    cases = [base, base.permute(3, 1, 0, 2), base[:, 1:3], base[..., ::2], base[::2, :, 1:4, ::3], base[0, 0, 0, 0],
             base[:, :, :, 0], base[1, 2], base[:, :1].expand(3, 7, 5, 6), base.transpose(1, 2)[:, 2:3]]
    for g in cases:
        for o in (torch.empty(g.shape), torch.empty(g.shape[::-1]).permute(tuple(range(g.dim()))[::-1]),
                  torch.empty([2 * n for n in g.shape])[tuple(slice(0, 2 * n, 2) for n in g.shape)]):
            got = []
            for x, y, rows_, cols, ra, ca, rb, cb in binding._views(g, o):
                r, c = np.arange(rows_)[:, None], np.arange(cols)[None, :]
                got.append(np.stack([(x + r * ra + c * ca).ravel(), (y + r * rb + c * cb).ravel()]))
            got = np.concatenate(got, axis=1)
            at = np.indices(tuple(g.shape)).reshape(g.dim(), -1) if g.dim() else np.zeros((0, 1), int)
            want = np.stack([(np.array(t.stride())[:, None] * at).sum(0) for t in (g, o)]) if g.dim() else np.zeros((2, 1), int)
            order = lambda v: v[:, np.lexsort(v)]   # noqa: E731
            assert np.array_equal(order(got), order(want))


def test_rows_of_tensors(binding):
    """Token numbers and rows with strides, in the two levels that the library reads."""
    import torch
    base = torch.arange(4 * 6 * 10).view(4, 6, 10)
    for t, lead in ((base, 2), (base, 3), (base[:, :-1], 2), (base[::2, ::3], 2), (base.transpose(0, 1), 2),
                    (base[:, 1:2], 2), (base[0, 0, 0], 0), (base[0, 0], 1), (base[0, 0], 0), (base[:, :, 3], 2),
                    (base[:1].expand(5, 6, 10), 2), (base[:, :1].expand(4, 9, 10), 2), (base[..., :7], 2)):
        r = binding._rows(t, lead, t.shape[-1] if lead < t.dim() else 1)
        n = int(np.prod(t.shape[:lead]))
        k = np.arange(n)
        at = k // r.inner * r.outer_stride + k % r.inner * r.inner_stride
        want = (np.indices(t.shape[:lead]).reshape(lead, -1) * np.array(t.stride()[:lead]).reshape(-1, 1)).sum(0) if lead else [0]
        assert np.array_equal(at, want), (t.shape, t.stride())
    assert binding._rows(base[..., ::2], 2, 5) is None
    assert binding._rows(base.permute(1, 0, 2)[::2, :, ::3], 3, 1) is None


def test_targets_that_share_memory(binding):
    """Windows over one another, and targets on what another gradient still has to be read from."""
    import torch
    x, y, z = torch.zeros(40), torch.zeros(40), torch.zeros(40, dtype=torch.bfloat16)
    share = binding._targets_share
    for grads, outs in (([x, y], [x, y]), ([x, y], [y.clone(), x.clone()]), ([x, x], [y[:20], y[20:]]), ([], []),
                        ([x[:20], x[20:]], [x[:20], x[20:]]), ([x[:20], x[20:]], [x[:20], y[20:]]),
                        ([x[::2], x[1::2]], [x[::2], x[1::2]]), ([x[5:5], x], [x[5:5], x]), ([x, y[:0]], [x, x[3:3]]),
                        ([x.view(5, 8), y], [x.view(8, 5).view(5, 8), y])):
        assert not share(grads, outs)
    for grads, outs in (([x, x], [x, x]), ([x[:21], x[20:]], [x[:21], x[20:]]), ([x, x[20:]], [x, x[20:]]),
                        ([x[:10], x, x[30:]], [x[:10], x, x[30:]]), ([x, y], [y, x]), ([x, y], [x.clone(), x]),
                        ([x[:20]], [x[1:21]]), ([z[:20], x], [x.view(torch.bfloat16)[:20], y]),
                        ([x[::2], y[:20]], [x[::2], x[::2]])):
        assert share(grads, outs)
