"""The expert layer and dropout under autograd, together as a model uses them: gate, order, rows
there, the experts' products, back, dropout into the residual; on streams, in graphs."""
import numpy as np
import pytest
import torch

from test_gpu_dropout import kept_of

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def layers():
    if not torch.cuda.is_available():
        pytest.fail("no GPU visible: the gpu-marked tests need an MI355X")
    from paper_2110_04478_amd import layers
    from paper_2110_04478_amd.csrc.build import ensure_built
    ensure_built()
    return layers


def normal(shape, seed, scale=1.0, dtype=F32):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * scale).to(dtype).cuda()


def the_layer(layers, x, router, up, down, k, capacity, p, seed, call, renormalize=True):
    """x + dropout(experts(x)), with the library's operators; the experts' products on their buffers."""
    n_experts, width = up.shape[0], x.shape[-1]
    weights, chosen = layers.gate(x @ router, k, renormalize)
    order = layers.sort(chosen, n_experts, capacity)
    h = layers.dispatch(x, order).view(n_experts, capacity, width)
    y = torch.bmm(torch.relu(torch.bmm(h, up)), down).view(order.slots, width)
    return layers.dropout(layers.combine(y, order, weights), p, seed, call, add=x), chosen, order


def the_layer_64(x, router, up, down, chosen, place, p, seed, call, renormalize):
    """The same from the definitions in binary64: every pair that has a slot by itself."""
    logits = x @ router
    k = chosen.shape[-1]
    has, e = (place >= 0), chosen.long()
    over = logits.gather(-1, e) if renormalize else logits
    weights = torch.exp(logits.gather(-1, e) - torch.logsumexp(over, -1, keepdim=True))
    out = torch.zeros_like(x)
    for j in range(k):
        y = torch.stack([torch.relu(row @ up[i]) @ down[i] for row, i in zip(x, e[:, j].tolist())])
        out = out + torch.where(has[:, j, None], weights[:, j, None] * y, 0.0)
    kept = torch.from_numpy(kept_of(x.shape[0], x.shape[1], p, seed, call))
    return x + torch.where(kept, out / (1 - p), 0.0)


@pytest.mark.parametrize("renormalize", [True, False])
@pytest.mark.parametrize("capacity", [9, 40])
def test_a_layer_and_its_gradients(layers, capacity, renormalize):
    """Against binary64.  Every value is a chain of sums of at most 40 terms (products with the
    weights, sums over experts, over tokens for the weights' gradients) of magnitude below 40:
    256 u per link, ten links, times the largest magnitude."""
    n, width, hidden, n_experts, k, p = 40, 24, 32, 6, 2, 0.2
    make = [normal((n, width), 1), normal((width, n_experts), 2, 0.3), normal((n_experts, width, hidden), 3, 0.2),
            normal((n_experts, hidden, width), 4, 0.2)]
    here = [t.clone().requires_grad_() for t in make]
    out, chosen, order = the_layer(layers, *here, k, capacity, p, 5, 6, renormalize)
    assert bool((order.place < 0).any()) == (capacity == 9)
    g = normal((n, width), 7)
    got = torch.autograd.grad(out, here, g)
    there = [t.cpu().double().requires_grad_() for t in make]
    want = the_layer_64(*there, chosen.cpu(), order.place.cpu(), p, 5, 6, renormalize)
    grads = torch.autograd.grad(want, there, g.cpu().double())
    for a, b in zip((out, *got), (want, *grads)):
        assert a.dtype == F32 and float((a.detach().cpu().double() - b.detach()).abs().max()) <= 2560 * U * float(b.detach().abs().max())


def test_gradients_of_each_against_those_of_the_formulas(layers):
    """Types of the gradients, and autograd's own wiring: sums, broadcasts, parts that need none."""
    x = normal((30, 16), 1, dtype=BF16).requires_grad_()
    logits = normal((30, 5), 2, dtype=F16).requires_grad_()
    weights, chosen = layers.gate(logits, 3)
    assert weights.dtype == F32 and not chosen.requires_grad
    order = layers.sort(chosen, 5)
    rows = layers.dispatch(x, order)
    out = layers.combine(rows, order, weights)
    (out.float().sum() * 2).backward()
    assert x.grad.dtype == BF16 and logits.grad.dtype == F16
    # every token comes back as itself times the sum of its weights, 1: three products of weights in
    # bf16, added in binary32 and rounded again; the logits' gradients cancel
    assert float((x.grad.float() - 2).abs().max()) <= 2 * (3 + 1) * 2.0 ** -8
    size = (2 * x.detach().float().sum(-1).abs()).max()
    assert float(logits.grad.float().abs().max()) <= float(size) * 2.0 ** -9
    alone = layers.combine(rows.detach(), order, weights.detach().requires_grad_())
    assert alone.requires_grad
    plain = layers.combine(layers.dispatch(x, order), order)
    x.grad = None
    plain.sum().backward()
    assert torch.equal(x.grad, torch.full_like(x, 3))


def test_a_second_derivative_is_an_error(layers):
    x = normal((8, 16), 1).requires_grad_()
    g, = torch.autograd.grad(layers.dropout(x, 0.5, 1, 2).square().sum(), x, create_graph=True)
    with pytest.raises(RuntimeError):
        torch.autograd.grad(g.sum(), x)


def test_what_changed_before_the_backward_is_an_error(layers):
    x = normal((8, 16), 1).requires_grad_()
    call = torch.zeros(1, dtype=torch.int64, device="cuda")
    out = layers.dropout(x, 0.5, 1, call)
    call += 1
    with pytest.raises(RuntimeError):
        out.sum().backward()
    order = layers.sort(torch.zeros((8, 1), dtype=torch.int32, device="cuda"), 2)
    out = layers.dispatch(x, order)
    order.place[0] = -1
    with pytest.raises(RuntimeError):
        out.sum().backward()


@pytest.mark.parametrize("capacity", [0, 6])
def test_counts_may_change_before_the_backward(layers, capacity):
    """Summed over ranks in place, say: the gradients do not read them."""
    x, w = normal((30, 16), 1).requires_grad_(), normal((30, 2), 2).requires_grad_()
    chosen = torch.arange(60, dtype=torch.int32, device="cuda").view(30, 2) % 5
    grads = []
    for change in (False, True):
        order = layers.sort(chosen, 5, capacity)
        out = layers.combine(layers.dispatch(x, order), order, w)
        if change:
            order.counts.mul_(8)
            order.starts.add_(3)
            assert order.counts.tolist() == [96] * 5 and order.place.max() < 60
        grads.append(torch.autograd.grad(out.square().sum(), (x, w)))
    assert all(torch.equal(a, b) for a, b in zip(*grads))


@pytest.mark.parametrize("kind", [F32, BF16])
@pytest.mark.parametrize("weighted", [False, True])
@pytest.mark.parametrize("width", [1, 24])
def test_rows_that_no_gradient_reads_are_not_kept(layers, width, weighted, kind):
    """Without gradients of weights y may change, and its memory is free, before the backward."""
    leaf, w = normal((60, width), 1, dtype=kind).requires_grad_(), normal((30, 2), 2) if weighted else None
    order = layers.sort(torch.arange(60, dtype=torch.int32, device="cuda").view(30, 2) % 5, 5)
    g = normal((30, width), 3)
    grads = []
    for change in (False, True):
        y = leaf * 1
        out = layers.combine(y, order, w, F32)
        if change:
            y.mul_(2)
        grads.append(torch.autograd.grad(out, leaf, g)[0])
    assert grads[0].dtype == kind and grads[0].shape == (60, width) and torch.equal(*grads)
    y = leaf * 1
    out = layers.combine(y, order, normal((30, 2), 2).requires_grad_())
    y.mul_(2)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        torch.autograd.grad(out, leaf, g.to(kind))


def test_dropout_of_zero_gradients_and_of_add_alone(layers):
    x, held = normal((9, 33), 1), normal((9, 33), 2).requires_grad_()
    layers.dropout(x, 0.5, 1, 2, add=held).sum().backward()
    assert torch.equal(held.grad, torch.ones_like(held))
    x.requires_grad_()
    layers.dropout(x, 1.0, 1, 2).sum().backward()
    assert torch.equal(x.grad, torch.zeros_like(x))


def test_refusals(layers):
    from paper_2110_04478_amd import binding
    x, e = normal((8, 16), 1), torch.zeros((8, 2), dtype=torch.int32, device="cuda")
    order = layers.sort(e, 3)
    y, w = normal((16, 16), 2), normal((8, 2), 3)
    bad = [lambda: binding.themis_expert_gate(x, 17), lambda: binding.themis_expert_gate(x.double(), 2),
           lambda: binding.themis_expert_gate(x, 2, out_dtype=torch.float64),
           lambda: binding.themis_expert_gate(x, 2, index_dtype=torch.int16),
           lambda: binding.themis_expert_gate_grad(w[:4], x, e), lambda: binding.themis_expert_gate_grad(w, x, e[:4]),
           lambda: binding.themis_expert_sort(e.float(), 3), lambda: binding.themis_expert_sort(e, 0),
           lambda: binding.themis_expert_sort(e, 1025), lambda: binding.themis_expert_sort(e, 3, -1),
           lambda: binding.themis_expert_sort(e, 1000, 1 << 30),
           lambda: binding.themis_expert_dispatch(x[:7], order), lambda: binding.themis_expert_dispatch(x.cpu(), order),
           lambda: binding.themis_expert_dispatch(x, order, out=y[:15]),
           lambda: binding.themis_expert_dispatch(x, order, out=y, out_dtype=BF16),
           lambda: binding.themis_expert_dispatch(y[:8], order, out=y),
           lambda: binding.themis_expert_dispatch(x, order, out=y[:1].expand(16, 16)),
           lambda: binding.themis_expert_dispatch(x, order, out=normal((16, 32), 1)[:, ::2]),
           lambda: binding.themis_expert_combine(y[:15], order), lambda: binding.themis_expert_combine(y, order, w[:, :1]),
           lambda: binding.themis_expert_combine(y, order, w.cpu()), lambda: binding.themis_expert_combine(y, order, w, out=y[:8]),
           lambda: binding.themis_expert_combine(y, order, w, accumulate=True),
           lambda: binding.themis_expert_combine_grad(x[:, :8], y, order, w),
           lambda: binding.themis_expert_combine_grad(x, y, order, w[:, :1]),
           lambda: binding.themis_dropout(x, -0.1, 1, 2), lambda: binding.themis_dropout(x, float("nan"), 1, 2),
           lambda: binding.themis_dropout(x, 0.1, 1, torch.zeros(1, device="cuda")),
           lambda: binding.themis_dropout(x, 0.1, 1, torch.zeros(2, dtype=torch.int64, device="cuda")),
           lambda: binding.themis_dropout(x, 0.1, 1, torch.zeros(1, dtype=torch.int64)),
           lambda: binding.themis_dropout(x, 0.1, 1, 2, add=x[:4]), lambda: binding.themis_dropout(x, 0.1, 1, 2, add=x, out_dtype=BF16),
           lambda: binding.themis_dropout(y[:8], 0.1, 1, 2, out=y[1:9]),
           lambda: binding.themis_dropout(x, 0.1, 1, 2, out=x.view(BF16)[:, :16])]
    for n, call in enumerate(bad):
        with pytest.raises(binding.ThemisError):
            call()
            pytest.fail("call %d was taken" % n)


def test_a_workspace_on_the_list_is_refused(layers):
    """The counts of the parts would be written over experts that are read again after them."""
    from paper_2110_04478_amd import binding
    n = 20000
    need = binding.themis_expert_sort_workspace_bytes(n, 1, 16)
    room = torch.zeros(need // 4 + n, dtype=torch.int32, device="cuda")
    chosen = room[need // 4:].random_(0, 16).view(n, 1)
    want = binding.themis_expert_sort(chosen.clone(), 16)
    for bad in (room, room[need // 4:], room[4:need // 4 + 4]):
        with pytest.raises(binding.ThemisError):
            binding.themis_expert_sort(chosen, 16, workspace=bad)
    beside = binding.themis_expert_sort(chosen, 16, workspace=room[:need // 4])
    assert torch.equal(beside.place, want.place) and torch.equal(beside.source, want.source)


def test_on_other_streams(layers):
    """An order made on one stream and used on another, and given up at once: its memory waits."""
    from paper_2110_04478_amd import binding
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    x, chosen = normal((4000, 512), 1), torch.randint(0, 16, (4000, 4), device="cuda", dtype=torch.int32)
    order = binding.themis_expert_sort(chosen, 16)
    want = binding.themis_expert_combine(binding.themis_expert_dispatch(x, order), order)
    torch.cuda.synchronize()
    for _ in range(5):
        order = binding.themis_expert_sort(chosen, 16)
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            got = binding.themis_expert_combine(binding.themis_expert_dispatch(x, order), order)
        del order
        torch.full((16000 * 3,), 1 << 30, dtype=torch.int32, device="cuda")   # (what takes freed memory)
        torch.cuda.synchronize()
        assert torch.equal(got, want)


def test_two_orders_at_once(layers):
    """Two captured graphs and eager calls between them: nothing is shared."""
    from paper_2110_04478_amd import binding
    made = []
    for seed in (1, 2):
        logits, x = normal((30000, 64), seed), normal((30000, 40), seed + 10)
        result = {}

        def run(logits=logits, x=x, result=result):
            weights, chosen = binding.themis_expert_gate(logits, 4)
            order = binding.themis_expert_sort(chosen, 64, 2000)
            rows = binding.themis_expert_dispatch(x, order)
            result["out"] = binding.themis_expert_combine(rows, order, weights)
            result["grad"] = binding.themis_expert_combine_grad(x, rows, order, weights)[1]
        run()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            run()
        made.append((graph, logits, x, result, run))
    for turn in range(3):
        for seed, (graph, logits, x, result, _) in enumerate(made):
            logits.copy_(normal(logits.shape, 100 + turn + seed))
            graph.replay()
        torch.cuda.synchronize()
        for graph, logits, x, result, run in made:
            held = {k: v.clone() for k, v in result.items()}
            mine = dict(result)
            run()
            torch.cuda.synchronize()
            assert all(torch.equal(held[k], result[k]) for k in held)
            result.clear()
            result.update(mine)


def test_a_captured_training_step(layers):
    """Forward and backward captured, replayed with other inputs and another call number.  (No eager
    graph of the leaves lives while it is captured: torch's engine ends the process then.)"""
    n, width, n_experts, k, capacity = 64, 32, 4, 2, 40
    leaves = [normal((width, n_experts), 2, 0.3).requires_grad_(), normal((n_experts, width, 48), 3, 0.2).requires_grad_(),
              normal((n_experts, 48, width), 4, 0.2).requires_grad_()]
    x, call = normal((n, width), 1), torch.zeros(1, dtype=torch.int64, device="cuda")

    def step(number):
        out, _, _ = the_layer(layers, x, *leaves, k, capacity, 0.3, 9, number)
        return out, torch.autograd.grad(out.square().sum(), leaves)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(call)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, grads = step(call)
    for turn in range(3):
        x.copy_(normal((n, width), 50 + turn))
        call.fill_(turn)
        graph.replay()
        torch.cuda.synchronize()
        want, expected = step(turn)
        for a, b in zip((out, *grads), (want, *expected)):
            # (matrix products may choose another order of sums in a graph)
            assert float((a - b).abs().max()) <= 64 * U * float(b.abs().max())
        del want, expected, a, b


def test_a_capture_beside_an_eager_graph_of_a_leaf_is_refused(layers, monkeypatch):
    """Of a leaf that these operators read themselves.  (The capture is only said to run: nothing of
    it is needed for the refusal.)"""
    from paper_2110_04478_amd import binding
    x, logits = normal((8, 16), 1).requires_grad_(), normal((8, 4), 2).requires_grad_()
    w = normal((8, 2), 3).requires_grad_()
    y = normal((16, 16), 4).requires_grad_()
    order = layers.sort(torch.zeros((8, 2), dtype=torch.int32, device="cuda"), 2)
    calls = [lambda: layers.gate(logits, 2)[0], lambda: layers.dispatch(x, order), lambda: layers.combine(y, order, w),
             lambda: layers.dropout(x, 0.5, 1, 2), lambda: layers.dropout(x.detach(), 0.5, 1, 2, add=x)]
    for call in calls:
        alive = call()
        with monkeypatch.context() as m:
            m.setattr(torch.cuda, "is_current_stream_capturing", lambda: True)
            with pytest.raises(binding.ThemisError):
                call()
        call().sum().backward()   # (eager: as ever)
        del alive
        with monkeypatch.context() as m:
            m.setattr(torch.cuda, "is_current_stream_capturing", lambda: True)
            call()
            with torch.no_grad():
                call()


def test_captures_on_two_streams_beside_each_other_are_refused(layers, monkeypatch):
    """While what the first one captured of a leaf lives.  (The captures are only said to run, as above.)"""
    from paper_2110_04478_amd import binding
    x = normal((8, 16), 1).requires_grad_()
    torch.cuda.synchronize()
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: True)
    one, other = torch.cuda.Stream(), torch.cuda.Stream()
    assert one.cuda_stream != other.cuda_stream
    with torch.cuda.stream(one):
        alive = layers.dropout(x, 0.5, 1, 2)
        layers.dropout(x, 0.5, 1, 3)   # (the same stream: as ever)
    with torch.cuda.stream(other):
        with pytest.raises(binding.ThemisError, match="another stream's graph of the same leaf"):
            layers.dropout(x, 0.5, 1, 2)
        del alive
        layers.dropout(x, 0.5, 1, 2)
    torch.cuda.synchronize()
