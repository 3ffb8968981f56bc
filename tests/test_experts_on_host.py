"""The host side of the expert layer's operators and of dropout, without a GPU: what is refused
before anything is launched, and what the launches look like (recorded in the place of HIP's own).
The pointers are numbers that nobody dereferences."""
import ctypes
import json
import os
import subprocess
import sys

import pytest
import torch

from test_gradient_launches import RECORDER

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
F32, BF16, F16, I32, I64 = range(5)
FAKE = 0x100000
MOST = (1 << 31) - 1


@pytest.fixture(scope="module")
def binding():
    from paper_2110_04478_amd.csrc.build import ensure_built
    ensure_built()
    from paper_2110_04478_amd import binding
    return binding


def rows(binding, type_, step=8, inner=1 << 20, outer_stride=0, data=FAKE):
    return binding._Rows(data, type_, inner, outer_stride, step)


def order(binding, n=5, k=2, n_experts=4, capacity=0, place=FAKE, counts=FAKE, starts=FAKE, source=FAKE):
    return binding._ExpertOrder(n, k, n_experts, capacity, place, counts, starts, source)


OVERLAPPING = (dict(step=7), dict(step=0), dict(step=-7), dict(inner=2, outer_stride=15),
               dict(inner=2, outer_stride=0), dict(inner=3, outer_stride=8))


def test_gate_refusals(binding):
    L = binding.lib()

    def call(logits=None, n_experts=16, n=5, k=8, weights=None, experts=None):
        return L.themis_expert_gate(logits or rows(binding, BF16, 16), n_experts, n, k, 1,
                                    weights or rows(binding, F32), experts or rows(binding, I32), None)

    assert call(n=0) == 0 and call(k=0) == 0 and call(k=17) == -1 and call(n_experts=0, k=1) == -1
    assert call(logits=rows(binding, I32)) == -1 and call(weights=rows(binding, I64)) == -1
    assert call(experts=rows(binding, F32)) == -1 and call(experts=rows(binding, 5)) == -1
    assert call(logits=rows(binding, F32, data=FAKE + 2)) == -1 and call(experts=rows(binding, I64, data=FAKE + 4)) == -1
    assert call(weights=rows(binding, BF16, data=0)) == -1 and call(logits=rows(binding, F32, inner=0)) == -1
    assert call(n=1 << 31) == -2 and call(n_experts=1025) == -2 and call(n_experts=1000, k=65) == -2
    for bad in OVERLAPPING:
        assert call(weights=rows(binding, F32, **bad)) == -1 and call(experts=rows(binding, I64, **bad)) == -1, bad
    assert L.themis_expert_gate(None, 16, 5, 8, 1, rows(binding, F32), rows(binding, I32), None) == -1


def test_gate_gradient_refusals(binding):
    L = binding.lib()

    def call(g=None, logits=None, n_experts=8, experts=None, n=5, k=3, out=None):
        return L.themis_expert_gate_grad(g or rows(binding, F32), logits or rows(binding, BF16), n_experts,
                                         experts or rows(binding, I32), n, k, 1, out or rows(binding, F16), None)

    assert call(n=0) == 0 and call(n_experts=0) == 0
    assert call(g=rows(binding, I32)) == -1 and call(logits=rows(binding, I32)) == -1
    assert call(experts=rows(binding, F32)) == -1 and call(out=rows(binding, I32)) == -1
    assert call(out=rows(binding, F32, data=FAKE + 2)) == -1 and call(g=rows(binding, F32, data=0)) == -1
    assert call(n=1 << 31) == -2 and call(n_experts=1025) == -2 and call(k=65) == -2
    for bad in OVERLAPPING:
        assert call(out=rows(binding, F32, **bad)) == -1, bad


def test_sort_refusals(binding):
    L = binding.lib()
    size = L.themis_expert_sort_workspace_bytes

    def call(experts=None, work=FAKE, work_bytes=1 << 40, **kw):
        return L.themis_expert_sort(experts or rows(binding, I64), order(binding, **kw), work, work_bytes, None)

    assert call(n_experts=0) == -1 and call(n_experts=1025) == -2
    assert call(n=1 << 31) == -2 and call(n=1 << 20, k=1 << 12) == -2 and call(k=1 << 40) == -2
    assert call(capacity=1 << 30) == -2 and call(capacity=1 << 62) == -2
    assert call(experts=rows(binding, F32)) == -1 and call(experts=rows(binding, I64, data=FAKE + 4)) == -1
    for name in ("place", "counts", "starts", "source"):
        assert call(**{name: 0}) == -1 and call(**{name: FAKE + 2}) == -1
    assert L.themis_expert_sort(rows(binding, I64), None, FAKE, 1 << 40, None) == -1
    assert L.themis_expert_sort(None, order(binding), FAKE, 1 << 40, None) == -1
    assert size(0, 4, 5) == size(100, 2, 8) == 0
    assert size(1 << 31, 1, 8) == size(1 << 20, 1 << 12, 8) == size(1 << 63, 1 << 63, 8) == 0
    assert size(100000, 8, 0) == size(100000, 8, 1025) == 0
    need = size(100000, 8, 64)
    assert need > 0 and need % 256 == 0
    big = dict(n=100000, k=8, n_experts=64)
    assert call(work=None, **big) == -4 and call(work_bytes=need - 1, **big) == -4 and call(work=FAKE + 8, **big) == -4


def test_row_refusals(binding):
    L = binding.lib()

    def dispatch(o=None, x=None, width=8, out=None):
        return L.themis_expert_dispatch(o or order(binding), x or rows(binding, F32), width, out or rows(binding, BF16), None)

    def combine(o=None, y=None, width=8, weights=None, out=None, add=0):
        return L.themis_expert_combine(o or order(binding), y or rows(binding, F32), width, weights, add,
                                       out or rows(binding, BF16), None)

    for call in (dispatch, combine):
        assert call(order(binding, n=0)) == 0 and call(width=0) == 0
        assert call(order(binding, n_experts=0)) == -1 and call(order(binding, place=0)) == -1
        assert call(order(binding, source=FAKE + 1)) == -1 and call(order(binding, n=1 << 30, k=2)) == -2
        assert call(width=(1 << 25) + 1) == -2
        assert call(out=rows(binding, I32)) == -1 and call(out=rows(binding, F32, data=FAKE + 2)) == -1
        for bad in OVERLAPPING:
            assert call(out=rows(binding, F32, **bad)) == -1, (call, bad)
    assert dispatch(order(binding, k=0)) == 0 and dispatch(x=rows(binding, I64)) == -1
    assert combine(order(binding, k=0), add=1) == 0 and combine(y=rows(binding, I32)) == -1
    assert combine(weights=rows(binding, I32)) == -1 and combine(weights=rows(binding, F32, data=FAKE + 1)) == -1
    assert L.themis_expert_dispatch(None, rows(binding, F32), 8, rows(binding, F32), None) == -1

    def grad(o=None, g=True, width=8, y=True, w=True, rows_=True, products=True):
        pick = [rows(binding, BF16) if x is True else x for x in (g, y, w, rows_, products)]
        return L.themis_expert_combine_grad(o or order(binding), pick[0], width, *pick[1:], None)

    assert grad(rows_=None, products=None) == 0 and grad(order(binding, n=0)) == 0
    assert grad(g=None) == -1 and grad(w=None) == -1 and grad(y=None) == -1
    assert grad(rows_=rows(binding, F32)) == -1 and grad(products=rows(binding, I32)) == -1   # another type than y's
    assert grad(g=rows(binding, I32)) == -1 and grad(w=rows(binding, I64)) == -1 and grad(width=(1 << 25) + 1) == -2
    assert grad(order(binding, n_experts=1025)) == -2
    for bad in OVERLAPPING:
        assert grad(rows_=rows(binding, BF16, **bad)) == -1, bad
    assert grad(products=rows(binding, F32, 1)) == -1


def test_dropout_refusals(binding):
    L = binding.lib()

    def call(x=None, n=5, width=8, p=0.1, at=None, add=None, out=None):
        return L.themis_dropout(x or rows(binding, F32), n, width, p, 1, 2, at, add, out or rows(binding, BF16), None)

    assert call(n=0) == 0 and call(width=0) == 0
    for bad in (-0.1, 1.1, float("nan"), float("inf")):
        assert call(p=bad) == -1
    assert call(x=rows(binding, I32)) == -1 and call(out=rows(binding, I64)) == -1 and call(at=FAKE + 4) == -1
    assert call(add=rows(binding, F32)) == -1 and call(add=rows(binding, BF16, data=FAKE + 1)) == -1
    assert call(n=1 << 31) == -2 and call(width=(1 << 25) + 1) == -2
    for bad in OVERLAPPING:
        assert call(out=rows(binding, F32, **bad)) == -1, bad


def test_tensors_on_the_host_are_refused(binding):
    x, e = torch.ones(4, 8), torch.zeros(4, 2, dtype=torch.int32)
    for call in (lambda: binding.themis_expert_gate(x, 2), lambda: binding.themis_expert_gate_grad(x[:, :2], x, e),
                 lambda: binding.themis_expert_sort(e, 3), lambda: binding.themis_dropout(x, 0.1, 1, 2)):
        with pytest.raises(binding.ThemisError):
            call()


def test_a_capture_beside_an_eager_graph_says_so(binding, monkeypatch):
    """Not as a wrong shape does: what has to change is the program's order, not the call."""
    from paper_2110_04478_amd import layers

    class Same(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x):
            return x.clone()

        @staticmethod
        def backward(ctx, grad):
            return grad

    x = torch.ones(3, requires_grad=True)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    alive = layers._apply(Same, (x,), x)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: True)
    with pytest.raises(binding.ThemisError, match="invalid argument.*eager graph of the same leaf") as e:
        layers._apply(Same, (x,), x)
    assert e.value.status == binding.INVALID_ARGUMENT and alive.requires_grad
    assert str(binding.ThemisError(-1)) == "themis: invalid argument (-1)"


CALLER = r"""
import ctypes, json, sys
ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)
from paper_2110_04478_amd import binding
L, fake, big = binding.lib(), 1 << 20, 1 << 62
def rows(kind, n, width):
    return binding._Rows(fake, kind, max(1, n), 0, width)
for call in json.loads(sys.argv[2]):
    name, n, k, experts, capacity, width = call
    o = binding._ExpertOrder(n, k, experts, capacity, fake, fake, fake, fake)
    slots = experts * capacity if capacity else n * k
    print("call", flush=True)
    if name == "gate":
        st = (L.themis_expert_gate(rows(1, n, experts), experts, n, k, 1, rows(0, n, k), rows(3, n, k), None) or
              L.themis_expert_gate_grad(rows(0, n, k), rows(1, n, experts), experts, rows(3, n, k), n, k, 1, rows(1, n, experts), None))
    elif name == "sort":
        st = L.themis_expert_sort(rows(3, n, k), o, fake, big, None)
    elif name == "rows":
        st = (L.themis_expert_dispatch(o, rows(1, n, width), width, rows(0, slots, width), None) or
              L.themis_expert_combine(o, rows(0, slots, width), width, rows(0, n, k), 0, rows(1, n, width), None) or
              L.themis_expert_combine_grad(o, rows(1, n, width), width, rows(1, slots, width), rows(0, n, k),
                                           rows(1, slots, width), rows(0, n, k), None))
    else:
        st = L.themis_dropout(rows(1, n, width), n, width, 0.1, 1, 2, None, None, rows(0, n, width), None)
    print("status", st, flush=True)
"""


def test_every_accepted_size_is_launched(binding, tmp_path):
    """At the ends of what is accepted no grid is one that HIP refuses, and what is not accepted
    launches nothing."""
    (tmp_path / "r.c").write_text(RECORDER)
    (tmp_path / "call.py").write_text(CALLER)
    subprocess.run(["gcc", "-O1", "-shared", "-fPIC", "-o", str(tmp_path / "r.so"), str(tmp_path / "r.c"), "-ldl"], check=True)
    calls = [("gate", n, k, e, 0, 0) for n in (1, 1000, MOST) for e in (1, 9, 65, 513, 1024) for k in (1, min(e, 64))]
    calls += [("sort", n, k, e, c, 0) for n in (0, 1, 40960, 40961, 1 << 20, MOST) for k in (1, 8) for e in (1, 1024)
              for c in (0, 5, 1 << 21)]
    calls += [("rows", n, k, e, c, w) for n in (1, 1000, MOST) for k in (1, 8) for e in (1, 1024) for c in (0, 5)
              for w in (1, 9, 2049, 1 << 20, 1 << 25)]
    calls += [("dropout", n, 1, 1, 0, w) for n in (1, 1000, MOST) for w in (1, 9, 2049, 1 << 20, 1 << 25)]
    out = subprocess.run([sys.executable, str(tmp_path / "call.py"), str(tmp_path / "r.so"), json.dumps(calls)],
                         env=dict(os.environ, PYTHONPATH=ROOT), check=True, capture_output=True, text=True).stdout
    got = []
    for line in out.splitlines():
        w = line.split()
        if w[0] == "call":
            got.append([None, []])
        elif w[0] == "status":
            got[-1][0] = int(w[1])
        else:
            got[-1][1].append((w[0], *map(int, w[1:])))
    assert len(got) == len(calls)
    for call, (status, found) in zip(calls, got):
        assert status in (0, -2), (call, status, found)
        assert not any(l[4] for l in found), (call, found)
        pairs, slots = call[1] * call[2], call[3] * call[4] if call[4] else call[1] * call[2]
        assert (status == 0) == (pairs <= MOST and slots <= MOST or call[0] in ("gate", "dropout")), (call, status)
        assert bool(found) == (status == 0), (call, status, found)


def test_lists_that_one_workgroup_sorts(binding, tmp_path):
    """Up to 8,192 pairs one launch without a workspace, beyond them two."""
    (tmp_path / "r.c").write_text(RECORDER)
    (tmp_path / "call.py").write_text(CALLER)
    subprocess.run(["gcc", "-O1", "-shared", "-fPIC", "-o", str(tmp_path / "r.so"), str(tmp_path / "r.c"), "-ldl"], check=True)
    calls = [("sort", n, k, e, c, 0) for n, k in ((8191, 1), (8192, 1), (4096, 2), (8193, 1), (2731, 3)) for e in (1, 61, 1024)
             for c in (0, 7)]
    out = subprocess.run([sys.executable, str(tmp_path / "call.py"), str(tmp_path / "r.so"), json.dumps(calls)],
                         env=dict(os.environ, PYTHONPATH=ROOT), check=True, capture_output=True, text=True).stdout
    got = [part.splitlines() for part in out.split("call\n")[1:]]
    assert len(got) == len(calls)
    size = binding.lib().themis_expert_sort_workspace_bytes
    for (_, n, k, e, _, _), lines in zip(calls, got):
        assert lines[-1] == "status 0" and len(lines) == (2 if n * k <= 8192 else 3), (n, k, e, lines)
        assert (size(n, k, e) > 0) == (n * k > 8192)
