"""How the gradient operators lay out their launches, without a GPU: the library's
hipLaunchKernel is one that writes down kernel, grid and workgroup, and refuses what HIP refuses
(2^32 threads or more along one direction of a grid, more than 65,535 workgroups along another).
The arrays exist as sizes only."""
import json
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

RECORDER = r"""
#define _GNU_SOURCE
#include <dlfcn.h>
#include <stdint.h>
#include <stdio.h>
typedef struct { uint32_t x, y, z; } dim3_t;
int hipLaunchKernel(const void* f, dim3_t g, dim3_t b, void** args, size_t lds, void* stream) {
  Dl_info at;
  const int refused = (uint64_t)g.x * b.x >> 32 || g.y > 65535u || g.z != 1 || lds > 163840u || !g.x || !g.y ||
                      b.x > 1024 || b.y != 1 || b.z != 1;
  (void)args; (void)stream;
  printf("%s %u %u %u %d\n", dladdr(f, &at) && at.dli_sname ? at.dli_sname : "?", g.x, g.y, b.x, refused);
  fflush(stdout);
  return refused ? 9 : 0;
}
"""

CALLER = r"""
import ctypes, json, sys
ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)
from paper_2110_04478_amd import binding
L, fake, big = binding.lib(), 1 << 20, 1 << 62
def rows(kind, n, width, step=None):
    return binding._Rows(fake, kind, max(1, n), 0, width if step is None else step)
for call in json.loads(sys.argv[2]):
    name, n, width, vocab, kind, to = call[:6]
    print("call", flush=True)
    if name == "lookup":
        st = L.themis_embedding_lookup(rows(kind, vocab, width), vocab, width, rows(4, n, 1), n, 1.0, rows(to, n, width), None)
    elif name == "grad":
        st = L.themis_embedding_grad(rows(kind, n, width), width, rows(4, n, 1), n, 1.0, -1, call[6],
                                     rows(to, vocab, width, call[7] if len(call) > 7 else None), vocab, fake, big, None)
    else:
        parts = (binding._Gradient * n)(*[binding._Gradient(fake, fake, i, kind, kind, 1, width, width, 1, width, 1) for i in range(n)])
        plan = binding._GradientPlan()
        st = L.themis_gradient_plan(parts, n, n, plan, None, 0)
        plan.image = fake
        if st == 0:
            st = L.themis_gradient_norm(plan, fake, fake, fake, big, None) or L.themis_gradient_clip(plan, 1.0, fake, fake, fake, big, None)
    print("status", st, flush=True)
"""


@pytest.fixture(scope="module")
def launches(tmp_path_factory):
    from paper_2110_04478_amd.csrc.build import ensure_built
    ensure_built()
    d = tmp_path_factory.mktemp("recorder")
    (d / "r.c").write_text(RECORDER)
    (d / "call.py").write_text(CALLER)
    subprocess.run(["gcc", "-O1", "-shared", "-fPIC", "-o", str(d / "r.so"), str(d / "r.c"), "-ldl"], check=True)

    def run(calls):
        out = subprocess.run([sys.executable, str(d / "call.py"), str(d / "r.so"), json.dumps(calls)],
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
        return got
    return run


MOST = (1 << 31) - 1


def test_every_accepted_size_is_launched(launches):
    """At the ends of what is accepted no grid is one that HIP refuses, and what is not accepted
    launches nothing."""
    calls = [("lookup", n, w, v, 0, 1) for n in (1, 1000, MOST) for w in (1, 9, 2049, 1 << 20, MOST) for v in (0, 1, MOST)]
    calls += [("grad", n, w, v, 1, t, a) for n in (1, 4096, 4097, 200000, MOST) for w in (1, 65, 513, 1 << 16, MOST)
              for v in (1, 1000, MOST) for t in (0, 1) for a in (0, 1)]
    calls += [("grad", n, w, v, 1, 0, 0, w + 3) for n in (0, 1, 5000) for w in (1, 513, 1 << 27) for v in (1, 1000, MOST)]
    calls += [("norm", n, w, 0, k, 0) for n, w in ((0, 1), (1, 1), (1, MOST), (3, 1 << 38), (5000, 7), (40, 1 << 34)) for k in (0, 1)]
    for call, (status, found) in zip(calls, launches(calls)):
        assert status in (0, -2), (call, status, found)
        assert not any(l[4] for l in found), (call, found)
        assert bool(found) == (status == 0), (call, status, found)
        if call[1] <= 200000 and call[2] <= 1 << 16:
            assert status == 0, call


@pytest.mark.parametrize("n,kernels", [(1, ["few_tokens"]), (4096, ["few_tokens"]),
                                       (4097, ["sort_count", "sort_move"] * 2 + ["tile_sum", "tile_join"])])
def test_launches_of_a_gradient(launches, n, kernels):
    (status, found), = launches([("grad", n, 1024, 32768, 1, 0, 1)])
    assert status == 0 and len(found) == len(kernels) and all(k in l[0] for k, l in zip(kernels, found)), found


def test_zeros_of_large_tables_come_first(launches):
    small, large, dense, half = launches([("grad", 10, 64, 1000, 1, 1, 0), ("grad", 10, 4096, 131072, 1, 1, 0),
                                          ("grad", 16384, 4096, 131072, 1, 1, 0), ("grad", 65536, 4096, 131072, 1, 1, 0)])
    assert len(small[1]) == 1 and small[1][0][1] == 10 + -(-1000 // 64)
    assert "clear" in large[1][0][0] and large[1][0][1] * 4096 == 2 * 4096 * 131072 and large[1][1][1] == 10
    assert "clear" in dense[1][0][0] and not any("clear" in l[0] for l in half[1])
