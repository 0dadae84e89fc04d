"""Calls of positions, draws and shared blocks whose first one in a process is
captured into a graph, against the same calls made at once."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu
HERE = os.path.dirname(os.path.abspath(__file__))

SET = """
import torch
import paper_2607_22578_gb300 as hs
i32 = dict(dtype=torch.int32, device="cuda")
g = torch.Generator(device="cuda").manual_seed(3)
"""

SAMPLE = """
l = torch.randn((40, 20000), generator=g, device="cuda").to(torch.bfloat16)
u = torch.rand(40, generator=g, device="cuda")
call = lambda: hs.hs_sample(l, u) + hs.hs_sample(l[:2], u[:2].clone())
"""

ROTARY = """
r, pos = hs.Rotary(64), torch.arange(40, **i32)
x = torch.randn((40, 3, 64), generator=g, device="cuda").to(torch.float16)
call = lambda: (hs.hs_rotary(x, r, positions=pos),)
"""

# n blocks; 4 requests of 0 .. 3 * 70 tokens in blocks of their own
PAGES = """
n = %d
lens, table = torch.arange(4, **i32) * 70, torch.arange(4 * 20, **i32).view(4, 20) + n - 100
shared, pool, cursor = torch.zeros(n, **i32), torch.arange(n, **i32), torch.tensor([0, n - 80]).cuda()
"""

FORK = PAGES + """
def call():
    t, s = table.clone(), shared.clone()
    src, dst = torch.full((1,), 2, **i32), torch.zeros(1, **i32)
    return hs.hs_kv_fork(src, dst, lens, t, s, pool, cursor, 16) + (t, s)
"""

RELEASE = PAGES + """
call = lambda: hs.hs_kv_release_shared(lens, table, shared, pool.clone(), cursor, 16)
"""

COMPACT = PAGES + """
call = lambda: hs.hs_kv_compact(lens, table, shared, 16)
"""

BOTH = """
side = torch.cuda.Stream()
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph, stream=side):
    out = call()
graph.replay()
torch.cuda.synchronize()
got = [x.clone() for x in out]
assert all(torch.equal(a, b) for a, b in zip(got, call()))
graph.replay()
torch.cuda.synchronize()
assert all(torch.equal(a, b) for a, b in zip(got, out))
hs.hs_get_device_error()
"""


@pytest.mark.parametrize("code", [SAMPLE, ROTARY, FORK % 200, RELEASE % 200, RELEASE % 50000, COMPACT % 200,
                                  COMPACT % 200000, COMPACT % 800000],
                         ids=["sample", "rotary", "fork", "release", "release_many", "compact", "compact_many",
                              "compact_most"])
def test_first_call_captured(code):
    begin = "import sys\nsys.path.insert(0, %r)\n" % os.path.dirname(HERE)
    r = subprocess.run([sys.executable, "-c", begin + SET + code + BOTH], capture_output=True, text=True,
                       timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]
