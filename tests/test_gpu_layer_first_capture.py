"""The first calls that a process makes of a decoder layer's operators are captured into a graph."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

CODE = """
import torch
from paper_2507_07990_b200 import cache, layer, prefix
gen = torch.Generator().manual_seed(1)
normal = lambda *shape: torch.randn(shape, generator=gen).bfloat16().cuda()
x, pool, own = normal(40, 512), cache.empty_cache(1, 300, 2, 128), cache.empty_cache(2, 40, 2, 128)
for c in (pool, own):
    c.k.copy_(normal(*c.k.shape)), c.v.copy_(normal(*c.v.shape))
ints = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")
offsets, lengths, held = torch.tensor([0, 25, 40], device="cuda"), ints(300), ints(25, 33)
w = layer.QuantRows(torch.randint(-127, 128, (768, 512), dtype=torch.int8, generator=gen).cuda(), torch.rand(768, generator=gen).cuda() / 3000)
norm = layer.NormPlan(512, torch.bfloat16, 40, pre_norm=torch.ones(512, device="cuda"), quantize=True)
up = layer.MatmulPlan(w, torch.bfloat16, 40)
act = layer.QuantizePlan(384, torch.bfloat16, 40, gated=True)
plans = [prefix.PrefixPlan(pool, 4, own, 40, fine=fine) for fine in (False, True)]
def call():
    rows = norm.run(x, x)
    a = act.run(up.run(rows.rows))
    return [rows.sum, rows.rows.q, a.q, a.scale] + [p.run(x.view(40, 4, 128), offsets, lengths, held).out for p in plans]
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    out = call()
graph.replay()
torch.cuda.synchronize()
got = [t.clone() for t in out]
[t.zero_() for t in out]
assert all(torch.equal(g, w) for g, w in zip(got, call()))
assert all(bool(g.any()) for g in got)
graph.reset()
print("all alike")
"""


def test_first_calls_in_a_graph():
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    out = subprocess.run([sys.executable, "-c", CODE], cwd=root, capture_output=True, text=True, timeout=120)
    assert out.returncode == 0 and "all alike" in out.stdout, out.stderr[-2000:]
