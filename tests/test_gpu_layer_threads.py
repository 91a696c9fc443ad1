"""First calls of a fresh process from several threads at once: each gets the product that one thread gets."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

CODE = """
import threading, torch
from paper_2507_07990_b200 import layer
x, w = (layer.QuantRows(torch.randint(-9, 9, (n, 4096), dtype=torch.int8, device="cuda"), torch.ones(n, device="cuda")) for n in (24, 512))
want = x.q.double() @ w.q.double().t()
plans = [layer.MatmulPlan(w, torch.float32, 24) for _ in range(8)]
torch.cuda.synchronize()
start, got = threading.Barrier(8), [None] * 8
def call(i):
    with torch.cuda.stream(torch.cuda.Stream()):
        start.wait()
        got[i] = plans[i].run(x)
threads = [threading.Thread(target=call, args=(i,)) for i in range(8)]
[t.start() for t in threads]
[t.join() for t in threads]
torch.cuda.synchronize()
assert all(torch.equal(g.double(), want) for g in got)
print("eight alike")
"""


def test_first_calls_at_once():
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    out = subprocess.run([sys.executable, "-c", CODE], cwd=root, capture_output=True, text=True, timeout=120)
    assert out.returncode == 0 and "eight alike" in out.stdout, out.stderr[-2000:]
