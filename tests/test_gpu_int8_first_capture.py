"""mw_quantise_rows needs no handle, so nothing has loaded its kernels when it is called first: that call may be one that is captured."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

CODE = """
import torch
from paper_2605_22428_b200 import binding as mw
cases = []
for dtype, T, H, act in ((torch.bfloat16, 4, 64, 0), (torch.float32, 300, 4096, 0), (torch.float16, 5, 9216, 1), (torch.float32, 2, 20000, 2)):
    x = torch.randn(T, H * (2 if act else 1), device="cuda").to(dtype)
    cases.append((x, T, H, torch.zeros(T, H, dtype=torch.int8, device="cuda"), torch.zeros(T, device="cuda"), act))
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    for c in cases:
        mw.mw_quantise_rows(*c)
graph.replay()
torch.cuda.synchronize()
for x, T, H, q, scale, act in cases:
    q2, scale2 = torch.zeros_like(q), torch.zeros_like(scale)
    mw.mw_quantise_rows(x, T, H, q2, scale2, act)
    torch.cuda.synchronize()
    assert torch.equal(q, q2) and torch.equal(scale, scale2) and bool(q.any())
print("the same")
"""


def test_the_first_call_may_be_captured():
    """In a process of its own, without a handle."""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    done = subprocess.run([sys.executable, "-c", CODE], cwd=root, env=dict(os.environ, PYTHONPATH=root), capture_output=True, text=True, timeout=300)
    assert done.returncode == 0 and "the same" in done.stdout, done.stderr[-2000:]
