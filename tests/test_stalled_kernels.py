"""Where the count of waits that ran out inside attention kernels lives."""
import os
import subprocess
import sys
from pathlib import Path

import pytest
pytestmark = pytest.mark.gpu
ROOT = Path(__file__).resolve().parent.parent


CAPTURED_FIRST = """
import torch
from paper_2407_15452_b200 import binding as B
for n in (40, 300):                                          # one kernel of each kind that counts
    q, k, v = (torch.randn((2, n, 2, 64), device="cuda", dtype=torch.bfloat16) for _ in range(3))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, lse = B.gs_attention_forward(q, k, v)
        grads = B.gs_attention_backward(q, q, k, v, out, lse)
    B.gs_release_workspace()                                 # what the graph has recorded stays valid
    graph.replay()
    torch.cuda.synchronize()
    want, lse = B.gs_attention_forward(q, k, v)
    again = B.gs_attention_backward(q, q, k, v, want, lse)
    assert torch.equal(out, want) and all(torch.equal(a, b) for a, b in zip(grads, again))
assert B.gs_stalled_kernels() == 0
print("replayed")
"""


def test_the_first_call_of_a_process_may_be_captured():
    r = subprocess.run([sys.executable, "-c", CAPTURED_FIRST], cwd=ROOT, capture_output=True, text=True, timeout=300,
                       env={**os.environ, "PYTHONPATH": str(ROOT)})
    assert r.returncode == 0 and "replayed" in r.stdout, r.stdout + r.stderr
