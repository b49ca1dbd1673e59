"""What happens when a wait inside an attention kernel runs out, and where the count of such waits lives."""
import os
import subprocess
import sys
from pathlib import Path

import pytest
import torch

from paper_2407_15452_b200 import binding as B
from paper_2407_15452_b200.attention import attention

pytestmark = pytest.mark.gpu
ROOT = Path(__file__).resolve().parent.parent


def test_a_wait_that_runs_out_is_reported_by_the_next_call():
    q, k, v = (torch.randn((2, 30, 2, 32), device="cuda", dtype=torch.bfloat16, requires_grad=True) for _ in range(3))
    out = attention(q, k, v)
    want = out.detach().clone()
    assert B.gs_stalled_kernels() == 0
    B.gs_stall_drill()                                      # nothing ever arrives at this block's barrier
    torch.cuda.synchronize()
    try:
        with pytest.raises(B.GsError, match="gave up a wait") as e:
            attention(q, k, v)
        assert e.value.status == -4
        with pytest.raises(B.GsError, match="gave up a wait"):
            out.sum().backward()
        assert B.gs_stalled_kernels() == 1                  # reading it does not clear it
        B.gs_release_workspace()
        assert B.gs_stalled_kernels() == 1
    finally:
        assert B.gs_stalled_kernels(clear=True) == 1
    assert B.gs_stalled_kernels() == 0
    assert torch.equal(attention(q, k, v), want)            # the device is none the worse for it
    attention(q, k, v).sum().backward()


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
