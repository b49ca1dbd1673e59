"""The limit on a kernel's dynamic shared memory, raised from several host threads."""
import subprocess
import threading
from pathlib import Path

import pytest
import torch

from paper_2407_15452_b200 import binding as B
from paper_2407_15452_b200 import build

HERE = Path(__file__).resolve().parent


def test_two_threads_that_ask_for_different_sizes(tmp_path):
    exe = tmp_path / "limit"
    subprocess.run(["nvcc", *build.NVCC_FLAGS, str(HERE / "shared_memory_limit.cu"), "-o", str(exe)], check=True)
    for _ in range(3):
        r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=60)
        assert r.returncode == 0, r.stdout + r.stderr


@pytest.mark.gpu
def test_first_calls_of_several_lengths_at_once():
    lengths = [17, 33, 49, 65, 81, 97, 113, 128]
    qkv = {n: [torch.randn((2, n, 2, 64), device="cuda", dtype=torch.bfloat16) for _ in range(3)] for n in lengths}
    got, start = {}, threading.Barrier(len(lengths))

    def call(n):
        start.wait()
        with torch.cuda.stream(torch.cuda.Stream()):
            out, lse = B.gs_attention_forward(*qkv[n])
            got[n] = (out, *B.gs_attention_backward(out, *qkv[n], out, lse))

    torch.cuda.synchronize()
    threads = [threading.Thread(target=call, args=(n,)) for n in lengths]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert sorted(got) == lengths                          # no call failed
    for n in lengths:
        out, lse = B.gs_attention_forward(*qkv[n])
        again = (out, *B.gs_attention_backward(out, *qkv[n], out, lse))
        assert all(torch.equal(a, b) for a, b in zip(got[n], again))
